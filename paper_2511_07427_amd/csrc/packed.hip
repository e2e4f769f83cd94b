// Packed caches: quantising rows as they are written, reading them back (dynakv_packed_write, dynakv_packed_read).
//
// A block of 32 values x shares the scale 2^e, e the smallest for which max|x| <= qmax 2^e (qmax = 127 or 7), within a range in
// which every code times 2^e is a finite value of the type, held exactly; codes are rint(x 2^-e).  2^e multiplies without
// rounding, so the codes are those of exact arithmetic, and reading back rounds nothing.  Both directions are bound by
// memory: a row is 128 elements and 132 or 68 bytes.  16 lanes hold a row, 8 values each, so that a lane's loads and stores of 16-bit values
// are 16 bytes wide and the rows of a wavefront lie one after the other; a block is one quad of lanes, and its maximum crosses them in two steps.
// 256 units of 4096 float16 tokens to 4 bits: writing 126 us (5.4 TB/s), reading 141 (4.9); reading 112 of 8192 bfloat16
// tokens from 8 bits 125 us (5.7).  Rows at scattered positions cost more than their bytes: a row's codes and scales lie in four places, of each of which
// memory gives 128 bytes (32768 rows of 136 bytes: 15.8 MiB read for 4.3).
#include "operators.hpp"

namespace dynakv {

namespace {

struct Range { int qbits, lo, hi; };                // qmax = 2^qbits - 1
__host__ __device__ constexpr Range scale_range(int dtype, int bits) {
  // hi: qmax 2^hi stays below 2^16 (float16) or 2^128; lo: no value of float16 is finer than 2^-24, no normal float32 or
  // bfloat16 than 2^-126
  return Range{bits - 1, dtype == DYNAKV_F16 ? -24 : -126, (dtype == DYNAKV_F16 ? 16 : 128) - (bits - 1)};
}

// Codes of the 8 values of a lane and the scale byte of its quad's block.
template <int DT, int BITS>
__device__ __forceinline__ uint32_t quantise(const float (&x)[8], int (&c)[8]) {
  constexpr Range r = scale_range(DT, BITS);
  constexpr int qmax = (1 << r.qbits) - 1;
  uint32_t m = 0;                                    // bits of |x| order like the values; a NaN's are the largest
#pragma unroll
  for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(x[e]) & 0x7FFFFFFFu);
  m = max(m, (uint32_t)dpp_or<kDppXor1>(0, (int)m));
  m = max(m, (uint32_t)dpp_or<kDppXor2>(0, (int)m));
  // max|x| = f 2^k, 1 <= f < 2: 2^(k - qbits + 1) is enough if f <= qmax / 2^(qbits - 1), a bound on the mantissa's bits
  constexpr uint32_t most = (uint32_t)((qmax << (24 - r.qbits)) & 0x7FFFFF);
  int e = (int)(m >> 23) - 127 - (r.qbits - 1) + ((m & 0x7FFFFFu) > most ? 1 : 0);
  e = min(max(e, r.lo), r.hi);
  const bool finite = m < 0x7F800000u;
  const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int q = (int)rintf(x[k] * inv);
    c[k] = finite ? min(max(q, -qmax), qmax) : 0;
  }
  return finite ? (uint32_t)(e + 127) : 255u;
}

template <int BITS>
__device__ __forceinline__ void store_codes(uint8_t* row, int lane, const int (&c)[8]) {
  if constexpr (BITS == 8) {
    uint2 w = {0, 0};
#pragma unroll
    for (int k = 0; k < 4; ++k) { w.x |= (uint32_t)(c[k] & 255) << (8 * k); w.y |= (uint32_t)(c[4 + k] & 255) << (8 * k); }
    *(uint2*)(row + 8 * lane) = w;
  } else {
    uint32_t w = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) w |= (uint32_t)(c[k] & 15) << (4 * k);
    *(uint32_t*)(row + 4 * lane) = w;
  }
}

template <int BITS>
__device__ __forceinline__ void load_values(const uint8_t* row, int lane, float scale, float (&x)[8]) {
  if constexpr (BITS == 8) {
    const uint2 w = *(const uint2*)(row + 8 * lane);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      x[k] = (float)((int)(w.x << (24 - 8 * k)) >> 24) * scale;
      x[4 + k] = (float)((int)(w.y << (24 - 8 * k)) >> 24) * scale;
    }
  } else {
    const uint32_t w = *(const uint32_t*)(row + 4 * lane);
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = (float)((int)(w << (28 - 4 * k)) >> 28) * scale;
  }
}

typedef uint32_t u4 __attribute__((ext_vector_type(4)));

// Elements i .. i + 7 of an array of values.
template <int DT, bool STREAM>
__device__ __forceinline__ void load_row8(const void* base, size_t i, float (&x)[8]) {
  if constexpr (DT == DYNAKV_F32) {
    const f4 a = get<STREAM>((const f4*)((const float*)base + i)), b = get<STREAM>((const f4*)((const float*)base + i + 4));
#pragma unroll
    for (int e = 0; e < 4; ++e) { x[e] = a[e]; x[4 + e] = b[e]; }
  } else {
    const u4 w = get<STREAM>((const u4*)((const uint16_t*)base + i));
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint16_t h = (uint16_t)(w[e >> 1] >> ((e & 1) * 16));
      x[e] = DT == DYNAKV_F16 ? f16_to_float(h) : bf16_to_float(h);
    }
  }
}

template <int DT, bool STREAM>
__device__ __forceinline__ void store8(void* base, size_t i, const float (&x)[8]) {
  if constexpr (DT == DYNAKV_F32) {
    put<STREAM>((f4*)((float*)base + i), f4{x[0], x[1], x[2], x[3]});
    put<STREAM>((f4*)((float*)base + i + 4), f4{x[4], x[5], x[6], x[7]});
  } else {
    u4 w;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint16_t h[2];
#pragma unroll
      for (int z = 0; z < 2; ++z)
        h[z] = DT == DYNAKV_F16 ? __builtin_bit_cast(uint16_t, (_Float16)x[2 * k + z])
                                : __builtin_bit_cast(uint16_t, (__bf16)x[2 * k + z]);
      w[k] = h[0] | ((uint32_t)h[1] << 16);
    }
    put<STREAM>((u4*)((uint16_t*)base + i), w);
  }
}

// One row of 16 lanes per row of K and of V.
template <int DT, int BITS, bool STREAM>
__global__ __launch_bounds__(256) void packed_write_kernel(dynakv_packed_t c, const void* K, const void* V, int n, const int* start,
                                                           const int* count) {
  const long long row = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int lane = threadIdx.x & 15;
  if (row >= (long long)c.n_units * n) return;
  const int u = (int)(row / n), i = (int)(row % n);
  if (count && i >= count[u]) return;
  const long long at = (long long)(start ? start[u] : 0) + i;
  if (at < 0 || at >= c.capacity) return;
  const size_t to = (size_t)u * c.capacity + (size_t)at;
#pragma unroll
  for (int z = 0; z < 2; ++z) {
    float x[8];
    load_row8<DT, STREAM>(z ? V : K, (size_t)row * kHeadDim + 8 * lane, x);
    int code[8];
    const uint32_t s = quantise<DT, BITS>(x, code);
    store_codes<BITS>((uint8_t*)(z ? c.v_codes : c.k_codes) + to * code_bytes(BITS), lane, code);
    if ((lane & 3) == 0) (z ? c.v_scales : c.k_scales)[to * kRowScales + (lane >> 2)] = (uint8_t)s;
  }
}

template <int DT, int BITS, bool STREAM>
__global__ __launch_bounds__(256) void packed_read_kernel(dynakv_packed_t c, const int* positions, int n, void* K, void* V) {
  const long long row = (long long)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int lane = threadIdx.x & 15;
  if (row >= (long long)c.n_units * n) return;
  const int u = (int)(row / n), at = positions ? positions[row] : (int)(row % n);
  if (at < 0 || at >= c.capacity) return;
  const size_t from = (size_t)u * c.capacity + at;
#pragma unroll
  for (int z = 0; z < 2; ++z) {
    const uint32_t s = (z ? c.v_scales : c.k_scales)[from * kRowScales + (lane >> 2)];
    float x[8];
    load_values<BITS>((const uint8_t*)(z ? c.v_codes : c.k_codes) + from * code_bytes(BITS), lane, scale_value(s), x);
    store8<DT, STREAM>(z ? V : K, (size_t)row * kHeadDim + 8 * lane, x);
  }
}

}  // namespace

// The rows of values go past the caches where they are more than those hold (112 units of bfloat16 and 8 bits, 448 MB: reading 118 us, so 99, writing
// 121, 110; 224 MB: 52, 51 and 55, 56; 56 MB, reading and a kernel that reads the keys: 25, 26.5, writing 15, 18).
#define DYNAKV_PACKED_AS(KERNEL, DT, ...)                                                               \
  do {                                                                                                  \
    const bool past = 2 * rows * kHeadDim * elem_size(DT) > kCacheBytes;                                \
    if (c.bits == 8) past ? KERNEL<DT, 8, true><<<grid, 256, 0, st>>>(__VA_ARGS__)                      \
                          : KERNEL<DT, 8, false><<<grid, 256, 0, st>>>(__VA_ARGS__);                    \
    else past ? KERNEL<DT, 4, true><<<grid, 256, 0, st>>>(__VA_ARGS__)                                  \
              : KERNEL<DT, 4, false><<<grid, 256, 0, st>>>(__VA_ARGS__);                                \
  } while (0)
#define DYNAKV_PACKED(KERNEL, ...)                                                                      \
  do {                                                                                                  \
    const long long rows = (long long)c.n_units * n;                                                    \
    const unsigned grid = (unsigned)((rows + 15) / 16);                                                 \
    if (c.dtype == DYNAKV_F32) DYNAKV_PACKED_AS(KERNEL, DYNAKV_F32, __VA_ARGS__);                       \
    else if (c.dtype == DYNAKV_F16) DYNAKV_PACKED_AS(KERNEL, DYNAKV_F16, __VA_ARGS__);                  \
    else DYNAKV_PACKED_AS(KERNEL, DYNAKV_BF16, __VA_ARGS__);                                            \
  } while (0)

hipError_t launch_packed_write(const dynakv_packed_t& c, const void* K, const void* V, int n, const int* start, const int* count,
                               hipStream_t st) {
  DYNAKV_PACKED(packed_write_kernel, c, K, V, n, start, count);
  return hipGetLastError();
}

hipError_t launch_packed_read(const dynakv_packed_t& c, const int* positions, int n, void* K, void* V, hipStream_t st) {
  DYNAKV_PACKED(packed_read_kernel, c, positions, n, K, V);
  return hipGetLastError();
}
#undef DYNAKV_PACKED
#undef DYNAKV_PACKED_AS

}  // namespace dynakv
