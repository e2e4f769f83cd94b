// Attention of a tree of drafted tokens over gathered or packed entries (dynakv_attend_tree, dynakv_packed_attend).
//
// A unit has R = nodes * G rows of queries, L entries that every row sees, and up to 64 drafted tokens of which a row sees
// those in its node's bits.  One pass over the entries with running maximum m and sum l per row:
//   x = sc q.k (log2 domain), m' = max(m, x), o = o 2^(m - m') + sum 2^(x - m') v, l likewise; out = o / l.
// A wavefront works on 32 rows and 32 entries at a time, transposed: S^T = K Q^T puts a row into a lane (both halves of the
// wavefront hold 16 of its 32 entries), so maxima and sums stay in the lane but for one exchange between the halves, and
// the probabilities are, as they lie in the registers, the B operand of O^T += V^T P^T: the matrix instruction sums over
// entries in whatever order both operands agree on.  V comes out of LDS transposed by the LDS's transposing read.
//
// K and V tiles lie in LDS row by row, 16-byte chunk c of row r at position c ^ fz(r): 16 rows at one chunk (K) and 4 rows
// at 4 neighbouring chunks (V) each fall on different banks.
#include "operators.hpp"

namespace dynakv {

namespace {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));

constexpr float kLn2 = 0.6931471805599453f;
constexpr int kSub = 32;                             // entries of one matrix tile, rows of a wavefront

__device__ __forceinline__ int fz(int row) { return ((row & 3) << 2) | ((row >> 2) & 3); }
// entry of accumulator register i of the lanes of half h
__device__ __forceinline__ constexpr int entry_of(int i, int h) { return 8 * (i >> 2) + 4 * h + (i & 3); }

// Matrix products of one storage type.  Rows of a tile are kRow bytes.
template <int DT>
struct Mma {
  static constexpr int kES = 2, kRow = kHeadDim * 2;
  struct Q { uint4 b[8]; };
  static __device__ __forceinline__ void load_q(Q& q, const void* base, size_t row, int h, bool ok) {
    const char* p = (const char*)base + row * kRow + 16 * h;
#pragma unroll
    for (int s = 0; s < 8; ++s) q.b[s] = ok ? *(const uint4*)(p + 32 * s) : uint4{0, 0, 0, 0};
  }
  static __device__ __forceinline__ f16v mma(uint4 a, uint4 b, f16v c) {
    if constexpr (DT == DYNAKV_BF16)
      return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
    else
      return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f16v qk(const char* k, const Q& q, int lane) {
    const int t = lane & 31, x = ((lane >> 5) ^ fz(t)) << 4;
    f16v c = {};
#pragma unroll
    for (int s = 0; s < 8; ++s) c = mma(*(const uint4*)(k + t * kRow + (x ^ (s << 5))), q.b[s], c);
    return c;
  }
  static __device__ __forceinline__ uint16_t round16(float x) {
    if constexpr (DT == DYNAKV_BF16) return __builtin_bit_cast(uint16_t, (__bf16)x);
    else return __builtin_bit_cast(uint16_t, (_Float16)x);
  }
  static __device__ __forceinline__ void pv(f16v (&o)[4], const char* v, const float (&p)[16], int lane) {
    const int h = lane >> 5, g = (lane >> 4) & 1, j = lane & 15;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      // the probability that weights V goes in rounded to V's type: an error of half a step relative to each term, as much
      // as rounding the output costs
      uint32_t w[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) w[k] = round16(p[8 * c + 2 * k]) | ((uint32_t)round16(p[8 * c + 2 * k + 1]) << 16);
      const uint4 b = {w[0], w[1], w[2], w[3]};
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        uint2 a[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          // a group of 16 lanes reads 4 entries (rows) of 16 columns and gets the 4 entries of one column per lane
          const int row = 16 * c + 8 * x + 4 * h + (j >> 2), chunk = 4 * d + 2 * g + ((j & 3) >> 1);
          const char* at = v + row * kRow + ((chunk ^ (((j >> 2) << 2) | (2 * x + h))) << 4) + (j & 1) * 8;
          a[x] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)at));
        }
        o[d] = mma(uint4{a[0].x, a[0].y, a[1].x, a[1].y}, b, o[d]);
      }
    }
  }
  static __device__ __forceinline__ float elem(const void* base, size_t i) { return load_elem(base, i, DT); }
  // four consecutive columns of an output row
  static __device__ __forceinline__ void store4(void* out, size_t i, f4 x) {
    *(uint2*)((uint16_t*)out + i) = uint2{round16(x[0]) | ((uint32_t)round16(x[1]) << 16), round16(x[2]) | ((uint32_t)round16(x[3]) << 16)};
  }
  // whether one of the elements of a chunk is no finite number
  static __device__ __forceinline__ uint4 only_finite(uint4 a, bool& bad) {
    constexpr uint32_t ex = DT == DYNAKV_BF16 ? 0x7F80u : 0x7C00u;
    uint32_t* w = (uint32_t*)&a;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if ((w[k] & ex) == ex) { bad = true; w[k] &= 0xFFFF0000u; }
      if (((w[k] >> 16) & ex) == ex) { bad = true; w[k] &= 0xFFFFu; }
    }
    return a;
  }
};

template <>
struct Mma<DYNAKV_F32> {
  static constexpr int kES = 4, kRow = kHeadDim * 4;
  struct Q { f4 b[16]; };
  static __device__ __forceinline__ void load_q(Q& q, const void* base, size_t row, int h, bool ok) {
    const char* p = (const char*)base + row * kRow + 16 * h;
#pragma unroll
    for (int s = 0; s < 16; ++s) q.b[s] = ok ? *(const f4*)(p + 32 * s) : f4{0, 0, 0, 0};
  }
  static __device__ __forceinline__ f16v qk(const char* k, const Q& q, int lane) {
    const int t = lane & 31, x = ((lane >> 5) ^ fz(t)) << 4;
    f16v c = {};
#pragma unroll
    for (int s = 0; s < 16; ++s) {
      const f4 a = *(const f4*)(k + t * kRow + (x ^ (s << 5)));
#pragma unroll
      for (int i = 0; i < 4; ++i) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], q.b[s][i], c, 0, 0, 0);
    }
    return c;
  }
  static __device__ __forceinline__ void pv(f16v (&o)[4], const char* v, const float (&p)[16], int lane) {
    const int h = lane >> 5, col = lane & 31;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const int row = entry_of(i, h);
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const float a = *(const float*)(v + row * kRow + (((8 * d + (col >> 2)) ^ fz(row)) << 4) + ((col & 3) << 2));
        o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, p[i], o[d], 0, 0, 0);
      }
    }
  }
  static __device__ __forceinline__ float elem(const void* base, size_t i) { return ((const float*)base)[i]; }
  static __device__ __forceinline__ void store4(void* out, size_t i, f4 x) { *(f4*)((float*)out + i) = x; }
  static __device__ __forceinline__ uint4 only_finite(uint4 a, bool& bad) {
    uint32_t* w = (uint32_t*)&a;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if ((w[k] & 0x7F800000u) == 0x7F800000u) { bad = true; w[k] = 0; }
    return a;
  }
};

// Running state of a wavefront's 32 rows: lane l has row l % 32, register i of o[d] column 32 d + entry_of(i, l / 32).
struct Rows {
  float m, l;                                        // log2 domain; l of the lane's half of the entries
  f16v o[4];
};

// One tile of 32 entries; `seen`: bit t is set if the lane's row sees entry t (0 where the slot holds none).  Slots that
// hold nothing have zeros in V.
template <int DT>
__device__ __forceinline__ void consume(Rows& st, const char* k, const char* v, const typename Mma<DT>::Q& q, uint32_t seen, float sc, int lane) {
  const f16v s = Mma<DT>::qk(k, q, lane);
  const uint32_t mine = seen >> (4 * (lane >> 5));
  float x[16], mx = -__builtin_inff();
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    x[i] = (mine >> entry_of(i, 0)) & 1u ? s[i] * sc : -__builtin_inff();
    mx = fmaxf(mx, x[i]);
  }
  const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
  const float mn = fmaxf(st.m, fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])));
  const float alpha = mn == st.m ? 1.f : __builtin_amdgcn_exp2f(st.m - mn);
  st.m = mn;
  st.l *= alpha;
#pragma unroll
  for (int d = 0; d < 4; ++d) st.o[d] *= alpha;
  const float base = mn == -__builtin_inff() ? 0.f : mn;      // nothing seen yet
  float p[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    p[i] = __builtin_amdgcn_exp2f(x[i] - base);
    st.l += p[i];
  }
  Mma<DT>::pv(st.o, v, p, lane);
}

enum Source { kList, kPacked8, kPacked4 };

struct Span { int splits, first, last; };            // tiles of 32 entries [first, last) of one split
// How the L entries of a unit are shared: the same in the kernel that works and in the one that joins.
__device__ __forceinline__ int splits_of(int L, int S, int chunk) { return min(S, max(1, L / chunk)); }

// 16 bytes of tile row `row`, chunk c -> its place
__device__ __forceinline__ char* place(char* tile, int rowb, int row, int c) { return tile + row * rowb + ((c ^ fz(row)) << 4); }

// Writes the values of 16 or 32 codes (16 bytes) of one block, tile row `row`, chunk by chunk of the row.
template <int DT, int BITS>
__device__ __forceinline__ void spread(char* tile, int row, int part, uint4 w4, float scale) {
  constexpr int rowb = Mma<DT>::kRow, kVals = 128 / BITS, per = 16 / Mma<DT>::kES;   // values per chunk of the tile
  const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
  for (int c = 0; c < kVals / per; ++c) {
    uint32_t o[4];
    float x[per];
#pragma unroll
    for (int k = 0; k < per; ++k) {
      const int i = c * per + k, bit = (i * BITS) & 31;
      x[k] = (float)((int)(w[(i * BITS) >> 5] << (32 - BITS - bit)) >> (32 - BITS)) * scale;
    }
    if constexpr (DT == DYNAKV_F32) {
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = __float_as_uint(x[k]);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = Mma<DT>::round16(x[2 * k]) | ((uint32_t)Mma<DT>::round16(x[2 * k + 1]) << 16);   // exact
    }
    *(uint4*)place(tile, rowb, row, part * (kVals / per) + c) = uint4{o[0], o[1], o[2], o[3]};
  }
}

// grid: XCD-interleaved (unit, split) x row blocks; 4 wavefronts, each with all its rows in registers and a tile of its own.
template <int DT, int SRC>
__global__ __launch_bounds__(256) void tree_kernel(TreeArgs a) {
  using M = Mma<DT>;
  constexpr int kTile = kSub * M::kRow, kOut = kHeadDim + 4;      // bytes of a K or V tile; floats of a row in the merge
  extern __shared__ __align__(16) char lds[];
  // workgroups with the same entries run on the same XCD, one after the other: they share its L2
  const int us = ((int)blockIdx.x >> 3) / a.RB * 8 + ((int)blockIdx.x & 7), rb = ((int)blockIdx.x >> 3) % a.RB;
  if (us >= a.U * a.S) return;
  const int u = us / a.S, s = us % a.S;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5;
  const int R = a.T * a.G, row = rb * kSub + (lane & 31);
  const bool live = row < R;

  int L, nlist = 0;
  if constexpr (SRC == kList) {
    nlist = a.n_list[u];
    L = 4 * nlist;
  } else {
    L = a.lengths ? min(max(a.lengths[u], 0), a.cache.capacity) : a.cache.capacity;
  }
  const int ns = splits_of(L, a.S, a.chunk);
  if (s >= ns) return;
  const int nt = (L + kSub - 1) / kSub, t0 = (int)((long long)nt * s / ns), t1 = (int)((long long)nt * (s + 1) / ns);

  typename M::Q q;
  M::load_q(q, a.Q, (size_t)u * R + (live ? row : 0), h, live);
  Rows st;
  st.m = -__builtin_inff(); st.l = 0.f;
#pragma unroll
  for (int d = 0; d < 4; ++d) st.o[d] = f16v{};
  char* kt = lds + wave * 2 * kTile;
  char* vt = kt + kTile;

  for (int t = t0 + wave; t < t1; t += 4) {
    uint32_t seen;
    if constexpr (SRC == kList) {
      constexpr int kPer = 64 * 16 / M::kRow;        // rows that 64 lanes load at once
      const char* pages = a.pages + (size_t)u * a.unit_pages;
      const int e = 8 * t + (lane >> 2 & 7);
      const int ent = e < nlist ? a.plist[(size_t)u * a.Lcap + e] : -1;
      seen = (uint32_t)__ballot(ent >= 0 && (lane & 3) <= (ent & 3));
#pragma unroll
      for (int i = 0; i < kSub / kPer; ++i) {
        const int r = i * kPer + lane * 16 / M::kRow, c = lane % (M::kRow / 16), en = __shfl(ent, r & ~3);
        uint4 kk = {0, 0, 0, 0}, vv = {0, 0, 0, 0};
        if ((seen >> r) & 1u) {
          const char* p = pages + (size_t)(en >> 4) * (kPageElems * M::kES) + (((en >> 2) & 3) * 4 + (r & 3)) * M::kRow + c * 16;
          kk = *(const uint4*)p;
          vv = *(const uint4*)(p + 2048 * M::kES);
        }
        *(uint4*)place(kt, M::kRow, r, c) = kk;
        *(uint4*)place(vt, M::kRow, r, c) = vv;
      }
    } else {
      constexpr int bits = SRC == kPacked8 ? 8 : 4, cb = kHeadDim * bits / 8, parts = cb / 16;
      const int n = min(kSub, L - t * kSub);
      seen = n >= kSub ? ~0u : (1u << n) - 1u;
      const size_t first = (size_t)u * a.cache.capacity + (size_t)t * kSub;
#pragma unroll
      for (int i = 0; i < kSub * parts / 64; ++i) {
        const int r = (i * 64 + lane) / parts, part = lane % parts;
        uint4 kk = {0, 0, 0, 0}, vv = {0, 0, 0, 0};
        uint32_t ks = 127, vs = 127;
        if (r < n) {
          kk = *(const uint4*)((const char*)a.cache.k_codes + (first + r) * cb + part * 16);
          vv = *(const uint4*)((const char*)a.cache.v_codes + (first + r) * cb + part * 16);
          ks = a.cache.k_scales[(first + r) * kRowScales + part * 4 / parts];
          vs = a.cache.v_scales[(first + r) * kRowScales + part * 4 / parts];
        }
        spread<DT, bits>(kt, r, part, kk, scale_value(ks));
        spread<DT, bits>(vt, r, part, vv, scale_value(vs));
      }
    }
    asm volatile("" ::: "memory");                   // the same wavefront's LDS operations keep their order; the compiler must too
    consume<DT>(st, kt, vt, q, seen, a.sc, lane);
    asm volatile("" ::: "memory");
  }

  // the drafted tokens: the unit's last split, one tile of 32 per wavefront
  if (s == ns - 1 && a.K1 && wave * kSub < a.T) {
    constexpr int kPer = 64 * 16 / M::kRow;
    const int j0 = wave * kSub;
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < kSub / kPer; ++i) {
      const int r = i * kPer + lane * 16 / M::kRow, c = lane % (M::kRow / 16);
      uint4 kk = {0, 0, 0, 0}, vv = {0, 0, 0, 0};
      bool b = false;
      if (j0 + r < a.T) {
        const size_t at = ((size_t)u * a.T + j0 + r) * M::kRow + c * 16;
        kk = *(const uint4*)((const char*)a.K1 + at);
        vv = M::only_finite(*(const uint4*)((const char*)a.V1 + at), b);
      }
      *(uint4*)place(kt, M::kRow, r, c) = kk;
      *(uint4*)place(vt, M::kRow, r, c) = vv;
      const unsigned long long any = __ballot(b);
#pragma unroll
      for (int z = 0; z < kPer; ++z)
        if ((any >> (z * (64 / kPer))) & (~0ull >> (64 - 64 / kPer))) bad |= 1u << (i * kPer + z);
    }
    const int node = (live ? row : 0) / a.G;
    unsigned long long bits = a.tree ? a.tree[(size_t)u * a.T + node] : ~0ull >> (63 - node);
    if (a.T < 64) bits &= (1ull << a.T) - 1;
    const uint32_t seen = (uint32_t)(bits >> j0);
    asm volatile("" ::: "memory");
    consume<DT>(st, kt, vt, q, seen, a.sc, lane);
    asm volatile("" ::: "memory");
    // values that are not finite went in as zeros, so that a row which does not see their token stays clean of them; the
    // rows that see it get them here
    while (bad) {
      const int j = __builtin_ctz(bad);
      bad &= bad - 1;
      const bool sees = (seen >> j) & 1u;
      const size_t at = ((size_t)u * a.T + j0 + j) * kHeadDim;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float x = M::elem(a.V1, at + 32 * d + entry_of(i, 0) + 4 * h);
          if (sees && !(fabsf(x) < __builtin_inff())) st.o[d][i] += x;
        }
    }
  }

  // join the four wavefronts: every one leaves its rows in LDS
  const auto lsum = __builtin_amdgcn_permlane32_swap(__float_as_uint(st.l), __float_as_uint(st.l), false, false);
  st.l = __uint_as_float(lsum[0]) + __uint_as_float(lsum[1]);
  __syncthreads();
  float* mo = (float*)lds;
  {
    float* mine = mo + ((size_t)wave * kSub + (lane & 31)) * kOut;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4) *(f4*)(mine + 32 * d + entry_of(i, h)) = f4{st.o[d][i], st.o[d][i + 1], st.o[d][i + 2], st.o[d][i + 3]};
    if (h == 0) { mine[kHeadDim] = st.m; mine[kHeadDim + 1] = st.l; }
  }
  __syncthreads();
  for (int t = threadIdx.x; t < kSub * (kHeadDim / 4); t += 256) {
    const int r = t >> 5, c = (t & 31) * 4, rr = rb * kSub + r;
    if (rr >= R) break;
    float mw[4], m = -__builtin_inff(), l = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) { mw[w] = mo[(w * kSub + r) * kOut + kHeadDim]; m = fmaxf(m, mw[w]); }
    f4 o = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      if (mw[w] == -__builtin_inff()) continue;       // that wavefront saw nothing of this row
      const float f = mw[w] == m ? 1.f : __builtin_amdgcn_exp2f(mw[w] - m);
      const float* x = mo + (w * kSub + r) * kOut;
      l += f * x[kHeadDim + 1];
      o += f * *(const f4*)(x + c);
    }
    const size_t to = (size_t)u * R + rr;
    if (ns == 1) {
      const bool none = m == -__builtin_inff();
      M::store4(a.out, to * kHeadDim + c, none ? f4{0, 0, 0, 0} : o / l);
      if (a.lse && c == 0) a.lse[to] = none ? m : (m + __builtin_amdgcn_logf(l)) * kLn2;
    } else {
      float* p = a.part + (((size_t)u * a.S + s) * R + rr) * kPartRow;
      *(f4*)(p + c) = o;
      if (c == 0) { p[kHeadDim] = m; p[kHeadDim + 1] = l; }
    }
  }
}

// Joins the splits of the units that have several: 32 lanes a row.
template <int DT>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeArgs a) {
  const int R = a.T * a.G;
  const long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (i >= (long long)a.U * R) return;
  const int u = (int)(i / R), r = (int)(i % R), c = (threadIdx.x & 31) * 4;
  const int L = a.pages ? 4 * a.n_list[u] : a.lengths ? min(max(a.lengths[u], 0), a.cache.capacity) : a.cache.capacity;
  const int ns = splits_of(L, a.S, a.chunk);
  if (ns == 1) return;
  const float* p = a.part + ((size_t)u * a.S * R + r) * kPartRow;
  float m = -__builtin_inff(), l = 0.f;
  for (int s = 0; s < ns; ++s) m = fmaxf(m, p[(size_t)s * R * kPartRow + kHeadDim]);
  f4 o = {0, 0, 0, 0};
  for (int s = 0; s < ns; ++s) {
    const float* x = p + (size_t)s * R * kPartRow;
    const float ms = x[kHeadDim];
    if (ms == -__builtin_inff()) continue;
    const float f = ms == m ? 1.f : __builtin_amdgcn_exp2f(ms - m);
    l += f * x[kHeadDim + 1];
    o += f * *(const f4*)(x + c);
  }
  const bool none = m == -__builtin_inff();
  Mma<DT>::store4(a.out, (size_t)i * kHeadDim + c, none ? f4{0, 0, 0, 0} : o / l);
  if (a.lse && c == 0) a.lse[i] = none ? m : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Workgroups that may share a unit's entries, so that about two workgroups per compute unit have work.
int most_splits(int U, int R) {
  const long long wgs = (long long)U * ((R + kSub - 1) / kSub);
  const long long s = (512 + wgs - 1) / wgs;
  return (int)(s < 1 ? 1 : s > 64 ? 64 : s);
}

template <int DT>
hipError_t launch(TreeArgs a, hipStream_t st) {
  const int R = a.T * a.G;
  a.RB = (R + kSub - 1) / kSub;
  a.S = most_splits(a.U, R);
  // a partial result costs a row 2 * 528 bytes of traffic: a workgroup's share of the entries is several times that
  a.chunk = max(256, 4 * R);
  while (a.S > 1 && (long long)a.chunk * (a.S - 1) >= a.most) --a.S;
  const long long us = ((long long)a.U * a.S + 7) / 8 * 8;
  const unsigned grid = (unsigned)(us * a.RB);
  const size_t tiles = 4 * 2 * kSub * Mma<DT>::kRow, merge = 4 * kSub * (kHeadDim + 4) * 4, lds = tiles > merge ? tiles : merge;
  const void* f;
  if (a.pages) f = (const void*)tree_kernel<DT, kList>;
  else if (a.cache.bits == 8) f = (const void*)tree_kernel<DT, kPacked8>;
  else f = (const void*)tree_kernel<DT, kPacked4>;
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(f, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  void* args[] = {&a};
  const hipError_t e = hipLaunchKernel(f, dim3(grid), dim3(256), args, lds, st);
  if (e != hipSuccess) return e;
  if (a.S > 1) tree_join_kernel<DT><<<(unsigned)(((long long)a.U * R + 7) / 8), 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace

size_t tree_scratch_bytes(int U, int T, int G) {
  const size_t R = (size_t)T * G;
  const int S = most_splits(U, (int)R);
  return 256 + (S > 1 ? (size_t)U * S * R * kPartRow * sizeof(float) : 0);
}

hipError_t launch_tree(const TreeArgs& a, hipStream_t st) {
  if (a.dtype == DYNAKV_F32) return launch<DYNAKV_F32>(a, st);
  if (a.dtype == DYNAKV_F16) return launch<DYNAKV_F16>(a, st);
  return launch<DYNAKV_BF16>(a, st);
}

}  // namespace dynakv
