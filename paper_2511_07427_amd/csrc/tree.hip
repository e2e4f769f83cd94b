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
// K and V tiles lie in LDS row by row, padded so that the lanes served together fall on different banks: 16 rows at one 16-byte
// chunk of K (pad 16: rows 4 banks apart), 4 rows at 32 neighbouring bytes of V (pad 32: rows 8 banks apart).  Padding, unlike a
// permutation of the chunks, leaves every place of a tile at a constant distance from one address per lane: a permutation cost some
// 40 registers of addresses, which the accumulators need.
#include <algorithm>

#include "operators.hpp"

namespace dynakv {

namespace {

typedef float f16v __attribute__((ext_vector_type(16)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef float f2v __attribute__((ext_vector_type(2)));
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));

constexpr float kLn2 = 0.6931471805599453f;
constexpr int kSub = 32;                             // entries of one matrix tile, rows of a wavefront
constexpr int kWorkgroups = 256;                     // that run at once: one per compute unit
constexpr int kPlanUnits = 512;                      // of more units none is shared

// Keeps the loads of what follows from being moved up in front of what came before, where their results fill the registers.
__device__ __forceinline__ void hold_order() { __builtin_amdgcn_sched_barrier(0); }

// entry of accumulator register i of the lanes of half h
__device__ __forceinline__ constexpr int entry_of(int i, int h) { return 8 * (i >> 2) + 4 * h + (i & 3); }

// Matrix products of one storage type.  Rows of a tile are kRow bytes.
template <int DT>
struct Mma {
  static constexpr int kES = 2, kRow = kHeadDim * 2, kRowK = kRow + 16, kRowV = kRow + 32;   // in memory, in LDS
  struct Q { uint4 b[8]; };
  static __device__ __forceinline__ void load_q(Q& q, const void* base, size_t row, int h) {
    const char* p = (const char*)base + row * kRow + 16 * h;
#pragma unroll
    for (int s = 0; s < 8; ++s) q.b[s] = *(const uint4*)(p + 32 * s);
  }
  static __device__ __forceinline__ f16v mma(uint4 a, uint4 b, f16v c) {
    if constexpr (DT == DYNAKV_BF16)
      return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
    else
      return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
  }
  // Adds the scores of N tiles of 32 entries each, kSub rows apart.  The operands of a step are requested two steps before it.
  template <int N>
  static __device__ __forceinline__ void qk(f16v (&c)[N], const char* k, const Q& q, int lane) {
    const char* at = k + (lane & 31) * kRowK + (lane >> 5) * 16;
    uint4 f[8][N];
    auto request = [&](int s) {
#pragma unroll
      for (int n = 0; n < N; ++n) f[s][n] = *(const uint4*)(at + n * kSub * kRowK + s * 32);
    };
    request(0);
    request(1);
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      if (s + 2 < 8) request(s + 2);
      hold_order();
#pragma unroll
      for (int n = 0; n < N; ++n) c[n] = mma(f[s][n], q.b[s], c[n]);
    }
  }
  static __device__ __forceinline__ uint16_t round16(float x) {
    if constexpr (DT == DYNAKV_BF16) return __builtin_bit_cast(uint16_t, (__bf16)x);
    else return __builtin_bit_cast(uint16_t, (_Float16)x);
  }
  static __device__ __forceinline__ uint32_t round2(float x, float y) {
    if constexpr (DT == DYNAKV_BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2v){x, y}, b2));
    else return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2v){x, y}, h2));
  }
  // c + the sum of two rounded values.
  static __device__ __forceinline__ float add2(uint32_t w, float c) {
    if constexpr (DT == DYNAKV_BF16) return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(b2, w), (b2){(__bf16)1.f, (__bf16)1.f}, c, false);
    else return __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, w), (h2){(_Float16)1.f, (_Float16)1.f}, c, false);
  }
  // V^T of the 16 entries of chunk c: a group of 16 lanes reads 4 entries (rows) of 16 columns and gets the 4 entries of one column
  // per lane
  struct VFrag { uint4 d[4]; };
  static __device__ __forceinline__ void load_v(VFrag& f, const char* v, int c, int lane) {
    const int j = lane & 15;
    const char* from = v + ((lane >> 5) * 4 + (j >> 2)) * kRowV + ((lane >> 4) & 1) * 32 + (j & 3) * 8 + c * 16 * kRowV;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      uint2 a[2];
#pragma unroll
      for (int x = 0; x < 2; ++x)
        a[x] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s4*)(from + 8 * x * kRowV + d * 64)));
      f.d[d] = uint4{a[0].x, a[0].y, a[1].x, a[1].y};
    }
  }
  static __device__ __forceinline__ float elem(const void* base, size_t i) { return load_elem(base, i, DT); }
  // four consecutive columns of an output row
  static __device__ __forceinline__ void store4(void* out, size_t i, f4 x) {
    *(uint2*)((uint16_t*)out + i) = uint2{round2(x[0], x[1]), round2(x[2], x[3])};
  }
  // Bits 15 and 31: whether the elements of w are no finite numbers (their exponent is all ones, and carries).
  static __device__ __forceinline__ uint32_t not_finite(uint32_t w) {
    constexpr uint32_t ex = DT == DYNAKV_BF16 ? 0x7F807F80u : 0x7C007C00u, low = DT == DYNAKV_BF16 ? 0x00800080u : 0x04000400u;
    return ((w & ex) + low) & 0x80008000u;
  }
  // a chunk with zeros for the elements that are no finite numbers; bad: there was one
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
  struct VFrag {};
  static constexpr int kES = 4, kRow = kHeadDim * 4, kRowK = kRow + 16, kRowV = kRow + 32;
  struct Q { f4 b[16]; };
  static __device__ __forceinline__ void load_q(Q& q, const void* base, size_t row, int h) {
    const char* p = (const char*)base + row * kRow + 16 * h;
#pragma unroll
    for (int s = 0; s < 16; ++s) q.b[s] = *(const f4*)(p + 32 * s);
  }
  template <int N>
  static __device__ __forceinline__ void qk(f16v (&c)[N], const char* k, const Q& q, int lane) {
    const char* at = k + (lane & 31) * kRowK + (lane >> 5) * 16;
#pragma unroll
    for (int s = 0; s < 16; ++s)
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const f4 a = *(const f4*)(at + n * kSub * kRowK + s * 32);
#pragma unroll
        for (int i = 0; i < 4; ++i) c[n] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[i], q.b[s][i], c[n], 0, 0, 0);
        if (s % 4 == 3) hold_order();
      }
  }
  static __device__ __forceinline__ void pv(f16v (&o)[4], const char* v, const float (&p)[16], int lane) {
    const char* from = v + (lane >> 5) * 4 * kRowV + (lane & 31) * 4;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const float a = *(const float*)(from + entry_of(i, 0) * kRowV + d * 128);
        o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, p[i], o[d], 0, 0, 0);
      }
      if (i % 4 == 3) hold_order();
    }
  }
  static __device__ __forceinline__ float elem(const void* base, size_t i) { return ((const float*)base)[i]; }
  static __device__ __forceinline__ void store4(void* out, size_t i, f4 x) { *(f4*)((float*)out + i) = x; }
  static __device__ __forceinline__ uint32_t not_finite(uint32_t w) { return ((w & 0x7F800000u) + 0x00800000u) & 0x80000000u; }
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
  float m, l;                                        // what the weights are relative to (log2), and their sum over the lane's half of the entries
  float w[2];                                        // the sum of the weights as they go into the products, in two parts (float32: l and 0)
  f16v o[4];
};
// Whether a part of a row's entries (a wavefront's, a piece's) has none that the row sees: its sum is 0 then.  The maximum alone does not say so: it
// passes over scores that are NaN, whose sum is NaN and has to come out.
__device__ __forceinline__ bool saw_nothing(float m, float l) { return m == -__builtin_inff() && l == 0.f; }

// What the scores of 32 slots begin with: 0, or -inf where a slot holds nothing.  (Conditions per slot on the finished scores, the same
// for every row, took as many instructions as the exponentials.)
__device__ __forceinline__ f16v begin_scores(const float* bias, int lane) {
  f16v c;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const f4 x = *(const f4*)(bias + 8 * g + 4 * (lane >> 5));
#pragma unroll
    for (int i = 0; i < 4; ++i) c[4 * g + i] = x[i];
  }
  return c;
}
// N tiles of 32 entries.  Of a tile of the cache every row sees the same slots, those with a bias of 0; of drafted tokens (their bias is 0) those
// whose bit is set in `seen`.  Slots that hold nothing have zeros in K and V.
// The accumulators are rescaled only when a maximum has grown by more than 2^kLazy since they last were: until then weights grow up to that,
// and 64 products per tile and row are saved in all but a few tiles (half a percent of the time of 128 packed units of 128 rows, one percent of that of
// 112 units of 427 rows).  Weights are relative to 2^-kShift times the maximum: those of float16, whose smallest step is 2^-24, so reach down to
// 2^-31 of the largest (many small ones beside a large one count), and stay below 2^15.
constexpr float kLazy = 8.f;
template <int DT>
constexpr float kShift = DT == DYNAKV_F16 ? 7.f : 0.f;
template <int DT, int N>
__device__ __forceinline__ void consume(Rows& st, const char* k, const char* v, const float* bias, const typename Mma<DT>::Q& q, bool drafts,
                                        unsigned long long seen, float sc, int lane) {
  using M = Mma<DT>;
  f16v s[N];
#pragma unroll
  for (int n = 0; n < N; ++n) s[n] = begin_scores(bias + n * kSub, lane);
  M::template qk<N>(s, k, q, lane);
  [[maybe_unused]] typename M::VFrag f[2];
  if constexpr (DT != DYNAKV_F32) M::load_v(f[0], v, 0, lane);       // arrives while the maxima are taken
  if (drafts) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const uint32_t mine = (uint32_t)(seen >> (32 * n)) >> (4 * (lane >> 5));
#pragma unroll
      for (int i = 0; i < 16; ++i) s[n][i] = (mine >> entry_of(i, 0)) & 1u ? s[n][i] : -__builtin_inff();
    }
  }
  float mx = -__builtin_inff();
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[n][i]);
  const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
  mx = fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])) * sc;
  if (__any(mx > st.m + (kLazy + kShift<DT>))) {     // (from -inf: any finite one)
    const float mn = fmaxf(st.m, mx - kShift<DT>), alpha = mn == st.m ? 1.f : __builtin_amdgcn_exp2f(st.m - mn);
    st.m = mn;
    st.l *= alpha;
    st.w[0] *= alpha;
    st.w[1] *= alpha;
#pragma unroll
    for (int d = 0; d < 4; ++d) st.o[d] *= alpha;
  }
  const float base = st.m == -__builtin_inff() ? 0.f : -st.m;      // nothing seen yet
  if constexpr (DT == DYNAKV_F32) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
      float p[16], sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        p[i] = __builtin_amdgcn_exp2f(fmaf(s[n][i], sc, base));
        sum[i & 3] += p[i];
      }
      st.w[0] = st.l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      M::pv(st.o, v + n * kSub * M::kRowV, p, lane);
    }
  } else {
    // 16 entries at a time: while the matrix cores take one chunk, the next one's weights are computed and its V is on its way.
    // A weight goes in rounded to V's type: an error of half a step relative to each term, as much as rounding the output costs.  What the sum of products is
    // divided by is the sum of the rounded weights, so that it is a mean: equal values come out as they are, none beyond the largest (32 of
    // float16's largest value came out as infinity with the sum before rounding).  The log-sum-exp has the other sum.  Both sums: 61 nodes on 112
    // bfloat16 units 84 us, one 80; the error against 64 bits 1.75e-3 instead of 1.88e-3 of the norm.
    auto weights = [&](int c) {
      float p[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) p[i] = __builtin_amdgcn_exp2f(fmaf(s[c >> 1][8 * (c & 1) + i], sc, base));
      st.l += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      const uint4 r = {M::round2(p[0], p[1]), M::round2(p[2], p[3]), M::round2(p[4], p[5]), M::round2(p[6], p[7])};
      st.w[0] = M::add2(r.y, M::add2(r.x, st.w[0]));
      st.w[1] = M::add2(r.w, M::add2(r.z, st.w[1]));
      return r;
    };
    uint4 w = weights(0);
#pragma unroll
    for (int c = 0; c < 2 * N; ++c) {
      if (c + 1 < 2 * N) M::load_v(f[(c + 1) & 1], v, c + 1, lane);
      hold_order();
      uint4 next = {};
      if (c + 1 < 2 * N) next = weights(c + 1);
#pragma unroll
      for (int d = 0; d < 4; ++d) st.o[d] = M::mma(f[c & 1].d[d], w, st.o[d]);
      w = next;
      hold_order();
    }
  }
}

enum Source { kList, kPacked8, kPacked4 };

template <int SRC>
__device__ __forceinline__ int slots_of(const TreeArgs& a, int u) {
  if constexpr (SRC == kList) return 4 * a.n_list[u];
  else return a.lengths ? min(max(a.lengths[u], 0), a.cache.capacity) : a.cache.capacity;
}

// A unit's entries are shared by ceil(entries / chunk) workgroups, `chunk` the smallest (to a sixteenth) with which all units together make no
// more than a.pieces: that many run in whole rounds of the chip, however much the units differ.  All workgroups find the same chunk,
// each for itself in one wavefront.  Piece q of all is piece `first` + s of unit u's `count`.
struct Piece { int u, s, count, first, slots; };
template <int SRC>
__device__ __forceinline__ Piece piece_of(const TreeArgs& a, int q, int lane) {
  if (a.pieces == a.U || a.U > kPlanUnits) return Piece{q, 0, 1, q, q < a.U ? slots_of<SRC>(a, q) : 0};   // whole units
  constexpr int kPer = kPlanUnits / 64;
  int len[kPer], most = 0;
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    const int u = lane + 64 * k;
    len[k] = u < a.U ? slots_of<SRC>(a, u) : -1;
    most = max(most, len[k]);
    sum += (float)max(len[k], 0);
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
  most = wave_max(most);
  // of a unit (the thousandth: a unit of no more than `chunk` entries is one piece, whatever the product's rounding)
  auto count_of = [](int n, float inv) { return max(1, (int)ceilf((float)n * inv - 1e-3f)); };
  auto fits = [&](int chunk) {
    const float inv = 1.f / (float)chunk;
    int c = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k)
      if (64 * k < a.U) c += len[k] >= 0 ? count_of(len[k], inv) : 0;
    return wave_sum(c) <= a.pieces;
  };
  // pieces >= sum / chunk, pieces <= sum / chunk + units
  int lo = max(a.least, (int)fminf(sum / (float)a.pieces, 1e9f)), hi = max(lo, most);
  if (!fits(lo)) {
    hi = max(lo + 1, min(hi, (int)fminf(sum / (float)(a.pieces - a.U), 1e9f) + 2));
    if (!fits(hi)) hi = max(hi, most);               // (one piece each)
    while (hi - lo > lo / 16 + 1) {
      const int mid = lo + (hi - lo) / 2;
      if (fits(mid)) hi = mid;
      else lo = mid;
    }
  } else {
    hi = lo;
  }
  const float inv = 1.f / (float)hi;
  int base = 0;
  Piece p = {-1, 0, 1, 0, 0};
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (64 * k >= a.U) break;
    const int c = len[k] >= 0 ? count_of(len[k], inv) : 0, end = base + wave_incl_scan(c);
    const unsigned long long here = __ballot(end - c <= q && q < end);
    if (here) {
      const int l = __builtin_ctzll(here);
      p = Piece{l + 64 * k, q - (__builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(c, l)), __builtin_amdgcn_readlane(c, l),
                __builtin_amdgcn_readlane(end, l) - __builtin_amdgcn_readlane(c, l), __builtin_amdgcn_readlane(len[k], l)};
    }
    base = __builtin_amdgcn_readlane(end, 63);
  }
  return p;                                          // u < 0: there are fewer pieces
}

// Two codes of a block (elements 2 i and 2 i + 1 of the eight or four in w) as float16 values.  A biased code c + 2^(BITS - 1) in the
// low bits of the float16 1024 is the value 1024 + c + 2^(BITS - 1), in bits 4..7 it is 1024 + 16 (c + 8): a byte permutation, and the
// arithmetic is packed and exact.  (Two instructions per value where conversion through float32 takes four and a half.)
template <int BITS>
__device__ __forceinline__ uint32_t pair_f16(uint32_t biased, int i, h2 scale) {
  if constexpr (BITS == 8) {
    const uint32_t x = __builtin_amdgcn_perm(0x64646464u, biased, i ? 0x04030402u : 0x04010400u);
    return __builtin_bit_cast(uint32_t, (__builtin_bit_cast(h2, x) - (h2){(_Float16)1152.f, (_Float16)1152.f}) * scale);
  } else {
    const uint32_t x = __builtin_amdgcn_perm(0x64646464u, biased, 0x04000400u + 0x00010001u * i) & 0xFFF0FF0Fu;
    const h2 c = __builtin_elementwise_fma(__builtin_bit_cast(h2, x), (h2){(_Float16)1.f, (_Float16)0.0625f}, (h2){(_Float16)-1032.f, (_Float16)-72.f});
    return __builtin_bit_cast(uint32_t, c * scale);
  }
}

// Writes the values of 16 or 32 codes (16 bytes) of one block to `to`.
template <int DT, int BITS>
__device__ __forceinline__ void spread(char* to, uint4 w4, float scale) {
  constexpr int kVals = 128 / BITS, per = 16 / Mma<DT>::kES;   // values per chunk of the tile
  const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
  if constexpr (DT == DYNAKV_F16) {
    const _Float16 s = (_Float16)scale;
    constexpr int kPairs = 16 / BITS;                // per word of codes
#pragma unroll
    for (int c = 0; c < kVals / per; ++c) {
      uint32_t o[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) o[k] = pair_f16<BITS>(w[(4 * c + k) / kPairs] ^ (BITS == 8 ? 0x80808080u : 0x88888888u), (4 * c + k) % kPairs, (h2){s, s});
      *(uint4*)(to + 16 * c) = uint4{o[0], o[1], o[2], o[3]};
    }
  } else {
    // a signed byte is converted in one instruction; a 4-bit code in the upper half of a byte counts 16 times
    const float s = BITS == 8 ? scale : scale * 0.0625f;
#pragma unroll
    for (int c = 0; c < kVals / per; ++c) {
      uint32_t o[4];
      float x[per];
#pragma unroll
      for (int k = 0; k < per; ++k) {
        const int i = c * per + k;
        const uint32_t from = BITS == 8 ? w[i / 4] : (i & 1 ? w[i / 8] : w[i / 8] << 4) & 0xF0F0F0F0u;
        x[k] = (float)(int8_t)(from >> (8 * (BITS == 8 ? i % 4 : i % 8 / 2))) * s;
      }
      if constexpr (DT == DYNAKV_F32) {
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = __float_as_uint(x[k]);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)                  // exact: the lower halves are zero
          o[k] = __builtin_amdgcn_perm(__float_as_uint(x[2 * k + 1]), __float_as_uint(x[2 * k]), 0x07060302u);
      }
      *(uint4*)(to + 16 * c) = uint4{o[0], o[1], o[2], o[3]};
    }
  }
}

// What a wavefront holds of the tile that is on its way: N rows of 16-bit or float32 storage or of codes, K and V.
// begin() requests rows r0 .. r0 + N - 1 of a tile, end() writes them to the tile in LDS, zeros in slots that hold nothing.
template <int DT, int SRC, int N>
struct Stage;

template <int DT, int N>
struct Stage<DT, kList, N> {
  using M = Mma<DT>;
  static constexpr int kPer = 64 * 16 / M::kRow, kLoads = N / kPer;      // rows that 64 lanes load at once
  uint4 k[kLoads], v[kLoads];
  // ent: lane 4 e holds list entry e of the tile (-1: none)
  __device__ __forceinline__ void begin(const TreeArgs& a, const char* pages, int ent, int r0, int lane) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      // an entry is four slots in a row; slots beyond its tokens and missing entries read slot 0 instead, of page 0
      const int first = r0 + i * kPer, sub = lane * 16 / M::kRow, en = max(0, __builtin_amdgcn_readlane(ent, first & ~3));
      const int slot = min((first & 3) + sub, en & 3);
      const char* p = pages + (size_t)(en >> 4) * (kPageElems * M::kES) + ((en >> 2) & 3) * 4 * M::kRow + slot * M::kRow + lane % (M::kRow / 16) * 16;
      k[i] = *(const uint4*)p;
      v[i] = *(const uint4*)(p + 2048 * M::kES);
    }
  }
  __device__ __forceinline__ void end(char* kt, char* vt, unsigned long long seen, bool full, int r0, int lane) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = r0 + i * kPer + lane * 16 / M::kRow, c = lane % (M::kRow / 16) * 16;
      if (!full && !((seen >> r) & 1u)) { k[i] = uint4{0, 0, 0, 0}; v[i] = uint4{0, 0, 0, 0}; }
      *(uint4*)(kt + r * M::kRowK + c) = k[i];
      *(uint4*)(vt + r * M::kRowV + c) = v[i];
    }
  }
};

template <int DT, int BITS, int N>
struct StagePacked {
  static constexpr int kBytes = kHeadDim * BITS / 8, kParts = kBytes / 16;         // 16-byte parts of a row
  static constexpr bool kSplit = N * kParts < 64;                                 // the lower 32 lanes take the K rows, the upper ones the V rows
  static constexpr int kLanes = kSplit ? 32 : 64, kLoads = N * kParts / kLanes;
  static_assert(kLoads * kLanes == N * kParts, "every row once");
  uint4 k[kLoads], v[kLoads];
  uint32_t ks[kLoads], vs[kLoads];
  // rows first + r of the cache; beyond `left` rows the last one instead
  __device__ __forceinline__ void begin(const TreeArgs& a, size_t first, int left, int r0, int lane) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = i * kLanes + lane % kLanes, r = min(r0 + at / kParts, left - 1), part = at % kParts;
      const size_t row = first + r, code = row * kBytes + part * 16, scale = row * kRowScales + part * 4 / kParts;
      const bool values = kSplit && lane >= 32;
      k[i] = *(const uint4*)((const char*)(values ? a.cache.v_codes : a.cache.k_codes) + code);
      ks[i] = (values ? a.cache.v_scales : a.cache.k_scales)[scale];
      if constexpr (!kSplit) {
        v[i] = *(const uint4*)((const char*)a.cache.v_codes + code);
        vs[i] = a.cache.v_scales[scale];
      }
    }
  }
  __device__ __forceinline__ void end(char* kt, char* vt, int left, int r0, int lane) {
    using M = Mma<DT>;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = i * kLanes + lane % kLanes, r = r0 + at / kParts, c = at % kParts * (M::kRow / kParts);
      const bool ok = r < left;
      char *kto = kt + r * M::kRowK + c, *vto = vt + r * M::kRowV + c;
      if constexpr (kSplit) kto = lane >= 32 ? vto : kto;
      spread<DT, BITS>(kto, ok ? k[i] : uint4{0, 0, 0, 0}, ok ? scale_value(ks[i]) : 0.f);
      if constexpr (!kSplit) spread<DT, BITS>(vto, ok ? v[i] : uint4{0, 0, 0, 0}, ok ? scale_value(vs[i]) : 0.f);
    }
  }
};
template <int DT, int N> struct Stage<DT, kPacked8, N> : StagePacked<DT, 8, N> {};
template <int DT, int N> struct Stage<DT, kPacked4, N> : StagePacked<DT, 4, N> {};

// Rows of the drafted tokens, as Stage has those of the entries; `bad` gets a bit for every row with a value that is not finite, which goes in
// as zero.
template <int DT, int N>
struct Drafts {
  using M = Mma<DT>;
  static constexpr int kPer = 64 * 16 / M::kRow, kLoads = N / kPer;
  uint4 k[kLoads], v[kLoads];
  __device__ __forceinline__ void begin(const TreeArgs& a, size_t first, int left, int r0, int lane) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const size_t at = (first + max(0, min(r0 + i * kPer + lane * 16 / M::kRow, left - 1))) * M::kRow + lane % (M::kRow / 16) * 16;
      k[i] = *(const uint4*)((const char*)a.K1 + at);
      v[i] = *(const uint4*)((const char*)a.V1 + at);
    }
  }
  __device__ __forceinline__ void end(char* kt, char* vt, int left, int r0, int lane, unsigned long long& bad) {
    uint32_t any = 0;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) any |= M::not_finite(v[i].x) | M::not_finite(v[i].y) | M::not_finite(v[i].z) | M::not_finite(v[i].w);
    if (__any(any != 0)) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = r0 + i * kPer + lane * 16 / M::kRow;
        bool b = false;
        v[i] = M::only_finite(v[i], b);
        const unsigned long long rows = __ballot(b && r < left);
#pragma unroll
        for (int z = 0; z < kPer; ++z)
          if ((rows >> (z * (64 / kPer))) & (~0ull >> (64 - 64 / kPer))) bad |= 1ull << (r0 + i * kPer + z);
      }
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int r = r0 + i * kPer + lane * 16 / M::kRow, c = lane % (M::kRow / 16) * 16;
      if (r >= left) { k[i] = uint4{0, 0, 0, 0}; v[i] = uint4{0, 0, 0, 0}; }
      *(uint4*)(kt + r * M::kRowK + c) = k[i];
      *(uint4*)(vt + r * M::kRowV + c) = v[i];
    }
  }
};

// A workgroup of W wavefronts, one per compute unit: WR of them take 32 rows each and share tiles of kSlots entries; W / WR such groups take
// the tiles in turn.  Shared tiles have two places, of which one is filled while the other is read, with one barrier per tile.  A wavefront
// that has its tiles alone (up to 32 rows: bound by memory) keeps 32 rows of K and V on their way in registers: 128 KB per compute unit.
// Measured after 30 ms of work (a card that was idle takes up to a quarter longer until then): 8 units of 131072 entries in 8 bits, one node of
// 8 heads: 56 us, 4.9 TB/s of codes and scales.  112 units of 2048 gathered entries and 427 rows: 83 us; the matrix units are busy 34 % of that, vector
// instructions 44 %, LDS 36 %: no unit alone bounds it.  The two wavefronts of a SIMD half a round apart, one reading keys while the other takes
// exponentials (two barriers a round), took 87 where this order took 79, both with one sum of the weights.
template <int DT, int SRC, int WR>
struct Shape {
  static constexpr int W = DT == DYNAKV_F32 ? 4 : 8, kThreads = 64 * W;
  static constexpr int kGroups = W / WR, kSlots = WR >= 4 ? 2 * kSub : kSub, kPlaces = WR == 1 ? 1 : 2;
  static constexpr int kMine = kSlots / WR;                                                         // rows of a tile that a wavefront loads
  static constexpr int kTileK = kSlots * Mma<DT>::kRowK, kTileV = kSlots * Mma<DT>::kRowV, kTile = kTileK + kTileV + kSlots * 4;   // bytes: K, V, bias
  static constexpr int kOut = kHeadDim + 4;                                                         // floats of a row in the merge
  static constexpr int kMerge = W * kSub * kOut * 4, kTiles = kGroups * kPlaces * kTile, kLds = kTiles > kMerge ? kTiles : kMerge;
  static_assert(kLds <= 163840 - 256, "LDS of a compute unit");
};

template <int DT, int SRC, int WR>
__global__ __launch_bounds__((Shape<DT, SRC, WR>::kThreads)) void tree_kernel(TreeArgs a) {
  using M = Mma<DT>;
  using Sh = Shape<DT, SRC, WR>;
  constexpr int kOut = Sh::kOut, kSlots = Sh::kSlots, N = kSlots / kSub, kGroups = Sh::kGroups, W = Sh::W;
  extern __shared__ __align__(16) char lds[];
  __shared__ unsigned long long sbad[W];
  // workgroups with the same entries run on the same XCD, one after the other: they share its L2
  const int piece = ((int)blockIdx.x >> 3) / a.RB * 8 + ((int)blockIdx.x & 7), rb = ((int)blockIdx.x >> 3) % a.RB;
  if (piece >= a.pieces) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int grp = wave / WR, wr = wave % WR;
  const int R = a.T * a.G, row = rb * a.rows + wr * kSub + (lane & 31);
  const bool some = WR == 1 || (wr * kSub < a.rows && rb * a.rows + wr * kSub < R);      // else the wavefront only helps to load
  const Piece pc = piece_of<SRC>(a, piece, lane);
  if (pc.u < 0) return;
  const int u = __builtin_amdgcn_readfirstlane(pc.u), ns = __builtin_amdgcn_readfirstlane(pc.count), s = __builtin_amdgcn_readfirstlane(pc.s);
  const int L = __builtin_amdgcn_readfirstlane(pc.slots);
  [[maybe_unused]] const int nlist = L / 4;
  const int nt = (L + kSlots - 1) / kSlots, t0 = (int)((long long)nt * s / ns), t1 = (int)((long long)nt * (s + 1) / ns);
  if (a.pieces != a.U && rb == 0 && s == 0 && threadIdx.x == 0) {      // for the kernel that joins
    a.where[2 * u] = __builtin_amdgcn_readfirstlane(pc.first);
    a.where[2 * u + 1] = ns;
  }

  // The queries, the drafted tokens and the first tile are requested together.  The drafted tokens are the unit's last piece's, there of the last
  // groups, which have the fewest tiles (of the first ones: 20.3 us for a float32 unit of 256 entries and five tokens; so 15.3).
  typename M::Q q;
  M::load_q(q, a.Q, (size_t)u * R + min(row, R - 1), h);      // (rows beyond the last: its queries; not written)
  const int r0 = wr * Sh::kMine, j0 = (kGroups - 1 - grp) * kSlots;
  const bool drafts = a.K1 && s == ns - 1, mine = drafts && j0 < a.T;
  unsigned long long word = 0;
  Drafts<DT, Sh::kMine> draft;
  auto node_bits = [&] {
    const int node = min(row, R - 1) / a.G;
    const unsigned long long w = a.tree ? a.tree[(size_t)u * a.T + node] : ~0ull >> (63 - node);
    return a.T < 64 ? w & ((1ull << a.T) - 1) : w;
  };
  if (mine) {
    draft.begin(a, (size_t)u * a.T + j0, a.T - j0, r0, lane);
    word = node_bits() >> j0;
  }

  Rows st;
  st.m = -__builtin_inff(); st.l = 0.f; st.w[0] = st.w[1] = 0.f;
#pragma unroll
  for (int d = 0; d < 4; ++d) st.o[d] = f16v{};
  char* tiles = lds + grp * Sh::kPlaces * Sh::kTile;

  // a wavefront's own tile needs no barrier: its LDS operations keep their order, and so must the compiler
  auto sync = [] {
    if constexpr (WR == 1) asm volatile("" ::: "memory");
    else lds_barrier();
  };
  const char* pages = a.pages + (size_t)u * a.unit_pages;
  const int* plist = a.plist + (size_t)u * a.Lcap;
  const size_t first = (size_t)u * a.cache.capacity;
  // List entry lane / 4 of tile t.  It is requested one tile before the tile's rows are, so that neither waits for the other, and looked
  // at only there: a conditional load here, or a copy of what is on its way, would wait for every load before it.
  auto entry_index = [&](int t) { return t * (kSlots / 4) + (lane >> 2) % (kSlots / 4); };
  Stage<DT, SRC, Sh::kMine> stage;
  constexpr unsigned long long kAll = kSlots == 64 ? ~0ull : 0xFFFFFFFFull;
  int t = t0 + grp, entry = 0;
  unsigned long long seen_next = 0;                  // slots of the tile on its way that hold an entry
  auto request_entry = [&](int tile) {
    if constexpr (SRC == kList) entry = plist[min(entry_index(tile), nlist - 1)];
  };
  auto begin = [&](int tile) {
    if constexpr (SRC == kList) {
      const int e = entry_index(tile) < nlist ? entry : -1;
      seen_next = __ballot(e >= 0 && (lane & 3) <= (e & 3)) & kAll;
      stage.begin(a, pages, e, r0, lane);
      request_entry(tile + kGroups);
    } else {
      const int left = L - tile * kSlots;
      seen_next = left >= kSlots ? kAll : (1ull << left) - 1;
      stage.begin(a, first + (size_t)tile * kSlots, left, r0, lane);
    }
  };
  auto end = [&](int tile, int place) {
    char* kt = tiles + place * Sh::kTile;
    if (lane < Sh::kMine) ((float*)(kt + Sh::kTileK + Sh::kTileV))[r0 + lane] = (seen_next >> (r0 + lane)) & 1 ? 0.f : -__builtin_inff();
    if constexpr (SRC == kList) stage.end(kt, kt + Sh::kTileK, seen_next, seen_next == kAll, r0, lane);
    else stage.end(kt, kt + Sh::kTileK, L - tile * kSlots, r0, lane);
  };
  constexpr int kLast = Sh::kPlaces - 1;
  unsigned long long bad = 0;
  if (t < t1) {
    request_entry(t);
    begin(t);
  }
  if (mine) {                                        // the drafted tokens, to the last place
    char* to = tiles + kLast * Sh::kTile;
    draft.end(to, to + Sh::kTileK, a.T - j0, r0, lane, bad);
    if (lane < Sh::kMine) ((float*)(to + Sh::kTileK + Sh::kTileV))[r0 + lane] = 0.f;
    if constexpr (WR > 1) sbad[wave] = bad;          // of the wavefront's share of the rows
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);                // vmcnt(0): the queries are there, and no round waits for them with a tile on its way
  sync();
  // Round i reads the tiles of place i & 1 (where there are two), writes the next ones to the other and requests those after them; round -1 reads
  // the drafted tokens.  One copy of the code for all of them: a workgroup's first rounds run from a cold instruction cache.
  const int rounds = (t1 - t0 + kGroups - 1) / kGroups;      // of the whole workgroup: barriers are common
  t -= kGroups;
  for (int i = -1; i < rounds; ++i, t += kGroups) {
    char* kt = tiles + (kLast ? i & 1 : 0) * Sh::kTile;
    auto next = [&] {
      if (t + kGroups < t1) {
        end(t + kGroups, kLast ? (i + 1) & 1 : 0);
        if (t + 2 * kGroups < t1) begin(t + 2 * kGroups);
      }
    };
    if constexpr (kLast) next();                     // into the other place
    if (some && (i < 0 ? mine : kGroups == 1 || t < t1))
      consume<DT, N>(st, kt, kt + Sh::kTileK, (const float*)(kt + Sh::kTileK + Sh::kTileV), q, i < 0, word, a.sc, lane);
    sync();
    if constexpr (!kLast) {
      next();
      sync();
    }
  }
  if constexpr (WR > 1) {
    bad = 0;
    if (mine)
      for (int w = 0; w < WR; ++w) bad |= sbad[grp * WR + w];
  }

  // Values of drafted tokens that are not finite went in as zeros, so that a row which does not see their token stays clean of them; the
  // rows that see it get them here.
  if (bad) {
    const unsigned long long sees = node_bits() >> j0;
    while (bad) {
      const int j = __builtin_ctzll(bad);
      bad &= bad - 1;
      const size_t at = ((size_t)u * a.T + j0 + j) * kHeadDim;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float x = M::elem(a.V1, at + 32 * d + entry_of(i, 0) + 4 * h);
          if (((sees >> j) & 1u) && !(fabsf(x) < __builtin_inff())) st.o[d][i] += x;
          if (i % 8 == 7) hold_order();
        }
    }
  }

  // join the groups: every wavefront leaves its rows in LDS
  const auto lsum = __builtin_amdgcn_permlane32_swap(__float_as_uint(st.l), __float_as_uint(st.l), false, false);
  st.l = __uint_as_float(lsum[0]) + __uint_as_float(lsum[1]);
  const float half = st.w[0] + st.w[1];
  const auto wsum = __builtin_amdgcn_permlane32_swap(__float_as_uint(half), __float_as_uint(half), false, false);
  lds_barrier();
  float* mo = (float*)lds;
  {
    float* at = mo + ((size_t)wave * kSub + (lane & 31)) * kOut;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4) *(f4*)(at + 32 * d + entry_of(i, h)) = f4{st.o[d][i], st.o[d][i + 1], st.o[d][i + 2], st.o[d][i + 3]};
    if (h == 0) { at[kHeadDim] = st.m; at[kHeadDim + 1] = st.l; at[kHeadDim + 2] = __uint_as_float(wsum[0]) + __uint_as_float(wsum[1]); }
  }
  lds_barrier();
  for (int i = threadIdx.x; i < WR * kSub * (kHeadDim / 4); i += Sh::kThreads) {
    const int r = i >> 5, c = (i & 31) * 4, rr = rb * a.rows + r;      // row r of the workgroup: wavefront r / 32 of every group
    if (r >= a.rows || rr >= R) break;
    float mw[kGroups], m = -__builtin_inff(), l = 0.f, sum = 0.f;
#pragma unroll
    for (int w = 0; w < kGroups; ++w) { mw[w] = mo[(w * WR * kSub + r) * kOut + kHeadDim]; m = fmaxf(m, mw[w]); }
    f4 o = {0, 0, 0, 0};
#pragma unroll
    for (int w = 0; w < kGroups; ++w) {
      const float* x = mo + (w * WR * kSub + r) * kOut;
      if (saw_nothing(mw[w], x[kHeadDim + 1])) continue;
      const float f = mw[w] == m ? 1.f : __builtin_amdgcn_exp2f(mw[w] - m);
      l += f * x[kHeadDim + 1];
      sum += f * x[kHeadDim + 2];
      o += f * *(const f4*)(x + c);
    }
    const size_t to = (size_t)u * R + rr;
    if (ns == 1) {
      const bool none = saw_nothing(m, l);
      M::store4(a.out, to * kHeadDim + c, none ? f4{0, 0, 0, 0} : o / sum);
      if (a.lse && c == 0) a.lse[to] = none ? m : (m + __builtin_amdgcn_logf(l)) * kLn2;
    } else {
      float* p = a.part + ((size_t)piece * R + rr) * kPartRow;
      *(f4*)(p + c) = o;
      if (c == 0) { p[kHeadDim] = m; p[kHeadDim + 1] = l; p[kHeadDim + 2] = sum; }
    }
  }
}

// Joins the pieces of the units that have several, in their order.  P groups of 32 lanes share a row and take eight pieces at once (64 of
// them one after the other, each a trip to memory, took 52 us).
template <int DT, int P>
__global__ __launch_bounds__(256) void tree_join_kernel(TreeArgs a) {
  __shared__ __align__(16) float sm[8][kPartRow];
  const int R = a.T * a.G, c = (threadIdx.x & 31) * 4, grp = threadIdx.x >> 5;
  const size_t i = (size_t)blockIdx.x * (8 / P) + grp / P;
  if (P < 8 && i >= (size_t)a.U * R) return;
  const int u = (int)(i / R), r = (int)(i % R);
  const int first = a.where[2 * u], ns = a.where[2 * u + 1];
  if (ns == 1) return;                               // (P = 8: the whole workgroup)
  const float* p = a.part + ((size_t)first * R + r) * kPartRow;
  float ms[8], ls[8], ws[8], m = -__builtin_inff(), l = 0.f, w = 0.f;
  f4 os[8], o = {0, 0, 0, 0};
  auto add = [&](float mk, float lk, float wk, const f4& ok) {
    if (saw_nothing(mk, lk)) return;
    const float f = mk == m ? 1.f : __builtin_amdgcn_exp2f(mk - m);
    l += f * lk;
    w += f * wk;
    o += f * ok;
  };
  for (int s0 = grp % P; s0 < ns; s0 += 8 * P) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int s = s0 + P * k;
      const float* x = p + (size_t)min(s, ns - 1) * R * kPartRow;
      ms[k] = s < ns ? x[kHeadDim] : -__builtin_inff();
      ls[k] = s < ns ? x[kHeadDim + 1] : 0.f;
      ws[k] = x[kHeadDim + 2];
      os[k] = *(const f4*)(x + c);
    }
    float top = m;
#pragma unroll
    for (int k = 0; k < 8; ++k) top = fmaxf(top, ms[k]);
    const float f = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top);
    m = top;
    l *= f;
    w *= f;
    o *= f;
#pragma unroll
    for (int k = 0; k < 8; ++k) add(ms[k], ls[k], ws[k], os[k]);
  }
  if constexpr (P == 8) {
    *(f4*)&sm[grp][c] = o;
    if (c == 0) { sm[grp][kHeadDim] = m; sm[grp][kHeadDim + 1] = l; sm[grp][kHeadDim + 2] = w; }
    __syncthreads();
    if (grp > 0) return;
    m = -__builtin_inff(); l = 0.f; w = 0.f;
    o = f4{0, 0, 0, 0};
#pragma unroll
    for (int k = 0; k < 8; ++k) m = fmaxf(m, sm[k][kHeadDim]);
#pragma unroll
    for (int k = 0; k < 8; ++k) add(sm[k][kHeadDim], sm[k][kHeadDim + 1], sm[k][kHeadDim + 2], *(const f4*)&sm[k][c]);
  }
  const bool none = saw_nothing(m, l);
  Mma<DT>::store4(a.out, i * kHeadDim + c, none ? f4{0, 0, 0, 0} : o / w);
  if (a.lse && c == 0) a.lse[i] = none ? m : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Most wavefronts of a workgroup that take rows of their own, up to eight times 32 of the R rows of a unit: what they read of LDS they share with none,
// what they load and unpack with all.  R = 427, 2048 entries of 112 units: 169 us with one, 147 with two, 103 with four, 83 with eight; R = 128 of
// 128 packed units: 130, 94, 71 with four.  For 32 rows a second wavefront would be idle: 8 long packed units 60 us, with two 72.  Several blocks of
// rows are made alike (R = 427: seven wavefronts of eight twice, 82.7 us, eight and six 82.9).  A float32 wavefront's queries and sums leave room
// for one on a SIMD; its matrix instructions are what bounds it, whoever loads the tiles.
int row_waves(int dtype, int R) { return dtype == DYNAKV_F32 || R <= kSub ? 1 : R <= 2 * kSub ? 2 : R <= 4 * kSub ? 4 : 8; }

// How the work is cut: `waves` of a workgroup take rows of their own, `pieces` are the workgroups that a call gets for each block of rows, `least` the
// fewest entries for which another one is worth it.  From a model in ns, fitted to 1 to 256 units: 256 workgroups run at once; one takes 8.8 us
// and 0.7 for each of its waves to begin and end, and per entry the larger of its bytes (at its share of 5 TB/s, at most 64 per ns, 36 where waves
// share tiles) and the work of its rows, 4 for each 32 (34 for float32's matrix instructions), and 4 or (not float16) 10 to unpack; the kernel that
// joins takes 6 us.  Units of one length would be cut into s pieces each; a multiple of 256 workgroups that has room for those is what units of any
// lengths share, which then weigh three quarters of the longest.  (8 units of 131072 packed entries: 60 us, whole 1270; 128 units of up to 8191: 71,
// whole 108.)  Fewer waves than there could be make more blocks of rows, for chips that would be idle otherwise: 5 units of 352 rows and 272
// entries 11 us (as many waves as could be: 19), 81 of 255 and 417 22 (34), 140 of 336 and 761 54 (73).
// The model's own numbers, over 60 calls of the sizes of a batch: another cut for 3 % (or for any gain, or for 10 %), half or all of the longest instead of
// three quarters, at most two or eight rounds: 1 % on the mean either way, single calls 8 % shorter to 6 % longer.  Fewer waves for 10 %: for any
// gain 1 % either way, for 25 % single calls take up to 1.58 times as long.
// More than kPlanUnits units fill the chip whole: 700 of up to 4096 packed entries 119 us, shared 133; 1000: 157, 193; alike 158, 174 and 224, 237.
struct Plan { int waves, pieces, least; };
constexpr int kMostRounds = 4;                       // bounds the scratch
// Fewer waves than there could be make at most this many workgroups of 512: a launch has fewer than 2^32 work-items.  (As many as could be make a
// workgroup per unit and every further 256 rows, which the limits of the call keep below that.)
constexpr long long kMostBlocks = 1ll << 22;
int row_blocks(int waves, int R) { return (R + waves * kSub - 1) / (waves * kSub); }
bool may_share(int waves, int U, int R) { return U <= kPlanUnits && (long long)U * row_blocks(waves, R) <= 2 * kWorkgroups; }
// Rounds of the chip: the blocks of rows of a piece run on one XCD, of which each takes every eighth piece (84 pieces of three blocks are 33
// workgroups on some of them: 37 us where 56 take 28).
constexpr int kXcds = 8, kPerXcd = kWorkgroups / kXcds;
long long rounds_of(long long pieces, int blocks) { return ((pieces + kXcds - 1) / kXcds * blocks + kPerXcd - 1) / kPerXcd; }
int pieces_for(int waves, int U, int R, int s) {     // a unit of s pieces: 0: more rounds than there may be
  const int blocks = row_blocks(waves, R);
  const long long rounds = rounds_of((long long)U * s, blocks);
  return rounds > kMostRounds ? 0 : max(U, kXcds * (kPerXcd * (int)rounds / blocks));
}
Plan plan(int dtype, int bytes, bool packed, int U, int R, long long most, bool ragged) {
  Plan best = {0, 0, 1};
  double least_time = 0.0;
  for (int waves = row_waves(dtype, R); waves >= 1; waves /= 2) {
    const int blocks = row_blocks(waves, R);
    const long long n = (long long)U * blocks;
    if (best.waves && n > kMostBlocks) break;
    const double work = dtype == DYNAKV_F32 ? 34.0 : 4.0 * waves + (!packed ? 0.0 : dtype == DYNAKV_F16 ? 4.0 : 10.0);
    auto entry = [&](long long workgroups) {
      const double share = 5120.0 / (double)std::min<long long>(workgroups, kWorkgroups), b = bytes / std::min(share, waves == 1 ? 64.0 : 36.0);
      return std::max(b, work);
    };
    const bool cut = may_share(waves, U, R) && entry(n) * (double)most >= 8e3;
    int pieces = 1;
    double time = 0.0;
    for (int s = 1; s == 1 || (cut && s <= 64 && pieces_for(waves, U, R, s)); ++s) {
      const double longest = (ragged && s > 1 ? 0.75 : 1.0) * (double)most / s;
      const double t = (double)rounds_of((long long)U * s, blocks) * (8.8e3 + 700.0 * waves + entry(n * s) * longest) + (s > 1 ? 6e3 : 0.0);
      if (s == 1 || t < 0.97 * time) { pieces = s; time = t; }
    }
    if (best.waves && time > 0.9 * least_time) continue;
    least_time = time;
    const int all = cut && (pieces > 1 || ragged) ? pieces_for(waves, U, R, pieces) : 0;
    best = all ? Plan{waves, all, (int)(4e3 / entry(kWorkgroups)) + 1} : Plan{waves, U, 1};
  }
  return best;
}

template <int DT, int SRC, int WR>
hipError_t launch_shape(TreeArgs& a, hipStream_t st) {
  using Sh = Shape<DT, SRC, WR>;
  const int R = a.T * a.G;
  a.RB = (R + WR * kSub - 1) / (WR * kSub);
  a.rows = ((R + kSub - 1) / kSub + a.RB - 1) / a.RB * kSub;
  tree_kernel<DT, SRC, WR><<<(unsigned)((a.pieces + 7ll) / 8 * 8 * a.RB), Sh::kThreads, Sh::kLds, st>>>(a);
  return hipGetLastError();
}

template <int DT, int SRC>
hipError_t launch_source(TreeArgs& a, int wr, hipStream_t st) {
  if constexpr (DT == DYNAKV_F32) {
    return launch_shape<DT, SRC, 1>(a, st);
  } else {
    return wr == 1   ? launch_shape<DT, SRC, 1>(a, st)
           : wr == 2 ? launch_shape<DT, SRC, 2>(a, st)
           : wr == 4 ? launch_shape<DT, SRC, 4>(a, st)
                     : launch_shape<DT, SRC, 8>(a, st);
  }
}

template <int DT>
hipError_t launch(TreeArgs a, hipStream_t st) {
  const int R = a.T * a.G, bytes = a.pages ? 2 * Mma<DT>::kRow : 2 * (kHeadDim * a.cache.bits / 8 + kRowScales);
  const Plan p = plan(DT, bytes, !a.pages, a.U, R, a.most, !a.pages && a.lengths);
  a.pieces = p.pieces;
  a.least = p.least;
  const hipError_t e = a.pages ? launch_source<DT, kList>(a, p.waves, st)
                               : a.cache.bits == 8 ? launch_source<DT, kPacked8>(a, p.waves, st) : launch_source<DT, kPacked4>(a, p.waves, st);
  if (e != hipSuccess || a.pieces == a.U) return e;
  // Few rows of many pieces: eight groups of lanes to a row; else one (4992 rows of 6 pieces 12 us with eight, 64 rows of 32 pieces 52 with one
  // that takes a piece at a time).
  const int each = min(a.pieces - a.U + 1, a.most / a.least + 1);
  if (each > 8 && (long long)a.U * R <= 2048) tree_join_kernel<DT, 8><<<(unsigned)((long long)a.U * R), 256, 0, st>>>(a);
  else tree_join_kernel<DT, 1><<<(unsigned)(((long long)a.U * R + 7) / 8), 256, 0, st>>>(a);
  return hipGetLastError();
}

// Scratch: where the pieces of each unit are, then a partial result of every row for each piece.  The most that any plan has: fewer waves make more
// blocks of rows, of which each gets fewer pieces.
size_t where_bytes(int U) { return ((size_t)U * 8 + 255) & ~(size_t)255; }
size_t part_bytes(int dtype, int U, int R) {
  const int waves = row_waves(dtype, R);
  if (!may_share(waves, U, R)) return 0;
  const int most = kMostRounds * kWorkgroups / row_blocks(waves, R);
  return (size_t)(most > U ? most : U) * R * kPartRow * sizeof(float);
}

}  // namespace

size_t tree_scratch_bytes(int U, int T, int G) {
  const size_t a = part_bytes(DYNAKV_F16, U, T * G), b = part_bytes(DYNAKV_F32, U, T * G);
  return where_bytes(U) + (a > b ? a : b);
}

hipError_t launch_tree(const TreeArgs& in, hipStream_t st) {
  TreeArgs a = in;
  a.where = (int*)a.scratch;
  a.part = (float*)((char*)a.scratch + where_bytes(a.U));
  if (a.dtype == DYNAKV_F32) return launch<DYNAKV_F32>(a, st);
  if (a.dtype == DYNAKV_F16) return launch<DYNAKV_F16>(a, st);
  return launch<DYNAKV_BF16>(a, st);
}

}  // namespace dynakv
