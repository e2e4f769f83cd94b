// Norm of queries and keys per head, their rotation by position, and the layout by unit (dynakv_norm_rope).
//
// y = x * rsqrt(mean(x^2) + eps) * w; pair (a, b) of index i -> (a cos t - b sin t, b cos t + a sin t), t = pos * inv_freq[i].
// Every row is read and written once: the kernel is bound by memory.  16 lanes hold a row of 128 elements, 8 each, chosen so
// that both members of a pair are in one lane: no lane needs a neighbour's element, and only the sum of squares crosses
// lanes.  The angles belong to the token: a lane takes sine and cosine of its four pairs once for all the heads it works on.
// t is reduced in float64, in turns: of a position of 10^5 float32 would leave the angle an error of 10^-2.
#include "common.hpp"
#include "operators.hpp"

namespace dynakv {

namespace {

typedef uint16_t us4 __attribute__((ext_vector_type(4)));

// Sum over a row of 16 lanes, the same bits in every lane.
__device__ __forceinline__ float row16_sum(float x) {
  auto add = [&](int y) { x += __int_as_float(y); };
  add(dpp_or<kDppXor1>(0, __float_as_int(x)));
  add(dpp_or<kDppXor2>(0, __float_as_int(x)));
  add(dpp_or<kDppHalfMirror>(0, __float_as_int(x)));
  add(dpp_or<kDppMirror>(0, __float_as_int(x)));
  return x;
}

// How a lane's eight elements of a row lie: kNear: 8 l .. 8 l + 7 (neighbouring pairs, or no rotation); kHalf: the whole head is rotated in pairs
// 64 apart: the lane loads those eight too, and lanes l and l + 8 exchange four of them; kApart: other pairs rotary_dim / 2 apart: two runs of four,
// loaded as they are needed (16384 tokens of 80 bfloat16 rows: 160 us so, 148 with the exchange).
enum Order { kNear, kHalf, kApart };

// Four elements as they lie in memory.
template <int DT>
struct Four;
template <>
struct Four<DYNAKV_F32> {
  typedef f4 T;
  static __device__ __forceinline__ void get(T a, float (&x)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = a[e];
  }
  static __device__ __forceinline__ T put(const float (&x)[4]) { return f4{x[0], x[1], x[2], x[3]}; }
};
template <int DT>
struct Four16 {
  typedef us4 T;
  static __device__ __forceinline__ void get(T a, float (&x)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = DT == DYNAKV_F16 ? f16_to_float(a[e]) : bf16_to_float(a[e]);
  }
  static __device__ __forceinline__ T put(const float (&x)[4]) {
    us4 a;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      a[e] = DT == DYNAKV_F16 ? __builtin_bit_cast(uint16_t, (_Float16)x[e]) : __builtin_bit_cast(uint16_t, (__bf16)x[e]);
    return a;
  }
};
template <> struct Four<DYNAKV_F16> : Four16<DYNAKV_F16> {};
template <> struct Four<DYNAKV_BF16> : Four16<DYNAKV_BF16> {};

// The four elements of the lane eight lanes away in the row of 16.
template <class T>
__device__ __forceinline__ T across(T x) {
  constexpr int n = sizeof(T) / 4;
  int w[n];
  __builtin_memcpy(w, &x, sizeof(T));
#pragma unroll
  for (int i = 0; i < n; ++i) w[i] = __builtin_amdgcn_update_dpp(0, w[i], 0x128, 0xF, 0xF, false);   // row_ror:8
  __builtin_memcpy(&x, w, sizeof(T));
  return x;
}
// kHalf: (elements 8 l .., 8 l + 4 ..) of lanes l and l + 8 <-> a lane's four first and four second members of pairs.  Its own inverse.
template <class T>
__device__ __forceinline__ void exchange(T& x, T& y, bool upper) {
  const T got = across(upper ? x : y);
  if (upper) x = got;
  else y = got;
}

// Workgroup (16 / HP tokens, chunk of HP a.per heads); HP rows of 16 lanes belong to a token, each takes `per` heads, kBatch of them on their way
// at once.  All rows go the same way through the code, values too (their result is dropped): with branches and 64-bit address arithmetic per
// kind of row the kernel had as much to issue as to move (191 us for 16384 tokens of 80 bfloat16 rows; now 134, 5.0 TB/s).
template <int DT, int ORDER, int HP, bool STREAM>
__global__ __launch_bounds__(256) void norm_rope_kernel(HeadsArgs a) {
  using F = Four<DT>;
  typedef typename F::T T;
  constexpr int kBatch = 4;
  constexpr size_t kRowBytes = kHeadDim / 4 * sizeof(T);
  const dynakv_heads_t& c = a.c;
  const int lane = threadIdx.x & 15, row = (threadIdx.x >> 4) % HP;
  const int token = HP == 16 ? (int)blockIdx.x : (int)blockIdx.x * (16 / HP) + (int)(threadIdx.x >> 4) / HP;
  if (HP < 16 && token >= c.n_seqs * c.n_tokens) return;
  const int b = token / c.n_tokens, t = token % c.n_tokens;
  const int pos = a.positions[token];
  if (pos < 0) return;
  const int H = c.n_kv_heads, G = c.group_size, nq = H * G, heads = nq + 2 * H, rot = c.rotary_dim;
  const bool upper = lane >= 8;
  const bool turns = 8 * lane < rot;
  // the lane's two runs of four elements in memory
  const int i0 = ORDER == kApart && turns ? 4 * lane : 8 * lane, i1 = ORDER == kApart && turns ? rot / 2 + 4 * lane : i0 + 4;
  const int pair = ORDER == kHalf ? 8 * (lane & 7) + (upper ? 4 : 0) : 4 * lane;      // the first of its four pairs

  // the token's rows: in, out, and what separates heads out there (in rows)
  const int64_t es = sizeof(T) / 4;
  const char* in[3] = {(const char*)a.q + ((int64_t)b * c.q_seq_stride + (int64_t)t * c.q_token_stride) * es,
                       (const char*)a.k + ((int64_t)b * c.k_seq_stride + (int64_t)t * c.k_token_stride) * es,
                       (const char*)a.v + ((int64_t)b * c.v_seq_stride + (int64_t)t * c.v_token_stride) * es};
  const size_t first = (size_t)b * H * c.n_tokens + t;
  char* out[3] = {(char*)a.Q + first * G * kRowBytes, (char*)a.K + first * kRowBytes, (char*)a.V + first * kRowBytes};
  const bool there[3] = {a.q != nullptr, a.k != nullptr, a.v != nullptr};
  const float per_group = 1.f / (float)G;
  const int past_group = G * (c.n_tokens - 1);
  struct Head { bool isq, isv, ok; const char* from; char* to; };
  auto head = [&](int h, int h1) {
    Head x;
    x.isq = h < nq;
    x.isv = h >= nq + H;
    const int hh = x.isq ? h : x.isv ? h - nq - H : h - nq;
    x.ok = h < h1 && (x.isq ? there[0] : x.isv ? there[2] : there[1]);
    x.from = (x.isq ? in[0] : x.isv ? in[2] : in[1]) + (size_t)((unsigned)hh * (unsigned)kRowBytes);
    const int kv = (int)(((float)hh + 0.5f) * per_group);        // hh / G (exact: hh < 2^19)
    x.to = (x.isq ? out[0] : x.isv ? out[2] : out[1]) + (size_t)(unsigned)(x.isq ? hh + kv * past_group : hh * c.n_tokens) * kRowBytes;
    return x;
  };

  const int h0 = blockIdx.y * HP * a.per + row, h1 = min(heads, (int)(blockIdx.y + 1) * HP * a.per);
  float cs[4], sn[4], w[2][8];
  for (int hb = h0; hb < h1; hb += HP * kBatch) {
    T lo[kBatch], hi[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const Head x = head(hb + HP * k, h1);
      if (!x.ok) continue;
      lo[k] = get<STREAM>((const T*)x.from + i0 / 4);
      hi[k] = get<STREAM>((const T*)x.from + i1 / 4);
    }
    if (hb == h0) {                                  // while the first rows are on their way
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const void* from = z ? a.wk : a.wq;
        float f[4] = {1.f, 1.f, 1.f, 1.f}, g[4] = {1.f, 1.f, 1.f, 1.f};
        if (from) {
          T x = ((const T*)from)[i0 / 4], y = ((const T*)from)[i1 / 4];
          if (ORDER == kHalf) exchange(x, y, upper);
          F::get(x, f);
          F::get(y, g);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) { w[z][e] = f[e]; w[z][4 + e] = g[e]; }
      }
      float freq[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) freq[e] = turns ? a.inv_freq[pair + e] : 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        double r = (double)pos * (double)freq[e] * 0.15915494309189533577;       // turns
        r -= rint(r);
        sincospif(2.f * (float)r, &sn[e], &cs[e]);
      }
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const Head d = head(hb + HP * k, h1);
      if (!d.ok) continue;
      T u = lo[k], v = hi[k];
      if (ORDER == kHalf) exchange(u, v, upper);
      float x[4], y[4];
      F::get(u, x);
      F::get(v, y);
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) s += x[e] * x[e];
#pragma unroll
      for (int e = 0; e < 4; ++e) s += y[e] * y[e];
      const bool normed = d.isq ? a.wq != nullptr : a.wk != nullptr;
      const float r = normed ? rsqrtf(row16_sum(s) * (1.f / kHeadDim) + c.eps) : 1.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = x[e] * r * (d.isq ? w[0][e] : w[1][e]);
        y[e] = y[e] * r * (d.isq ? w[0][4 + e] : w[1][4 + e]);
      }
      if (turns) {
        if (ORDER != kNear) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = x[e], q = y[e];
            x[e] = p * cs[e] - q * sn[e];
            y[e] = q * cs[e] + p * sn[e];
          }
        } else {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float p = x[2 * e], q = x[2 * e + 1], f = y[2 * e], g = y[2 * e + 1];
            x[2 * e] = p * cs[e] - q * sn[e];
            x[2 * e + 1] = q * cs[e] + p * sn[e];
            y[2 * e] = f * cs[2 + e] - g * sn[2 + e];
            y[2 * e + 1] = g * cs[2 + e] + f * sn[2 + e];
          }
        }
      }
      u = F::put(x);
      v = F::put(y);
      if (ORDER == kHalf) exchange(u, v, upper);
      put<STREAM>((T*)d.to + i0 / 4, d.isv ? lo[k] : u);
      put<STREAM>((T*)d.to + i1 / 4, d.isv ? hi[k] : v);
    }
  }
}

// Past the caches where rows in and out are more than they hold (80 rows of bfloat16 a token: 16384 tokens 148 us, so 142; 8192: 76, 70; but
// 4096, 160 MB: 35, 39, and with a kernel that reads the queries after it 54, 65).
template <int DT, int ORDER, int HP>
void launch_rows(const HeadsArgs& a, dim3 grid, hipStream_t st) {
  const long long rows = (long long)a.c.n_seqs * a.c.n_tokens * a.c.n_kv_heads * ((a.q ? a.c.group_size : 0) + (a.k ? 1 : 0) + (a.v ? 1 : 0));
  if (2 * rows * kHeadDim * elem_size(DT) > kCacheBytes) norm_rope_kernel<DT, ORDER, HP, true><<<grid, 256, 0, st>>>(a);
  else norm_rope_kernel<DT, ORDER, HP, false><<<grid, 256, 0, st>>>(a);
}

template <int DT, int ORDER>
hipError_t launch(HeadsArgs& a, hipStream_t st) {
  const int heads = a.c.n_kv_heads * (a.c.group_size + 2);
  const long long tokens = (long long)a.c.n_seqs * a.c.n_tokens;
  // Few tokens: one head to a row of lanes, so that the chip has work (one token of 48 rows 3.9 us, as many would be 4.2).  Many: the angles of a
  // token are what its rows of lanes each work out, for kBatch heads or more, so few rows share a token (5664 tokens of 9 heads: 18.6 us with 16 rows
  // each, 15.4 with 8, 12.3 with 4).
  const bool many = tokens * ((heads + 15) / 16) > 2048;
  const int hp = many ? (heads > 32 ? 16 : heads > 16 ? 8 : 4) : heads > 8 ? 16 : heads > 4 ? 8 : 4;
  a.per = many ? 8 : 1;
  const dim3 grid((unsigned)((tokens * hp + 15) / 16), (heads + hp * a.per - 1) / (hp * a.per));
  if (hp == 16) launch_rows<DT, ORDER, 16>(a, grid, st);
  else if (hp == 8) launch_rows<DT, ORDER, 8>(a, grid, st);
  else launch_rows<DT, ORDER, 4>(a, grid, st);
  return hipGetLastError();
}
template <int DT>
hipError_t launch_order(HeadsArgs& a, hipStream_t st) {
  if (a.c.interleaved || a.c.rotary_dim == 0) return launch<DT, kNear>(a, st);
  return a.c.rotary_dim == kHeadDim ? launch<DT, kHalf>(a, st) : launch<DT, kApart>(a, st);
}

}  // namespace

hipError_t launch_norm_rope(const HeadsArgs& in, hipStream_t st) {
  HeadsArgs a = in;
  return a.c.dtype == DYNAKV_F32 ? launch_order<DYNAKV_F32>(a, st) : a.c.dtype == DYNAKV_F16 ? launch_order<DYNAKV_F16>(a, st) : launch_order<DYNAKV_BF16>(a, st);
}

}  // namespace dynakv
