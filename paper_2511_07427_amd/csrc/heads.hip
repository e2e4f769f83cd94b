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

// Four consecutive elements (8-byte aligned for 16-bit types, 16 for float32).
template <int DT>
__device__ __forceinline__ void load4(const void* base, size_t i, float (&x)[4]) {
  if constexpr (DT == DYNAKV_F32) {
    const f4 a = *(const f4*)((const float*)base + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = a[e];
  } else {
    const us4 a = *(const us4*)((const uint16_t*)base + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = DT == DYNAKV_F16 ? f16_to_float(a[e]) : bf16_to_float(a[e]);
  }
}
template <int DT>
__device__ __forceinline__ void store4(void* base, size_t i, const float (&x)[4]) {
  if constexpr (DT == DYNAKV_F32) {
    *(f4*)((float*)base + i) = f4{x[0], x[1], x[2], x[3]};
  } else {
    us4 a;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      a[e] = DT == DYNAKV_F16 ? __builtin_bit_cast(uint16_t, (_Float16)x[e]) : __builtin_bit_cast(uint16_t, (__bf16)x[e]);
    *(us4*)((uint16_t*)base + i) = a;
  }
}

// Sum over a row of 16 lanes, the same bits in every lane.
__device__ __forceinline__ float row16_sum(float x) {
  auto add = [&](int y) { x += __int_as_float(y); };
  add(dpp_or<kDppXor1>(0, __float_as_int(x)));
  add(dpp_or<kDppXor2>(0, __float_as_int(x)));
  add(dpp_or<kDppHalfMirror>(0, __float_as_int(x)));
  add(dpp_or<kDppMirror>(0, __float_as_int(x)));
  return x;
}

// grid (tokens, chunks of heads); 16 rows at a time, `per` of them by each row of 16 lanes.
template <int DT>
__global__ __launch_bounds__(256) void norm_rope_kernel(HeadsArgs a) {
  const dynakv_heads_t& c = a.c;
  const int b = blockIdx.x / c.n_tokens, t = blockIdx.x % c.n_tokens;
  const int pos = a.positions[blockIdx.x];
  if (pos < 0) return;
  const int lane = threadIdx.x & 15, row = threadIdx.x >> 4;
  const int H = c.n_kv_heads, G = c.group_size, nq = H * G, heads = nq + 2 * H, rot = c.rotary_dim;
  const bool turns = 8 * lane < rot;
  // the lane's two runs of four elements
  const bool apart = !c.interleaved && rot > 0;      // pairs half the rotated part apart
  const int i0 = apart ? (turns ? 4 * lane : 8 * lane) : 8 * lane, i1 = apart && turns ? rot / 2 + 4 * lane : i0 + 4;
  float cs[4], sn[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    cs[e] = 1.f; sn[e] = 0.f;
    if (turns) {
      double r = (double)pos * (double)a.inv_freq[4 * lane + e] * 0.15915494309189533577;
      r -= rint(r);
      sincospif(2.f * (float)r, &sn[e], &cs[e]);
    }
  }
  const int h0 = blockIdx.y * 16 * a.per + row;
  for (int k = 0; k < a.per; ++k) {
    const int h = h0 + 16 * k;
    if (h >= heads) break;
    const int what = h < nq ? 0 : h < nq + H ? 1 : 2, hh = what == 0 ? h : what == 1 ? h - nq : h - nq - H;
    const void* src = what == 0 ? a.q : what == 1 ? a.k : a.v;
    if (!src) continue;
    const int64_t ss = what == 0 ? c.q_seq_stride : what == 1 ? c.k_seq_stride : c.v_seq_stride;
    const int64_t st = what == 0 ? c.q_token_stride : what == 1 ? c.k_token_stride : c.v_token_stride;
    const size_t from = (size_t)((int64_t)b * ss + (int64_t)t * st) + (size_t)hh * kHeadDim;
    float x[4], y[4];
    load4<DT>(src, from + i0, x);
    load4<DT>(src, from + i1, y);
    size_t to;
    if (what == 0) to = (((size_t)(b * H + hh / G) * c.n_tokens + t) * G + hh % G) * kHeadDim;
    else to = ((size_t)(b * H + hh) * c.n_tokens + t) * kHeadDim;
    if (what < 2) {
      const void* w = what == 0 ? a.wq : a.wk;
      if (w) {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) s += x[e] * x[e];
#pragma unroll
        for (int e = 0; e < 4; ++e) s += y[e] * y[e];
        const float r = rsqrtf(row16_sum(s) * (1.f / kHeadDim) + c.eps);
        float wx[4], wy[4];
        load4<DT>(w, i0, wx);
        load4<DT>(w, i1, wy);
#pragma unroll
        for (int e = 0; e < 4; ++e) { x[e] = x[e] * r * wx[e]; y[e] = y[e] * r * wy[e]; }
      }
      if (turns) {
        if (apart) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float p = x[e], q = y[e];
            x[e] = p * cs[e] - q * sn[e];
            y[e] = q * cs[e] + p * sn[e];
          }
        } else {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float p = x[2 * e], q = x[2 * e + 1], r = y[2 * e], s = y[2 * e + 1];
            x[2 * e] = p * cs[e] - q * sn[e];
            x[2 * e + 1] = q * cs[e] + p * sn[e];
            y[2 * e] = r * cs[2 + e] - s * sn[2 + e];
            y[2 * e + 1] = s * cs[2 + e] + r * sn[2 + e];
          }
        }
      }
    }
    void* dst = what == 0 ? a.Q : what == 1 ? a.K : a.V;
    store4<DT>(dst, to + i0, x);
    store4<DT>(dst, to + i1, y);
  }
}

}  // namespace

hipError_t launch_norm_rope(const HeadsArgs& in, hipStream_t st) {
  HeadsArgs a = in;
  const int heads = a.c.n_kv_heads * (a.c.group_size + 2);
  const size_t tokens = (size_t)a.c.n_seqs * a.c.n_tokens;
  a.per = 1;
  const dim3 grid((unsigned)tokens, (heads + 16 * a.per - 1) / (16 * a.per));
  if (a.c.dtype == DYNAKV_F32) norm_rope_kernel<DYNAKV_F32><<<grid, 256, 0, st>>>(a);
  else if (a.c.dtype == DYNAKV_F16) norm_rope_kernel<DYNAKV_F16><<<grid, 256, 0, st>>>(a);
  else norm_rope_kernel<DYNAKV_BF16><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace dynakv
