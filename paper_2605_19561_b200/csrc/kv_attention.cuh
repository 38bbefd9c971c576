// Attention of the new tokens of every sequence over its cached tokens:
//   x_j = cap(f q k_j) - slope |p - j|,   out = sum_j softmax(x)_j v_j,   lse = log sum_j exp(x_j)
// over the tokens j that a query at place p may see:  p - window < j <= max(p, prefix - 1),  first <= j < length.
// cap(x) = c tanh(x / c).  A query that sees nothing gets zeros and -inf.
#pragma once
#include "kv_cache.cuh"

namespace torq {

struct KvScoring {
  float scale, softcap;                  // softcap 0: none
  const float* slopes;                   // [query heads], or null
  const int32_t* prefix;                 // [batch], or null
  const int32_t* first;                  // [tokens], or null
  int window;                            // 0: none
};

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// The range [lo, hi) of cached tokens that row `i`, place p of sequence b with `length` tokens, sees.
__device__ __forceinline__ void kv_range(const KvScoring& a, int b, int i, int p, int length, int& lo, int& hi) {
  hi = lo = 0;
  if (p < 0) return;                     // a row without a place
  hi = p + 1;
  if (a.prefix && a.prefix[b] > hi) hi = a.prefix[b];
  if (hi > length) hi = length;
  if (a.window > 0 && p - a.window + 1 > 0) lo = p - a.window + 1;
  if (a.first && a.first[i] > lo) lo = a.first[i];
}
// A scaled score with what comes behind, in powers of two.
__device__ __forceinline__ float kv_score(float x, float softcap, float slope, int distance) {
  if (softcap > 0.f) {
    const float e = exp2f(fabsf(x) * (-2.f * kLog2e / softcap));
    x = copysignf(softcap * __fdividef(1.f - e, 1.f + e), x);
  }
  return (x - slope * (float)distance) * kLog2e;
}

// A lane's share of a row: DPL consecutive elements.
template <int FMT, int DPL>
__device__ __forceinline__ void kv_row_share(const uint8_t* codes, const uint8_t* scales, int lane, float ts, float (&v)[DPL]) {
  const float s = kv_scale<FMT>(scales[lane * DPL / kv_block(FMT)], ts);
  const int at = lane * (DPL / 2);
  const uint32_t w = *reinterpret_cast<const uint32_t*>(codes + (at & ~3)) >> (8 * (at & 3));
  float all[8];
  kv_codes8<FMT>(w, all);
#pragma unroll
  for (int i = 0; i < DPL; ++i) v[i] = all[i] * s;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, o);
  return v;
}

// One warp per row and head.
template <int FMT, int D>
__global__ void __launch_bounds__(128) kv_attention_simple_kernel(const KvView c, const KvScoring a, const __nv_bfloat16* Q, int64_t q_stride, int heads,
                                                                  __nv_bfloat16* out, float* lse) {
  griddep_wait_and_launch();
  constexpr int DPL = D / 32;
  const int lane = threadIdx.x & 31;
  const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (item >= (int64_t)c.tokens * heads) return;
  const int i = (int)(item / heads), h = (int)(item % heads), kvh = h / (heads / c.heads);
  float q[DPL], o[DPL] = {}, m = -INFINITY, l = 0.f;
  const int b = kv_sequence_of(c, i);
  int lo = 0, hi = 0, p = 0;
  if (b >= 0) {
    int first, count;
    kv_new_tokens(c, b, first, count);
    const int length = kv_length(c, b);
    p = length - count + i - first;
    kv_range(a, b, i, p, length, lo, hi);
  }
#pragma unroll
  for (int e = 0; e < DPL; ++e) q[e] = __bfloat162float(Q[i * q_stride + h * D + lane * DPL + e]) * a.scale;
  const float slope = a.slopes ? a.slopes[h] : 0.f;
  for (int j = lo; j < hi; ++j) {
    const int page = kv_page(c, c.table, c.width, b, j);
    if (page < 0) continue;
    const uint8_t* at = kv_head_page(c, page, kvh);
    const int slot = j & ((1 << c.page_shift) - 1);
    constexpr int blocks = D / kv_block(FMT);
    float k[DPL], v[DPL], x = 0.f;
    kv_row_share<FMT, DPL>(at + slot * (D / 2), at + c.k_scales + slot * blocks, lane, c.k_ts, k);
    kv_row_share<FMT, DPL>(at + c.v_codes + slot * (D / 2), at + c.v_scales + slot * blocks, lane, c.v_ts, v);
#pragma unroll
    for (int e = 0; e < DPL; ++e) x += q[e] * k[e];
    x = kv_score(warp_sum(x), a.softcap, slope, abs(p - j));
    const float top = fmaxf(m, x), old = exp2f(m - top), w = exp2f(x - top);
    m = top;
    l = l * old + w;
#pragma unroll
    for (int e = 0; e < DPL; ++e) o[e] = o[e] * old + w * v[e];
  }
#pragma unroll
  for (int e = 0; e < DPL; ++e) out[item * D + lane * DPL + e] = __float2bfloat16(l > 0.f ? o[e] / l : 0.f);
  if (lse && lane == 0) lse[item] = l > 0.f ? (m + log2f(l)) * kLn2 : -INFINITY;
}

// One warp per cached token and head: what the queries of its sequence gave it, added to what it had (new tokens had nothing).
template <int FMT, int D>
__global__ void __launch_bounds__(128) kv_weights_simple_kernel(const KvView c, const KvScoring a, const __nv_bfloat16* Q, int64_t q_stride, int heads,
                                                                const float* lse, const float* weights, float* weights_out) {
  griddep_wait_and_launch();
  constexpr int DPL = D / 32;
  const int lane = threadIdx.x & 31, kvh = blockIdx.y % c.heads, b = blockIdx.y / c.heads, group = heads / c.heads;
  const int length = kv_length(c, b);
  int first, count;
  kv_new_tokens(c, b, first, count);
  for (int j = blockIdx.x * 4 + (threadIdx.x >> 5); j < length; j += gridDim.x * 4) {
    const int page = kv_page(c, c.table, c.width, b, j);
    if (page < 0) continue;
    const uint8_t* at = kv_head_page(c, page, kvh);
    const int slot = j & ((1 << c.page_shift) - 1);
    float k[DPL], sum = 0.f;
    kv_row_share<FMT, DPL>(at + slot * (D / 2), at + c.k_scales + slot * (D / kv_block(FMT)), lane, c.k_ts, k);
    for (int r = 0; r < count * group; ++r) {
      const int i = first + r / group, h = kvh * group + r % group, p = length - count + r / group;
      int lo, hi;
      kv_range(a, b, i, p, length, lo, hi);
      const float y = lse[(int64_t)i * heads + h];
      if (j < lo || j >= hi || y == -INFINITY) continue;
      float x = 0.f;
#pragma unroll
      for (int e = 0; e < DPL; ++e) x += __bfloat162float(Q[i * q_stride + h * D + lane * DPL + e]) * k[e];
      x = kv_score(warp_sum(x) * a.scale, a.softcap, a.slopes ? a.slopes[h] : 0.f, abs(p - j));
      sum += exp2f(x - y * kLog2e);
    }
    const int64_t w = (((int64_t)page * c.heads + kvh) << c.page_shift) + slot;
    if (lane == 0) weights_out[w] = sum + (j < length - count ? weights[w] : 0.f);
  }
}

}  // namespace torq
