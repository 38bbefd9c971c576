// Eviction: of each sequence and head the `recent` newest tokens stay and, of the others, those with the largest weights, `keep` in all; equal
// weights go to the lower place.  They are copied in their order to other pages, so the sequence afterwards is as long for every head.
#pragma once
#include "kv_cache.cuh"

namespace torq {

// Larger numbers have larger keys.
__device__ __forceinline__ uint32_t ordered_key(float v) {
  const uint32_t u = __float_as_uint(v);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// One CTA per sequence and head writes the places of what stays, in their order, and -1 behind them.  The smallest weight that stays is found
// eight bits of its key at a time (a count of every value of these bits among the keys that share the bits above).
struct KvSelectCfg { static constexpr int THREADS = 1024, EACH = 4; };
static __global__ void __launch_bounds__(KvSelectCfg::THREADS) kv_select_kernel(const KvView c, const float* weights, int keep, int recent,
                                                                                int32_t* new_lengths, int32_t* kept) {
  griddep_wait_and_launch();
  __shared__ uint32_t count[256], chosen[2], sums[2][33];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, head = blockIdx.x % c.heads, b = blockIdx.x / c.heads;
  const int length = kv_length(c, b), stay = length < keep ? length : keep, newest = recent < stay ? recent : stay;
  int32_t* to = kept + (int64_t)blockIdx.x * keep;
  if (head == 0 && tid == 0) new_lengths[b] = stay;
  const int others = length - newest, room = stay - newest;     // `room` of `others` stay
  auto key_of = [&](int j) {
    const int page = kv_page(c, c.table, c.width, b, j);
    return page < 0 ? 0u : ordered_key(weights[(((int64_t)page * c.heads + head) << c.page_shift) + (j & ((1 << c.page_shift) - 1))]);
  };
  uint32_t edge = 0, left = (uint32_t)room;                      // of the keys that equal `edge`, `left` stay
  if (room < others && room > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) count[tid] = 0;
      __syncthreads();
      for (int j = tid; j < others; j += KvSelectCfg::THREADS) {
        const uint32_t key = key_of(j);
        if (shift == 24 || (key >> (shift + 8)) == (edge >> (shift + 8))) atomicAdd(&count[key >> shift & 255u], 1u);
      }
      __syncthreads();
      if (warp == 0) {                                           // the value at which the count from above reaches `left`
        uint32_t own[8], sum = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += own[i] = count[255 - (lane * 8 + i)];
        uint32_t above = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t t = __shfl_up_sync(0xFFFFFFFFu, above, o);
          if (lane >= o) above += t;
        }
        above -= sum;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (above < left && left <= above + own[i]) {
            chosen[0] = 255u - (lane * 8 + i);
            chosen[1] = left - above;
          }
          above += own[i];
        }
      }
      __syncthreads();
      edge |= chosen[0] << shift;
      left = chosen[1];
    }
  }
  // places in their order: a thread takes EACH consecutive ones
  uint32_t equal_before = 0, kept_before = 0;
  for (int base = 0; base < others && room > 0; base += KvSelectCfg::THREADS * KvSelectCfg::EACH) {
    uint32_t above[KvSelectCfg::EACH], equal[KvSelectCfg::EACH], equals = 0;
#pragma unroll
    for (int i = 0; i < KvSelectCfg::EACH; ++i) {
      const int j = base + tid * KvSelectCfg::EACH + i;
      const uint32_t key = j < others ? (room == others ? 1u : key_of(j)) : 0u;
      above[i] = j < others && key > edge;
      equals += equal[i] = j < others && key == edge;
    }
    auto before = [&](uint32_t mine, int which, uint32_t& total) {       // of the threads in front; the same for all in `total`
      uint32_t s = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t t = __shfl_up_sync(0xFFFFFFFFu, s, o);
        if (lane >= o) s += t;
      }
      if (lane == 31) sums[which][warp] = s;
      __syncthreads();
      if (warp == 0) {
        uint32_t w = sums[which][lane], v = w;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const uint32_t t = __shfl_up_sync(0xFFFFFFFFu, v, o);
          if (lane >= o) v += t;
        }
        sums[which][lane] = v - w;
        if (lane == 31) sums[which][32] = v;
      }
      __syncthreads();
      total = sums[which][32];
      return s - mine + sums[which][warp];
    };
    uint32_t total, rank = equal_before + before(equals, 0, total), stays = 0, flag[KvSelectCfg::EACH];
    equal_before += total;
#pragma unroll
    for (int i = 0; i < KvSelectCfg::EACH; ++i) {
      flag[i] = above[i] | (equal[i] & (uint32_t)(rank < left));
      rank += equal[i];
      stays += flag[i];
    }
    uint32_t at = kept_before + before(stays, 1, total);
    kept_before += total;
#pragma unroll
    for (int i = 0; i < KvSelectCfg::EACH; ++i)
      if (flag[i]) to[at++] = base + tid * KvSelectCfg::EACH + i;
    __syncthreads();                                             // `sums` is written again
  }
  for (int r = room + tid; r < keep; r += KvSelectCfg::THREADS) to[r] = r < stay ? others + (r - room) : -1;
}

// D / 16 threads per token that stays, 32 codes and their scales each.
template <int FMT>
__global__ void __launch_bounds__(256) kv_move_kernel(const KvView c, float* weights, const int32_t* new_table, int new_width, int keep,
                                                      const int32_t* kept) {
  griddep_wait_and_launch();
  const int per_token = c.dim / 16, head = blockIdx.y % c.heads, b = blockIdx.y / c.heads;
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < (int64_t)keep * per_token; at += (int64_t)gridDim.x * 256) {
    const int r = (int)(at / per_token), e = (int)(at % per_token);
    const int j = kept[(int64_t)blockIdx.y * keep + r];
    if (j < 0) break;                                            // nothing behind it either
    const int from = kv_page(c, c.table, c.width, b, j), to = (r >> c.page_shift) < new_width ? kv_page(c, new_table, new_width, b, r) : -1;
    if (from < 0 || to < 0) continue;
    const int mask = (1 << c.page_shift) - 1, blocks = c.dim / kv_block(FMT), half = per_token / 2, chunk = e < half ? e : e - half;
    const uint8_t* s = kv_head_page(c, from, head);
    uint8_t* d = kv_head_page(c, to, head);
    const int codes = (e < half ? 0 : c.v_codes) + chunk * 16, scales = (e < half ? c.k_scales : c.v_scales) + chunk * (32 / kv_block(FMT));
    *reinterpret_cast<uint4*>(d + codes + (r & mask) * (c.dim / 2)) = *reinterpret_cast<const uint4*>(s + codes + (j & mask) * (c.dim / 2));
    if constexpr (FMT == FMT_NVFP4)
      *reinterpret_cast<uint16_t*>(d + scales + (r & mask) * blocks) = *reinterpret_cast<const uint16_t*>(s + scales + (j & mask) * blocks);
    else
      d[scales + (r & mask) * blocks] = s[scales + (j & mask) * blocks];
    if (e == 0)
      weights[(((int64_t)to * c.heads + head) << c.page_shift) + (r & mask)] =
          weights[(((int64_t)from * c.heads + head) << c.page_shift) + (j & mask)];
  }
}

}  // namespace torq
