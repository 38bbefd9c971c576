// Eviction: of each sequence and head the `recent` newest tokens stay and, of the others, those with the largest weights, `keep` in all; equal
// weights go to the lower place.  They are copied in their order to other pages, so the sequence afterwards is as long for every head.
#pragma once
#include "kv_cache.cuh"

namespace torq {

// Larger numbers have larger keys; zeros of either sign the same.
__device__ __forceinline__ uint32_t ordered_key(float v) {
  const uint32_t u = v == 0.f ? 0u : __float_as_uint(v);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// A cluster of 1 to 8 CTAs per sequence and head (more where there are few of these) writes the places of what stays, in their order, and -1 behind them.
// The smallest weight that stays is found 11 bits of its key at a time, 10 the last: every CTA counts the values of these bits among its keys that share
// the bits above, all add up the counts of all through distributed shared memory, and the value is where the sum from above reaches the room.
// A CTA reads its weights once, into shared memory, up to KEYS of them; longer parts are read again every time.
// (One CTA with digits of eight bits, weights read five times: 65000 tokens, 8 heads 128 us, 64 times 4500 tokens 17 us.)
struct KvSelectCfg {
  static constexpr int THREADS = 1024, EACH = 4, KEYS = 24576, BINS = 2048, SMEM = KEYS * 4;
};
static __global__ void __launch_bounds__(KvSelectCfg::THREADS) kv_select_kernel(const KvView c, const float* weights, int keep, int recent, int cluster,
                                                                                int32_t* new_lengths, int32_t* kept) {
  griddep_wait_and_launch();
  using C = KvSelectCfg;
  extern __shared__ uint32_t keys[];
  __shared__ uint32_t count[2][C::BINS], chosen[2], sums[2][33], mine[2];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, rank = blockIdx.x % cluster, item = blockIdx.x / cluster, head = item % c.heads,
            b = item / c.heads;
  const int length = kv_length(c, b), stay = length < keep ? length : keep, newest = recent < stay ? recent : stay;
  int32_t* to = kept + (int64_t)item * keep;
  if (head == 0 && rank == 0 && tid == 0) new_lengths[b] = stay;
  const int others = length - newest, room = stay - newest;     // `room` of `others` stay
  const int part = ((others + cluster - 1) / cluster + 31) & ~31, first = min(rank * part, others), n = min(part, others - first);
  const bool held = part <= C::KEYS;
  auto read = [&](int i) {
    const int j = first + i, page = kv_page(c, c.table, c.width, b, j);
    return page < 0 ? 0u : ordered_key(weights[(((int64_t)page * c.heads + head) << c.page_shift) + (j & ((1 << c.page_shift) - 1))]);
  };
  uint32_t edge = 0, left = (uint32_t)room;                      // of the keys that equal `edge`, `left` stay
  const bool all = room == others, select = !all && room > 0;
  if (select) {
    if (held) {
      // eight at a time, all loads of one kind before the first is looked at
      constexpr int EACH = 8;
      for (int i0 = tid; i0 < n; i0 += EACH * C::THREADS) {
        int page[EACH];
        float w[EACH];
#pragma unroll
        for (int u = 0; u < EACH; ++u) {
          const int i = i0 + u * C::THREADS;
          page[u] = i < n ? c.table[(int64_t)b * c.width + ((first + i) >> c.page_shift)] : 0;
        }
#pragma unroll
        for (int u = 0; u < EACH; ++u) {
          const int i = i0 + u * C::THREADS, j = first + i;
          w[u] = 0.f;
          if (i < n && (unsigned)page[u] < (unsigned)c.num_pages)
            w[u] = weights[(((int64_t)page[u] * c.heads + head) << c.page_shift) + (j & ((1 << c.page_shift) - 1))];
        }
#pragma unroll
        for (int u = 0; u < EACH; ++u) {
          const int i = i0 + u * C::THREADS;
          if (i >= n) break;
          const bool good = (unsigned)page[u] < (unsigned)c.num_pages;
          if (!good) kv_bad_page(c);
          keys[i] = good ? ordered_key(w[u]) : 0u;
        }
      }
    }
    int above = 32;                                              // bits above which `edge` is known
    for (int pass = 0; pass < 3; ++pass) {
      const int bits = pass < 2 ? 11 : 10, shift = above - bits;
      uint32_t* own = count[pass & 1];
      own[tid] = own[tid + C::THREADS] = 0;
      __syncthreads();
      for (int i = tid; i < n; i += C::THREADS) {
        const uint32_t key = held ? keys[i] : read(i);
        if (pass == 0 || key >> above == edge >> above) atomicAdd(&own[key >> shift & ((1u << bits) - 1)], 1u);
      }
      if (cluster > 1) cluster_sync_all();
      else __syncthreads();
      // two bins to a thread, the largest values first
      uint32_t bin[2], of[8][2];                                 // all loads on their way before the first is used
#pragma unroll
      for (int r = 0; r < 8; ++r)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int value = C::BINS - 1 - (2 * tid + i);
          of[r][i] = 0;
          if (r < cluster) of[r][i] = cluster > 1 ? load_cluster_u32(map_to_cta(smem_u32(own + value), (uint32_t)r)) : own[value];
        }
#pragma unroll
      for (int i = 0; i < 2; ++i) bin[i] = ((of[0][i] + of[1][i]) + (of[2][i] + of[3][i])) + ((of[4][i] + of[5][i]) + (of[6][i] + of[7][i]));
      uint32_t s = bin[0] + bin[1];
      const uint32_t both = s;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t t = __shfl_up_sync(0xFFFFFFFFu, s, o);
        if (lane >= o) s += t;
      }
      if (lane == 31) sums[0][warp] = s;
      __syncthreads();
      uint32_t over = s - both + __reduce_add_sync(0xFFFFFFFFu, lane < warp ? sums[0][lane] : 0u);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (over < left && left <= over + bin[i]) {
          chosen[0] = (uint32_t)(C::BINS - 1 - (2 * tid + i));
          chosen[1] = left - over;
        }
        over += bin[i];
      }
      __syncthreads();
      edge |= chosen[0] << shift;
      left = chosen[1];
      above = shift;
      __syncthreads();                                           // `sums` and `chosen` are written again
    }
  }
  auto key_of = [&](int i) { return held ? keys[i] : read(i); };
  // how many of the parts in front stay, and equal the edge
  uint32_t equal_before = 0, kept_before = 0;
  if (room > 0 && cluster > 1) {
    if (tid < 2) mine[tid] = 0;
    __syncthreads();
    uint32_t more = 0, same = 0;
    for (int i = tid; i < n; i += C::THREADS) {
      const uint32_t key = all ? 1u : key_of(i);
      more += key > edge;
      same += key == edge;
    }
    more = __reduce_add_sync(0xFFFFFFFFu, more);
    same = __reduce_add_sync(0xFFFFFFFFu, same);
    if (lane == 0) {
      atomicAdd(&mine[0], more);
      atomicAdd(&mine[1], same);
    }
    cluster_sync_all();
    for (int r = 0; r < rank; ++r) {
      const uint32_t m = load_cluster_u32(map_to_cta(smem_u32(&mine[0]), (uint32_t)r)), e = load_cluster_u32(map_to_cta(smem_u32(&mine[1]), (uint32_t)r));
      kept_before += m + (equal_before >= left ? 0u : min(e, left - equal_before));
      equal_before += e;
    }
  }
  // places in their order: a thread takes EACH consecutive ones
  for (int base = 0; base < n && room > 0; base += C::THREADS * C::EACH) {
    uint32_t above[C::EACH], equal[C::EACH], equals = 0;
#pragma unroll
    for (int i = 0; i < C::EACH; ++i) {
      const int j = base + tid * C::EACH + i;
      const uint32_t key = j < n ? (all ? 1u : key_of(j)) : 0u;
      above[i] = j < n && key > edge;
      equals += equal[i] = j < n && key == edge;
    }
    auto before = [&](uint32_t own, int which, uint32_t& total) {        // of the threads in front; the same for all in `total`
      uint32_t s = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t t = __shfl_up_sync(0xFFFFFFFFu, s, o);
        if (lane >= o) s += t;
      }
      if (lane == 31) sums[which][warp] = s;
      __syncthreads();
      uint32_t front = 0;
      total = 0;
      const uint32_t w = sums[which][lane];
      total = __reduce_add_sync(0xFFFFFFFFu, w);
      front = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? w : 0u);
      return s - own + front;
    };
    uint32_t total, order = equal_before + before(equals, 0, total), stays = 0, flag[C::EACH];
    equal_before += total;
#pragma unroll
    for (int i = 0; i < C::EACH; ++i) {
      flag[i] = above[i] | (equal[i] & (uint32_t)(order < left));
      order += equal[i];
      stays += flag[i];
    }
    uint32_t at = kept_before + before(stays, 1, total);
    kept_before += total;
#pragma unroll
    for (int i = 0; i < C::EACH; ++i)
      if (flag[i]) to[at++] = first + base + tid * C::EACH + i;
    __syncthreads();                                             // `sums` is written again
  }
  for (int r = room + rank * C::THREADS + tid; r < keep; r += cluster * C::THREADS) to[r] = r < stay ? others + (r - room) : -1;
  if (cluster > 1) cluster_sync_all();                           // others may still read this CTA's shared memory
}

// D / 16 threads per token that stays, 32 codes and their scales each, EACH tokens at a time: a copy hangs on three loads one behind the other.
template <int FMT>
__global__ void __launch_bounds__(256) kv_move_kernel(const KvView c, float* weights, const int32_t* new_table, int new_width, int keep,
                                                      const int32_t* kept) {
  griddep_wait_and_launch();
  constexpr int EACH = 4;
  const int shift = 31 - __clz(c.dim / 16), head = blockIdx.y % c.heads, b = blockIdx.y / c.heads, mask = (1 << c.page_shift) - 1;
  const int e = threadIdx.x & ((1 << shift) - 1), half = 1 << shift >> 1, chunk = e & (half - 1), blocks = c.dim / kv_block(FMT);
  const int codes_at = (e < half ? 0 : c.v_codes) + chunk * 16, scales_at = (e < half ? c.k_scales : c.v_scales) + chunk * (32 / kv_block(FMT));
  const int per_cta = 256 >> shift;
  for (int64_t r0 = (int64_t)blockIdx.x * per_cta * EACH + (threadIdx.x >> shift); r0 < keep; r0 += (int64_t)gridDim.x * per_cta * EACH) {
    int j[EACH];
    const uint8_t* from[EACH];
    uint8_t* to[EACH];
    int64_t w_from[EACH], w_to[EACH];
#pragma unroll
    for (int u = 0; u < EACH; ++u) {
      const int64_t r = r0 + u * per_cta;
      j[u] = r < keep ? kept[(int64_t)blockIdx.y * keep + r] : -1;
    }
    int page_of[EACH], there_of[EACH];                           // all loads before the first is looked at
#pragma unroll
    for (int u = 0; u < EACH; ++u) {
      const int r = (int)(r0 + u * per_cta);
      page_of[u] = there_of[u] = 0;
      if (j[u] < 0) continue;
      page_of[u] = c.table[(int64_t)b * c.width + (j[u] >> c.page_shift)];
      there_of[u] = (r >> c.page_shift) < new_width ? new_table[(int64_t)b * new_width + (r >> c.page_shift)] : -1;
    }
#pragma unroll
    for (int u = 0; u < EACH; ++u) {
      const int r = (int)(r0 + u * per_cta), page = page_of[u], there = there_of[u];
      to[u] = nullptr;
      if (j[u] < 0) continue;
      if ((unsigned)page >= (unsigned)c.num_pages || (unsigned)there >= (unsigned)c.num_pages) {
        kv_bad_page(c);
        continue;
      }
      from[u] = kv_head_page(c, page, head);
      to[u] = kv_head_page(c, there, head);
      w_from[u] = (((int64_t)page * c.heads + head) << c.page_shift) + (j[u] & mask);
      w_to[u] = (((int64_t)there * c.heads + head) << c.page_shift) + (r & mask);
    }
    uint4 codes[EACH];
    uint32_t scales[EACH];
    float weight[EACH];
#pragma unroll
    for (int u = 0; u < EACH; ++u) {
      if (!to[u]) continue;
      codes[u] = *reinterpret_cast<const uint4*>(from[u] + codes_at + (j[u] & mask) * (c.dim / 2));
      const uint8_t* s = from[u] + scales_at + (j[u] & mask) * blocks;
      scales[u] = FMT == FMT_NVFP4 ? *reinterpret_cast<const uint16_t*>(s) : *s;
      if (e == 0) weight[u] = weights[w_from[u]];
    }
#pragma unroll
    for (int u = 0; u < EACH; ++u) {
      if (!to[u]) continue;
      const int slot = (int)(r0 + u * per_cta) & mask;
      *reinterpret_cast<uint4*>(to[u] + codes_at + slot * (c.dim / 2)) = codes[u];
      uint8_t* s = to[u] + scales_at + slot * blocks;
      if constexpr (FMT == FMT_NVFP4) *reinterpret_cast<uint16_t*>(s) = (uint16_t)scales[u];
      else *s = (uint8_t)scales[u];
      if (e == 0) weights[w_to[u]] = weight[u];
    }
  }
}

}  // namespace torq
