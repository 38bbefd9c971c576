// Attention of the new tokens of every sequence over its cached tokens:
//   x_j = cap(f q k_j) - slope |p - j|,   out = sum_j softmax(x)_j v_j,   lse = log sum_j exp(x_j)
// over the tokens j that a query at place p may see:  p - window < j <= max(p, prefix - 1),  first <= j < length.
// cap(x) = c tanh(x / c).  A query that sees nothing gets zeros and -inf.
#pragma once
#include "kv_cache.cuh"
#include "kv_fragments.cuh"

namespace torq {

struct KvScoring {
  float scale, softcap, per_cap;         // softcap, times log2 e as scores are: 0: none; per_cap = 1 / softcap
  const float* slopes;                   // [query heads], or null
  const int32_t* prefix;                 // [batch], or null
  const int32_t* first;                  // [tokens], or null
  int window;                            // 0: none
};

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// Weights are exp2(x - m + kShift), m raised when a score exceeds it by kSlack: in float16 they are at most 2^15, and those of 2^-14 - kShift keep 11 bits.
constexpr float kShift = 10.f, kSlack = 5.f;
// Where a maximum starts: below every score that float32 has room for, and finite.
constexpr float kLowest = -3.4e38f;
// From here on a maximum is so far from zero that the rounding of the product that it comes from may count in an exponent: scores are rounded as it was before
// it is taken off (fused, a score of 2^27 could be 8 more than itself, and a float16 weight infinite).
constexpr float kFar = 1048576.f;
__device__ __forceinline__ bool kv_far(float m) { return fabsf(m) > kFar && m > kLowest; }

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
// softcap tanh(x / softcap), with u = |x| / softcap.  From u = 1/4 on by (1 - e) / (1 + e), e = exp(-2 u).  Below, 1 - e would cancel (at u = 2^-24 to nothing), so
// there the series of tanh, x (1 - u^2/3 + 2 u^4/15 - 17 u^6/315 + 62 u^8/2835): what it leaves out is at most 0.0089 u^10 < 2^-26 of x.  (Both computed and one
// taken: the account of 32 sequences 47 us instead of 42, for registers; attention takes as long.)
__device__ __forceinline__ float kv_cap(float x, float softcap, float per_cap) {
  const float u = fabsf(x) * per_cap;
  if (u < 0.25f) {
    const float v = u * u;
    return fmaf(x * v, fmaf(v, fmaf(v, fmaf(v, 62.f / 2835.f, -17.f / 315.f), 2.f / 15.f), -1.f / 3.f), x);
  }
  const float e = exp2f(u * (-2.f * kLog2e));
  return copysignf(softcap * __fdividef(1.f - e, 1.f + e), x);
}
// A slope times log2 e, finite: at distance zero it counts nothing, however steep.
__device__ __forceinline__ float kv_slope(const KvScoring& a, int head) { return fminf(fmaxf(a.slopes[head] * kLog2e, kLowest), -kLowest); }
// What comes behind a scaled score; all of it, the slope too, times log2 e.
__device__ __forceinline__ float kv_score(float x, const KvScoring& a, float slope, int distance) {
  if (a.softcap > 0.f) x = kv_cap(x, a.softcap, a.per_cap);
  return x - slope * (float)distance;
}


// ---- few queries per sequence -----------------------------------------------------------------------------------------------------------------
// The cache is streamed once, by all warps alike: the work is a list of steps of 32 cached tokens (sequence after sequence, key/value head after head,
// group of 8 NT rows after group), cut into as many equal ranges as there are warps, whatever the lengths are.  Lengths are known on the device
// alone, so every warp counts the steps itself.  An item (sequence, head, group) that lies in one range is finished by its warp; of one that crosses a
// border each warp leaves sums, maximum and a partial result, and a second kernel joins them in the order of the ranges.  A warp works alone, through a
// ring of its own filled by cp.async: there is no barrier in the kernel.  (Ranges for CTAs of four warps that share an item and meet at its end:
// 32 sequences of up to 8192 tokens 73.6 us, SMs idle for a quarter of it, since a CTA with more items in its range took longer.)
//
// A warp keeps a maximum m of its scores in powers of two that is raised only when a score exceeds it by 5, so weights are exp2(x - m + 10) <= 2^15 in
// float16; they keep 11 bits down to 2^-24 of the largest.  The same goes for the values' scales (see kv_fragments.cuh).  float16 because the values are exact in it and
// both operands have one type; a weight is off by 2^-12 then, where the result is rounded by 2^-9: against 64 bits results are off by 0.0017 of their norm,
// as they are with weights in float32.
template <int FMT_, int D_, int NT_>
struct KvDecodeCfg {
  static constexpr int FMT = FMT_, D = D_, NT = NT_;
  static constexpr int WARPS = 4, THREADS = 32 * WARPS, STEP = 32, ROWS = 8 * NT;
  static constexpr int CH = D / 32, SB = D / kv_block(FMT);
  static constexpr int K_BYTES = STEP * D / 2, S_BYTES = STEP * SB, STAGE = 2 * (K_BYTES + S_BYTES);      // keys, values, their scales
  static constexpr int CTAS = D == 256 || NT >= 2 ? 2 : 3;                 // per SM (four with registers spilled: 32 sequences 62.6 us, three 55.6)
  static constexpr int STAGES = D == 64 ? 4 : 3 - (FMT == FMT_NVFP4 ? 1 : 0);
  static constexpr int ROOM = KvScaleRoom<FMT, D>::BYTES;                  // scales made ready, per warp
  static constexpr int SMEM = WARPS * (STAGES * STAGE + ROOM);
  static constexpr int PARTIAL = ROWS * (D + 2);                           // floats: results, maxima, sums
};

// An item: `rows` rows of sequence b from its first_row on (count * group in all), a key/value head, and cached tokens [lo, hi) that any row of the
// sequence sees; base = lo / 32 * 32.
struct KvItem {
  int b, head, first_token, count, length, first_row, rows, lo, base, hi;
};

__device__ __forceinline__ long long kv_range_begin(long long units, int which, int ranges) { return units * which / ranges; }

// Of sequence b: groups of ROWS rows, steps per group and head.
template <int ROWS>
__device__ __forceinline__ void kv_sequence_steps(const KvView& c, const KvScoring& a, int b, int group, KvItem& it, int& groups, int& per) {
  it.b = b;
  kv_new_tokens(c, b, it.first_token, it.count);
  it.length = kv_length(c, b);
  groups = (it.count * group + ROWS - 1) / ROWS;
  const int p0 = it.length - it.count;
  it.lo = a.window > 0 && p0 - a.window + 1 > 0 ? p0 - a.window + 1 : 0;
  it.hi = it.length;
  it.base = it.lo & ~31;
  per = (it.hi - it.base + 31) / 32;
  if (it.length == 0) groups = 0;
}
__device__ __forceinline__ long long warp_scan(long long v, int lane) {    // inclusive
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long x = __shfl_up_sync(0xFFFFFFFFu, v, o);
    if (lane >= o) v += x;
  }
  return v;
}
__device__ __forceinline__ int64_t kv_out_row(const KvItem& it, int r, int heads, int group) {
  const int rr = it.first_row + r;
  return (int64_t)(it.first_token + rr / group) * heads + it.head * group + rr % group;
}

template <class C>
__global__ void __launch_bounds__(C::THREADS, C::CTAS) kv_decode_kernel(const KvView c, const KvScoring a, const __nv_bfloat16* Q, int64_t q_stride, int heads,
                                                                        __nv_bfloat16* out, float* lse, float* partials) {
  constexpr int FMT = C::FMT, D = C::D, NT = C::NT, CH = C::CH, SB = C::SB, ROWS = C::ROWS;
  extern __shared__ __align__(128) uint8_t smem[];
  griddep_wait_and_launch();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3, group = heads / c.heads;
  const int range = blockIdx.x * C::WARPS + warp, ranges = gridDim.x * C::WARPS;

  // rows of the batch that no sequence has, or an empty one
  auto nothing = [&](int i) {
    const int64_t row = (int64_t)i * heads;
    for (int e = lane; e < heads * D / 8; e += 32) reinterpret_cast<uint4*>(out + row * D)[e] = make_uint4(0, 0, 0, 0);
    if (lse)
      for (int e = lane; e < heads; e += 32) lse[row + e] = -INFINITY;
  };
  if (c.starts) {
    const int before = min(max(c.starts[0], 0), c.tokens), behind = min(max(c.starts[c.batch], before), c.tokens), none = before + c.tokens - behind;
    for (int i = range; i < none; i += ranges) nothing(i < before ? i : behind + i - before);
  }
  for (int b = range; b < c.batch; b += ranges)
    if (c.lengths[b] <= 0) {
      int first, count;
      kv_new_tokens(c, b, first, count);
      for (int i = 0; i < count; ++i) nothing(first + i);
    }

  // steps in all, then where this warp's range begins
  KvItem it;
  int groups, per;
  auto steps_of = [&](int b) -> long long {
    if (b >= c.batch) return 0;
    kv_sequence_steps<ROWS>(c, a, b, group, it, groups, per);
    return (long long)groups * c.heads * per;
  };
  const long long mine = steps_of(lane);
  long long units = mine;
#pragma unroll 4
  for (int b0 = 32; b0 < c.batch; b0 += 32) units += steps_of(b0 + lane);
#pragma unroll
  for (int o = 16; o; o >>= 1) units += __shfl_xor_sync(0xFFFFFFFFu, units, o);
  const long long begin = kv_range_begin(units, range, ranges), end = kv_range_begin(units, range + 1, ranges);
  if (begin >= end) return;
  int b = 0;
  long long sequence_begin = 0;
  for (int b0 = 0;; b0 += 32) {                                            // ends, since begin < units
    const long long v = b0 ? steps_of(b0 + lane) : mine, sum = warp_scan(v, lane);
    const uint32_t here = __ballot_sync(0xFFFFFFFFu, begin < sequence_begin + sum);
    if (here) {
      const int first = __ffs(here) - 1;
      b = b0 + first;
      sequence_begin += __shfl_sync(0xFFFFFFFFu, sum - v, first);
      break;
    }
    sequence_begin += __shfl_sync(0xFFFFFFFFu, sum, 31);
  }
  long long at = begin, sequence_units = steps_of(b);

  const uint32_t ring = smem_u32(smem) + warp * C::STAGES * C::STAGE;
  uint8_t *ring_p = smem + warp * C::STAGES * C::STAGE, *room = smem + C::WARPS * C::STAGES * C::STAGE + warp * C::ROOM;
  uint8_t* v_room = room + KvScaleRoom<FMT, D>::KEYS;
  const int row_of = lane & 15, chunk_of = lane >> 4;
  // Where a lane's pieces of 16 bytes come from and go to.  The codes of 16 tokens are dense in their page; a lane takes every 32nd chunk of them.
  constexpr int PER_GROUP = CH / 2;                                        // copies of a lane for the codes of 16 tokens
  uint32_t to_chunk[CH == 8 ? 2 : 1];
#pragma unroll
  for (int i = 0; i < (CH == 8 ? 2 : 1); ++i) to_chunk[i] = 16 * kv_swizzled<D>((32 * i + lane) / CH, lane % CH) - 512 * i;
  constexpr int PIECES = 16 * SB / 16;                                     // of the scale bytes of 16 tokens, of keys or of values
  const int my_piece = lane % PIECES, my_group = lane / PIECES & 1, my_half = lane / (2 * PIECES);   // keys, values
  const int scale_from = (my_half ? c.v_scales : c.k_scales) + my_piece * 16;

  while (at < end) {
    while (at >= sequence_begin + sequence_units) {                        // sequences without rows have no steps
      sequence_begin += sequence_units;
      sequence_units = steps_of(++b);
    }
    const int local = (int)((at - sequence_begin) / per), step0 = (int)((at - sequence_begin) - (long long)local * per);   // (head, group) of the sequence; its step
    const long long left = end - at;
    const int steps = (int)(left < per - step0 ? left : per - step0);
    it.head = local / groups;
    it.first_row = local % groups * ROWS;
    it.rows = min(ROWS, it.count * group - it.first_row);
    at += steps;

    const int first = it.base + step0 * C::STEP;
    const int32_t* table = c.table + (int64_t)b * c.width;
    const uint8_t* head_pages = c.pages + (int64_t)it.head * c.head_bytes;
    const int mask = (1 << c.page_shift) - 1;
    int64_t page[2];                                                       // where the pages of the next step's two groups of 16 tokens begin
    bool there[2];
    auto look_up = [&](int k) {
      int p[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int j = first + k * C::STEP + 16 * i;
        there[i] = k < steps && j < it.hi && j + 16 > it.lo;
        p[i] = there[i] ? table[j >> c.page_shift] : 0;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (there[i] && (unsigned)p[i] >= (unsigned)c.num_pages) {
          kv_bad_page(c);
          there[i] = false;
        }
        page[i] = there[i] ? p[i] * c.page_bytes : 0;
      }
    };
    uint32_t dst = ring;                                                   // the stage that is filled next
    auto fetch = [&](int k) {
      const int j0 = first + k * C::STEP;
      if (k < steps) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int slot = (j0 + 16 * i) & mask;
          const uint8_t* src = head_pages + page[i] + slot * (D / 2) + lane * 16;
          const int bytes = there[i] ? 16 : 0;
#pragma unroll
          for (int x = 0; x < PER_GROUP; ++x) {
            const int y = i * PER_GROUP + x;
            cp_async_16(dst + to_chunk[CH == 8 ? y & 1 : 0] + 512 * y, src + 512 * x, bytes);
            cp_async_16(dst + C::K_BYTES + to_chunk[CH == 8 ? y & 1 : 0] + 512 * y, src + c.v_codes + 512 * x, bytes);
          }
        }
        const bool mine = my_group ? there[1] : there[0];
        const uint8_t* src = head_pages + (my_group ? page[1] : page[0]) + ((j0 + 16 * my_group) & mask) * SB + scale_from;
        const uint32_t to = dst + 2 * C::K_BYTES + my_half * C::S_BYTES + (my_group * PIECES + my_piece) * 16;
        if constexpr (4 * PIECES <= 32) {
          if (lane < 4 * PIECES) cp_async_16(to, src, mine ? 16 : 0);
        } else {
          cp_async_16(to, src, mine ? 16 : 0);
          cp_async_16(to + C::S_BYTES, src + (c.v_scales - c.k_scales), mine ? 16 : 0);
        }
      }
      cp_async_commit();
      dst = dst == ring + (C::STAGES - 1) * C::STAGE ? ring : dst + C::STAGE;
    };
    look_up(0);
#pragma unroll
    for (int k = 0; k < C::STAGES - 1; ++k) {
      fetch(k);
      look_up(k + 1);
    }

    // the queries, and what each row sees
    KvQuery<D> q[NT];
    const float unit = a.scale * (FMT == FMT_NVFP4 ? c.k_ts : 1.f) * kLog2e;
    float factor[NT][2], slope[NT][2], m[NT][2], l[NT][2];                 // a score's factor: times `unit` and what keys are taken smaller by
    int place[NT][2], lo[NT][2], hi[NT][2], all_lo = 0, all_hi = INT32_MAX, any_lo = INT32_MAX, any_hi = 0;   // what all rows see, what any does
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int r = it.first_row + 8 * n + g;
      const int i = it.first_token + r / group, h = it.head * group + r % group;
      const float back = kv_load_query<FMT, D>(8 * n + g < it.rows ? Q + i * q_stride + h * D : nullptr, t, q[n]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int col = 8 * n + 2 * t + e, rr = it.first_row + col;
        factor[n][e] = __shfl_sync(0xFFFFFFFFu, back, 8 * t + 4 * e);
        lo[n][e] = hi[n][e] = place[n][e] = 0;
        slope[n][e] = 0.f;
        if (col < it.rows) {
          const int token = rr / group;
          place[n][e] = it.length - it.count + token;
          kv_range(a, it.b, it.first_token + token, place[n][e], it.length, lo[n][e], hi[n][e]);
          if (a.slopes) slope[n][e] = kv_slope(a, it.head * group + rr % group);
          all_lo = max(all_lo, lo[n][e]);
          all_hi = min(all_hi, hi[n][e]);
          if (lo[n][e] < hi[n][e]) any_lo = min(any_lo, lo[n][e]);
          any_hi = max(any_hi, hi[n][e]);
        }
        m[n][e] = kLowest;
        l[n][e] = 0.f;
      }
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      all_lo = max(all_lo, __shfl_xor_sync(0xFFFFFFFFu, all_lo, o));
      all_hi = min(all_hi, __shfl_xor_sync(0xFFFFFFFFu, all_hi, o));
    }
    any_lo = __reduce_min_sync(0xFFFFFFFFu, any_lo);
    any_hi = __reduce_max_sync(0xFFFFFFFFu, any_hi);
    const bool special = a.softcap > 0.f || a.slopes;
    float o[NT][CH][2][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < CH * 8; ++i) o[n][i / 8][i / 4 % 2][i % 4] = 0.f;
    int top_scale[CH];                                                     // MXFP4, MXINT4: E of each chunk
    uint32_t top_pair[CH / 2];                                             // the same in halves: chunks i and i + 2 of four (CH = 2: both)
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      top_scale[i] = 27;
      top_pair[i / 2] = 0x001B001Bu;
    }

    bool far = false;                                                      // whether some row's maximum is
    uint32_t stage = ring;
    for (int k = 0; k < steps; ++k) {
      cp_async_wait<C::STAGES - 2>();
      __syncwarp();
      fetch(k + C::STAGES - 1);                                            // into the stage that the last step has left
      look_up(k + C::STAGES);
      const int j0 = first + k * C::STEP;
      const uint8_t* scales = ring_p + (stage - ring) + 2 * C::K_BYTES;
      const bool border = j0 < all_lo || j0 + C::STEP > all_hi;

      // scales of the 32 tokens; those that no row sees may be no numbers, or larger than all others
      const bool seen = j0 + lane >= any_lo && j0 + lane < any_hi;
      const float now = unit * kv_ready_key_scales<FMT, D>(scales, lane, seen, room);
      {
        uint32_t w[(SB + 3) / 4];
        kv_scale_words<SB>(scales + C::S_BYTES + lane * SB, w);
        if (border && !seen) {
#pragma unroll
          for (int i = 0; i < (SB + 3) / 4; ++i) w[i] = 0;
        }
        uint16_t* to = reinterpret_cast<uint16_t*>(v_room) + kv_value_order(lane);
        if constexpr (FMT == FMT_NVFP4) {
#pragma unroll
          for (int i = 0; i < SB; i += 2) {
            const uint32_t f = e4m3x2_f16x2(w[i / 4] >> (8 * (i & 2)));
            to[32 * i] = (uint16_t)f;
            to[32 * (i + 1)] = (uint16_t)(f >> 16);
          }
        } else {
          uint32_t pair[CH / 2];                                           // chunks i and i + 2 of four
          bool above = false;
#pragma unroll
          for (int i = 0; i < CH / 2; ++i) {
            if constexpr (CH == 2) pair[i] = (w[0] & 0xFFu) | (w[0] & 0xFF00u) << 8;
            else pair[i] = (w[i / 2] >> (8 * (i % 2))) & 0x00FF00FFu;
            above |= __vmaxu2(pair[i], top_pair[i]) != top_pair[i];
          }
          if (__any_sync(0xFFFFFFFFu, above)) {
#pragma unroll
            for (int i = 0; i < CH; ++i) {
              const int word = CH == 2 ? 0 : i / 4 * 2 + i % 2, half = CH == 2 ? i : i % 4 / 2;
              const int top = max(top_scale[i], (int)__reduce_max_sync(0xFFFFFFFFu, pair[word] >> (16 * half) & 0xFFFFu));
              const float old = top - top_scale[i] > 126 ? 0.f : __uint_as_float((uint32_t)(127 - (top - top_scale[i])) << 23);
              top_scale[i] = top;
              top_pair[word] = half ? (top_pair[word] & 0xFFFFu) | (uint32_t)top << 16 : (top_pair[word] & 0xFFFF0000u) | (uint32_t)top;
#pragma unroll
              for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int x = 0; x < 8; ++x) o[n][i][x / 4][x % 4] *= old;
            }
          }
#pragma unroll
          for (int i = 0; i < CH / 2; ++i) {
            const uint32_t f = __viaddmax_s16x2_relu(pair[i], __vsub2(0x001B001Bu, top_pair[i]), 0u) << 10;
            const int low = CH == 2 ? 0 : i / 2 * 4 + i % 2, high = CH == 2 ? 1 : low + 2;
            to[32 * low] = (uint16_t)f;
            to[32 * high] = (uint16_t)(f >> 16);
          }
        }
      }
      __syncwarp();

      // scores, weights
      uint32_t p[NT][2][2];
      float s[2][NT][4];
#pragma unroll
      for (int u = 0; u < 2; ++u) kv_tile_scores<FMT, D, NT>(stage, room, 16 * u, lane, q, s[u]);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float f[2] = {factor[n][0] * now, factor[n][1] * now};
        if (special || border) {
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int e = i & 1, j = j0 + 16 * u + g + 8 * (i >> 1);
              float x = s[u][n][i] * f[e];
              if (special) x = kv_score(x, a, slope[n][e], abs(place[n][e] - j));
              s[u][n][i] = j >= lo[n][e] && j < hi[n][e] ? x : -INFINITY;
            }
          f[0] = f[1] = 1.f;
        }
        bool raise = false;
        float most[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          most[e] = fmaxf(fmaxf(s[0][n][e], s[0][n][e + 2]), fmaxf(s[1][n][e], s[1][n][e + 2])) * f[e];
          raise |= most[e] - m[n][e] > kSlack;
        }
        if (__any_sync(0xFFFFFFFFu, raise)) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float top = fmaxf(most[e], m[n][e]);
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, x));
            const float old = ex2(m[n][e] - top);
            m[n][e] = top;
            l[n][e] *= old;
#pragma unroll
            for (int i = 0; i < CH * 2; ++i) {
              o[n][i / 2][i % 2][e] *= old;
              o[n][i / 2][i % 2][e + 2] *= old;
            }
          }
          far |= __any_sync(0xFFFFFFFFu, kv_far(m[n][0]) || kv_far(m[n][1]));
        }
        float off[2] = {kShift - m[n][0], kShift - m[n][1]};
        if (far) {
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[u][n][i] = __fsub_rn(__fmul_rn(s[u][n][i], f[i & 1]), m[n][i & 1]);
          f[0] = f[1] = 1.f;
          off[0] = off[1] = kShift;
        }
#pragma unroll
        for (int u = 0; u < 2; ++u) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            s[u][n][i] = ex2(fmaf(s[u][n][i], f[i & 1], off[i & 1]));
            l[n][i & 1] += s[u][n][i];
          }
          p[n][u][0] = movmatrix_t(pack_f16(s[u][n][0], s[u][n][1]));
          p[n][u][1] = movmatrix_t(pack_f16(s[u][n][2], s[u][n][3]));
        }
      }

      // values
#pragma unroll
      for (int u = 0; u < 2; ++u) {
#pragma unroll
        for (int c2 = 0; c2 < CH; c2 += 2) {
          uint32_t raw[4];
          ldmatrix_x4_t(stage + C::K_BYTES + 16 * kv_swizzled<D>(16 * u + row_of, c2 + chunk_of), raw);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int ch = c2 + e;
            const int blk = FMT == FMT_NVFP4 ? 2 * ch + (g >> 2) : ch;
            const uint2 f = *reinterpret_cast<const uint2*>(v_room + 64 * blk + 32 * u + 8 * t);   // tokens 2t, 2t + 1; 2t + 8, 2t + 9
            uint32_t v[2][4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              kv_value_pairs<FMT>(raw[2 * e + i], v[i]);
#pragma unroll
              for (int x = 0; x < 4; ++x) v[i][x] = mul_f16x2(v[i][x], i ? f.y : f.x);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              mma_f16(o[n][ch][0], v[0][0], v[0][1], v[1][0], v[1][1], p[n][u][0], p[n][u][1], o[n][ch][0]);
              mma_f16(o[n][ch][1], v[0][2], v[0][3], v[1][2], v[1][3], p[n][u][0], p[n][u][1], o[n][ch][1]);
            }
          }
        }
      }
      stage = stage == ring + (C::STAGES - 1) * C::STAGE ? ring : stage + C::STAGE;
    }
    cp_async_wait<0>();
    __syncwarp();                                                          // before the ring is filled again

    const bool begins = step0 == 0, whole = begins && steps == per;
    float* part = partials + (int64_t)(2 * range + (begins ? 1 : 0)) * C::PARTIAL;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l[n][e] += __shfl_xor_sync(0xFFFFFFFFu, l[n][e], x);
        const int r = 8 * n + 2 * t + e;
        if (r >= it.rows) continue;
        const float inv = l[n][e] > 0.f ? 1.f / l[n][e] : 0.f;            // of a part too: its result is as large as its values, its sum stands beside it
        const int64_t row = kv_out_row(it, r, heads, group);
#pragma unroll
        for (int ch = 0; ch < CH; ++ch) {
          const float fs = FMT == FMT_NVFP4 ? c.v_ts : __uint_as_float((uint32_t)(top_scale[ch] - 12) << 23);      // inv times it may be too small a number
          const float4 v = make_float4(o[n][ch][0][e] * inv * fs, o[n][ch][0][e + 2] * inv * fs, o[n][ch][1][e] * inv * fs, o[n][ch][1][e + 2] * inv * fs);
          if (whole) {
            uint2 y;
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y.x) : "f"(v.y), "f"(v.x));
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y.y) : "f"(v.w), "f"(v.z));
            *reinterpret_cast<uint2*>(out + row * D + 32 * ch + 4 * g) = y;
          } else {
            *reinterpret_cast<float4*>(part + r * D + 32 * ch + 4 * g) = v;
          }
        }
        if (g) continue;
        if (!whole) {
          part[ROWS * D + r] = m[n][e];
          part[ROWS * D + ROWS + r] = l[n][e];
        } else if (lse) {
          lse[row] = l[n][e] > 0.f ? (m[n][e] - kShift + log2f(l[n][e])) * kLn2 : -INFINITY;
        }
      }
  }
}

// N parts with maxima pm, sums pl and results v, into m, l and o; `top`: the largest of all maxima.  Results are averages, of the parts and of what is joined so
// far: the factors add up to one, so nothing is larger than the values are.
template <int N, int EACH>
__device__ __forceinline__ void kv_join(const float (&pm)[N], const float (&pl)[N], const float (&v)[N][EACH], float top, float& m, float& l, float (&o)[EACH]) {
  const float before = l * ex2(m - top);
  float w[N], sum = before;
#pragma unroll
  for (int x = 0; x < N; ++x) sum += w[x] = pl[x] * ex2(pm[x] - top);
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
#pragma unroll
  for (int e = 0; e < EACH; ++e) o[e] *= before * inv;
#pragma unroll
  for (int x = 0; x < N; ++x)
#pragma unroll
    for (int e = 0; e < EACH; ++e) o[e] += v[x][e] * (w[x] * inv);
  l = sum;
  m = top;
}

// Joins the results of an item that more than one warp has worked on.  CTA (i, j): item i of the list, its rows from j (8 / SPLIT) on; SPLIT warps to a
// row, each with its share of the ranges.  With more items than borders between ranges (`by_border`) CTA (i, j) has the item that lies across the border
// behind range i, if it begins in that range: then no CTA stands for an item that nothing cuts.  (A CTA for every item, each warp counting the list for itself: 512
// sequences of up to 300 tokens, 8 heads, 137 us, 4096 8.5 ms.)  The list is counted before the wait for the streaming kernel: that one has waited for all before it.
template <int D, int NT, int SPLIT>
__global__ void __launch_bounds__(256) kv_join_kernel(const KvView c, const KvScoring a, int ranges, bool by_border, int heads, const float* partials,
                                                      __nv_bfloat16* out, float* lse) {
  constexpr int ROWS = 8 * NT, PARTIAL = ROWS * (D + 2), EACH = D / 32;
  __shared__ float parts[SPLIT == 1 ? 1 : 8][D + 2];
  __shared__ long long found_at[2];                                        // where the item begins, steps of all
  __shared__ int found[2];                                                 // its sequence, or -1; its number there
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, which = warp % SPLIT, group = heads / c.heads;
  const int r = blockIdx.y * (8 / SPLIT) + warp / SPLIT;
  KvItem it;
  int groups = 0, per = 1;
  auto steps_of = [&](int b, long long& items) -> long long {
    items = 0;
    if (b >= c.batch) return 0;
    kv_sequence_steps<ROWS>(c, a, b, group, it, groups, per);
    items = (long long)groups * c.heads;
    return items * per;
  };
  // the range that has this step: the last that begins at or before it
  auto range_of = [&](long long unit, long long units) { return (int)(((unit + 1) * ranges + units - 1) / units) - 1; };
  if (warp == 0) {
    long long all = 0, at = blockIdx.x, before = 0, steps_before = 0, begin = -1;          // `at`: the item, or the step behind the border
    int b_of = -1, local = 0;
    long long mine_items;
    const long long mine = steps_of(lane, mine_items);
    const int mine_per = per;
    all = mine;
    for (int b0 = 32; b0 < c.batch; b0 += 32) {
      long long items;
      all += steps_of(b0 + lane, items);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) all += __shfl_xor_sync(0xFFFFFFFFu, all, o);
    if (by_border) at = kv_range_begin(all, blockIdx.x + 1, ranges);
    for (int b0 = 0; b0 < c.batch && b_of < 0; b0 += 32) {
      long long items = mine_items;
      const long long steps = b0 ? steps_of(b0 + lane, items) : mine, count = by_border ? steps : items, sum = warp_scan(count, lane), step_sum = warp_scan(steps, lane);
      const uint32_t here = __ballot_sync(0xFFFFFFFFu, at < before + sum);
      if (here) {
        const int first = __ffs(here) - 1;
        const long long rest = at - before - __shfl_sync(0xFFFFFFFFu, sum - count, first);
        const int each = __shfl_sync(0xFFFFFFFFu, b0 ? per : mine_per, first);
        b_of = b0 + first;
        local = (int)(by_border ? rest / each : rest);
        begin = steps_before + __shfl_sync(0xFFFFFFFFu, step_sum - steps, first) + (long long)local * each;
      }
      before += __shfl_sync(0xFFFFFFFFu, sum, 31);
      steps_before += __shfl_sync(0xFFFFFFFFu, step_sum, 31);
    }
    if (b_of >= 0 && by_border && (begin == at || range_of(begin, all) != (int)blockIdx.x)) b_of = -1;
    if (lane == 0) {
      found_at[0] = begin;
      found_at[1] = all;
      found[0] = b_of;
      found[1] = local;
    }
  }
  __syncthreads();
  const long long begin = found_at[0], units = found_at[1];
  const int found_b = found[0], local = found[1];
  if (found_b < 0) return griddep_wait();                                  // every CTA waits: what stands behind this kernel relies on that
  long long items;
  steps_of(found_b, items);
  it.head = local / groups;
  it.first_row = local % groups * ROWS;
  it.rows = min(ROWS, it.count * group - it.first_row);
  const long long end = begin + per;
  const int from = range_of(begin, units), to = range_of(end - 1, units);
  griddep_wait_and_launch();
  if (from == to) return;                                                  // finished
  float m = kLowest, l = 0.f, o[EACH] = {};
  constexpr int BATCH = 4;
  const bool dense = units >= ranges;                                      // else a range has one step at most, and most have none
  const int parts_n = dense ? to - from + 1 : per;
  for (int i = which; i < parts_n && r < it.rows; i += SPLIT * BATCH) {
    float pm[BATCH], pl[BATCH], v[BATCH][EACH];
#pragma unroll
    for (int x = 0; x < BATCH; ++x) {
      const int k = i + x * SPLIT;
      pm[x] = kLowest;
      pl[x] = 0.f;
#pragma unroll
      for (int e = 0; e < EACH; ++e) v[x][e] = 0.f;
      if (k < parts_n) {
        const int at = dense ? from + k : range_of(begin + k, units);
        const float* p = partials + (int64_t)(2 * at + (at == from ? 1 : 0)) * PARTIAL;
        pm[x] = p[ROWS * D + r];
        pl[x] = p[ROWS * D + ROWS + r];
#pragma unroll
        for (int e = 0; e < EACH; ++e) v[x][e] = p[r * D + e * 32 + lane];
      }
    }
    float top = m;
#pragma unroll
    for (int x = 0; x < BATCH; ++x) top = fmaxf(top, pm[x]);
    kv_join<BATCH, EACH>(pm, pl, v, top, m, l, o);
  }
  if constexpr (SPLIT > 1) {
#pragma unroll
    for (int e = 0; e < EACH; ++e) parts[warp][e * 32 + lane] = o[e];
    if (lane == 0) {
      parts[warp][D] = m;
      parts[warp][D + 1] = l;
    }
    __syncthreads();
    if (which) return;
    float top = m, pm[SPLIT], pl[SPLIT], v[SPLIT][EACH];
#pragma unroll
    for (int x = 0; x < SPLIT; ++x) {
      pm[x] = parts[warp + x][D];
      pl[x] = parts[warp + x][D + 1];
      top = fmaxf(top, pm[x]);
#pragma unroll
      for (int e = 0; e < EACH; ++e) v[x][e] = parts[warp + x][e * 32 + lane];
    }
    l = 0.f;
    kv_join<SPLIT, EACH>(pm, pl, v, top, m, l, o);
  }
  if (r >= it.rows) return;
  const int64_t row = kv_out_row(it, r, heads, group);
#pragma unroll
  for (int e = 0; e < EACH; ++e) out[row * D + e * 32 + lane] = __float2bfloat16(o[e]);
  if (lse && lane == 0) lse[row] = l > 0.f ? (m - kShift + log2f(l)) * kLn2 : -INFINITY;
}

// ---- the account ------------------------------------------------------------------------------------------------------------------------------
// weights_out[token] = (old or, of a new token, 0) + sum over the rows of its sequence and the heads of its group of exp2(x log2 e - lse log2 e).
// Only keys are read.  The list of steps of 32 cached tokens is cut into equal ranges for warps as above, a step counting as often as its sequence
// has groups of eight rows; a step belongs to the range that it begins in, so every slot is written once and the order of its sum is fixed.  A warp holds
// the keys of a step as operands (D = 256: of half a step, with 112 bytes of registers spilled all the same) and goes through the groups.
template <int FMT_, int D_>
struct KvWeightsCfg {
  static constexpr int FMT = FMT_, D = D_, WARPS = 4, THREADS = 128, CH = D / 32, SB = D / kv_block(FMT), CTAS = D == 64 ? 4 : 3;
  static constexpr int K_BYTES = 16 * D, S_BYTES = 32 * SB, STAGE = K_BYTES + S_BYTES, STAGES = D == 256 ? 3 : 4;
  static constexpr int ROOM = KvScaleRoom<FMT, D>::KEYS, SMEM = WARPS * (STAGES * STAGE + ROOM), TILES = D == 256 ? 1 : 2;
};

// The first token that any new row of the item's sequence sees, by `first`: what lies in front is not looked at, since it may hold anything.
__device__ __forceinline__ void kv_first_seen(const KvScoring& a, int lane, KvItem& it) {
  if (!a.first) return;
  int least = INT32_MAX;
  for (int i = it.first_token + lane; i < it.first_token + it.count; i += 32) least = min(least, a.first[i]);
  it.lo = max(it.lo, __reduce_min_sync(0xFFFFFFFFu, least));
}

template <class C>
__global__ void __launch_bounds__(C::THREADS, C::CTAS) kv_weights_kernel(const KvView c, const KvScoring a, const __nv_bfloat16* Q, int64_t q_stride, int heads,
                                                                         const float* lse, const float* weights, float* weights_out) {
  constexpr int FMT = C::FMT, D = C::D, CH = C::CH, SB = C::SB, TILES = C::TILES;
  extern __shared__ __align__(128) uint8_t smem[];
  griddep_wait_and_launch();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3, group = heads / c.heads;
  const int range = blockIdx.x * C::WARPS + warp, ranges = gridDim.x * C::WARPS;
  KvItem it;
  int groups, cost, per;                                                   // groups of rows; what a step counts; steps of a head
  auto units_of = [&](int b) -> long long {
    if (b >= c.batch) return 0;
    it.b = b;
    kv_new_tokens(c, b, it.first_token, it.count);
    it.length = kv_length(c, b);
    groups = (it.count * group + 7) / 8;
    cost = groups > 1 ? groups : 1;
    per = (it.length + 31) / 32;
    const int p0 = it.length - it.count;
    it.lo = a.window > 0 && p0 - a.window + 1 > 0 ? p0 - a.window + 1 : 0;
    return (long long)cost * c.heads * per;
  };
  const long long mine = units_of(lane);
  long long units = mine;
#pragma unroll 4
  for (int b0 = 32; b0 < c.batch; b0 += 32) units += units_of(b0 + lane);
#pragma unroll
  for (int o = 16; o; o >>= 1) units += __shfl_xor_sync(0xFFFFFFFFu, units, o);
  const long long begin = kv_range_begin(units, range, ranges), end = kv_range_begin(units, range + 1, ranges);
  if (begin >= end) return;
  int b = 0;
  long long sequence_begin = 0;
  for (int b0 = 0;; b0 += 32) {                                            // ends, since begin < units
    const long long v = b0 ? units_of(b0 + lane) : mine, sum = warp_scan(v, lane);
    const uint32_t here = __ballot_sync(0xFFFFFFFFu, begin < sequence_begin + sum);
    if (here) {
      const int first = __ffs(here) - 1;
      b = b0 + first;
      sequence_begin += __shfl_sync(0xFFFFFFFFu, sum - v, first);
      break;
    }
    sequence_begin += __shfl_sync(0xFFFFFFFFu, sum, 31);
  }
  long long sequence_units = units_of(b);
  long long at = (begin - sequence_begin + cost - 1) / cost * cost + sequence_begin;       // the first step that begins in the range

  const uint32_t ring = smem_u32(smem) + warp * C::STAGES * C::STAGE;
  uint8_t *ring_p = smem + warp * C::STAGES * C::STAGE, *room = smem + C::WARPS * C::STAGES * C::STAGE + warp * C::ROOM;
  const int row_of = lane & 15, chunk_of = lane >> 4, mask = (1 << c.page_shift) - 1;
  constexpr int PER_GROUP = CH / 2;
  uint32_t to_chunk[CH == 8 ? 2 : 1];
#pragma unroll
  for (int i = 0; i < (CH == 8 ? 2 : 1); ++i) to_chunk[i] = 16 * kv_swizzled<D>((32 * i + lane) / CH, lane % CH) - 512 * i;
  constexpr int PIECES = SB;                                               // of 16 bytes: the scale bytes of 16 tokens
  const int my_piece = lane % PIECES, my_group = lane / PIECES & 1;

  while (at < end) {
    while (at >= sequence_begin + sequence_units) {
      sequence_begin += sequence_units;
      sequence_units = units_of(++b);
    }
    const long long step_of = (at - sequence_begin) / cost;
    it.head = (int)(step_of / per);
    const int step0 = (int)(step_of - (long long)it.head * per);
    kv_first_seen(a, lane, it);
    const long long left = (end - at + cost - 1) / cost;                   // steps that begin in the range
    const int steps = (int)(left < per - step0 ? left : per - step0);
    at += (long long)steps * cost;

    const int first = 32 * step0;
    const int32_t* table = c.table + (int64_t)b * c.width;
    const uint8_t* head_pages = c.pages + (int64_t)it.head * c.head_bytes;
    int64_t page[2];
    bool there[2];
    auto look_up = [&](int k) {
      int p[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int j = first + 32 * k + 16 * i;
        there[i] = k < steps && j < it.length && j + 16 > it.lo;
        p[i] = there[i] ? table[j >> c.page_shift] : 0;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (there[i] && (unsigned)p[i] >= (unsigned)c.num_pages) {
          kv_bad_page(c);
          there[i] = false;
        }
        page[i] = there[i] ? p[i] * c.page_bytes : 0;
      }
    };
    uint32_t dst = ring;
    auto fetch = [&](int k) {
      const int j0 = first + 32 * k;
      if (k < steps) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint8_t* src = head_pages + page[i] + ((j0 + 16 * i) & mask) * (D / 2) + lane * 16;
#pragma unroll
          for (int x = 0; x < PER_GROUP; ++x) {
            const int y = i * PER_GROUP + x;
            cp_async_16(dst + to_chunk[CH == 8 ? y & 1 : 0] + 512 * y, src + 512 * x, there[i] ? 16 : 0);
          }
        }
        if (lane < 2 * PIECES) {
          const bool have = my_group ? there[1] : there[0];
          cp_async_16(dst + C::K_BYTES + lane * 16, head_pages + (my_group ? page[1] : page[0]) + c.k_scales + ((j0 + 16 * my_group) & mask) * SB + my_piece * 16,
                      have ? 16 : 0);
        }
      }
      cp_async_commit();
      dst = dst == ring + (C::STAGES - 1) * C::STAGE ? ring : dst + C::STAGE;
    };
    look_up(0);
#pragma unroll
    for (int k = 0; k < C::STAGES - 1; ++k) {
      fetch(k);
      look_up(k + 1);
    }

    const float unit = a.scale * (FMT == FMT_NVFP4 ? c.k_ts : 1.f) * kLog2e;
    // eight rows: their operand, factors to powers of two (times `unit` and what keys are taken smaller by: a product for each score, since one for each group
    // would need two registers that there are not: 47 us instead of 42), ranges.  A row that is not there, or that saw nothing, counts exp2(-inf).
    KvQuery<D> q[1];
    float factor[2], off[2], slope[2];
    int place[2], lo[2], hi[2], all_lo, all_hi;
    auto load_rows = [&](int n) {
      const int r = 8 * n + g, rows = it.count * group;
      const float back = kv_load_query<FMT, D>(r < rows ? Q + (it.first_token + r / group) * q_stride + (it.head * group + r % group) * D : nullptr, t, q[0]);
      all_lo = 0;
      all_hi = INT32_MAX;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int rr = 8 * n + 2 * t + e;
        factor[e] = __shfl_sync(0xFFFFFFFFu, back, 8 * t + 4 * e);
        lo[e] = hi[e] = place[e] = 0;
        slope[e] = 0.f;
        off[e] = -INFINITY;
        if (rr < rows) {
          const int i = it.first_token + rr / group, h = it.head * group + rr % group;
          const float y = lse[(int64_t)i * heads + h];
          place[e] = it.length - it.count + rr / group;
          if (y != -INFINITY) {
            off[e] = -y * kLog2e;
            kv_range(a, it.b, i, place[e], it.length, lo[e], hi[e]);
          }
          all_lo = max(all_lo, lo[e]);
          all_hi = min(all_hi, hi[e]);                                     // 0 where a row saw nothing: its scores may be no numbers
          if (a.slopes) slope[e] = kv_slope(a, h);
        }
      }
#pragma unroll
      for (int o = 1; o < 4; o <<= 1) {
        all_lo = max(all_lo, __shfl_xor_sync(0xFFFFFFFFu, all_lo, o));
        all_hi = min(all_hi, __shfl_xor_sync(0xFFFFFFFFu, all_hi, o));
      }
    };
    if (groups == 1) load_rows(0);
    const bool special = a.softcap > 0.f || a.slopes;

    uint32_t stage = ring;
    for (int k = 0; k < steps; ++k) {
      cp_async_wait<C::STAGES - 2>();
      __syncwarp();
      fetch(k + C::STAGES - 1);
      look_up(k + C::STAGES);
      const int j0 = first + 32 * k, mine_j = j0 + lane;
      // this lane's slot in the account
      int64_t slot = -1;
      float old = 0.f;
      if (mine_j < it.length) {
        const int p = table[mine_j >> c.page_shift];
        if ((unsigned)p < (unsigned)c.num_pages) {
          slot = (((int64_t)p * c.heads + it.head) << c.page_shift) + (mine_j & mask);
          if (mine_j < it.length - it.count) old = weights[slot];
        }
      }
      float sum[2][2] = {};                                                // tokens g, g + 8, g + 16, g + 24, of this lane's columns
      if (groups > 0 && j0 + 32 > it.lo) {
        const float now = unit * kv_ready_key_scales<FMT, D>(ring_p + (stage - ring) + C::K_BYTES, lane, mine_j >= it.lo && mine_j < it.length, room);
        __syncwarp();
#pragma unroll 1
        for (int u0 = 0; u0 < 2; u0 += TILES) {
          uint32_t keys[TILES][CH][2][4], scale[TILES][2][CH];
          float part[TILES][2] = {};
#pragma unroll
          for (int u = 0; u < TILES; ++u) {
            kv_key_scales<FMT, D>(room, 16 * (u0 + u) + g, t, scale[u][0]);
            kv_key_scales<FMT, D>(room, 16 * (u0 + u) + g + 8, t, scale[u][1]);
#pragma unroll
            for (int c2 = 0; c2 < CH; c2 += 2) {
              uint32_t raw[4];
              ldmatrix_x4(stage + 16 * kv_swizzled<D>(16 * (u0 + u) + row_of, c2 + chunk_of), raw);
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                kv_key_pairs<FMT>(raw[x], keys[u][c2 + x / 2][x & 1]);
                if constexpr (FMT == FMT_NVFP4) {
#pragma unroll
                  for (int i = 0; i < 4; ++i) keys[u][c2 + x / 2][x & 1][i] = mul_f16x2(keys[u][c2 + x / 2][x & 1][i], scale[u][x & 1][c2 + x / 2]);
                }
              }
            }
          }
#pragma unroll 1
          for (int n = 0; n < groups; ++n) {
            if (groups > 1) load_rows(n);
            const bool border = j0 < all_lo || j0 + 32 > all_hi;
#pragma unroll
            for (int u = 0; u < TILES; ++u) {
              float s[4] = {};
              const float zero[4] = {};
#pragma unroll
              for (int ch = 0; ch < CH; ++ch) {
                const uint32_t(&x)[2][4] = keys[u][ch];
                if constexpr (FMT == FMT_NVFP4) {
                  mma_f16(s, x[0][0], x[1][0], x[0][1], x[1][1], q[0].q[ch][0], q[0].q[ch][1], s);
                  mma_f16(s, x[0][2], x[1][2], x[0][3], x[1][3], q[0].q[ch][2], q[0].q[ch][3], s);
                } else {
                  float y[4];
                  mma_f16(y, x[0][0], x[1][0], x[0][1], x[1][1], q[0].q[ch][0], q[0].q[ch][1], zero);
                  mma_f16(y, x[0][2], x[1][2], x[0][3], x[1][3], q[0].q[ch][2], q[0].q[ch][3], y);
#pragma unroll
                  for (int i = 0; i < 4; ++i) s[i] = fmaf(y[i], __uint_as_float(scale[u][i >> 1][ch]), s[i]);
                }
              }
              if (special || border) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  const int e = i & 1, j = j0 + 16 * (u0 + u) + g + 8 * (i >> 1);
                  float x = s[i] * factor[e] * now;
                  if (special) x = kv_score(x, a, slope[e], abs(place[e] - j));
                  part[u][i >> 1] += j >= lo[e] && j < hi[e] ? ex2(x + off[e]) : 0.f;
                }
              } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) part[u][i >> 1] += ex2(fmaf(s[i] * factor[i & 1], now, off[i & 1]));
              }
            }
          }
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (TILES == 2 || u0 == 0) sum[0][i] = part[0][i];
            if (TILES == 2 || u0 == 1) sum[1][i] = part[TILES - 1][i];
          }
        }
      }
#pragma unroll
      for (int o = 1; o < 4; o <<= 1)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i >> 1][i & 1] += __shfl_xor_sync(0xFFFFFFFFu, sum[i >> 1][i & 1], o);
      const float own = t & 2 ? (t & 1 ? sum[1][1] : sum[1][0]) : (t & 1 ? sum[0][1] : sum[0][0]);         // token g + 8 t
      const float w = __shfl_sync(0xFFFFFFFFu, own, (lane & 7) * 4 + (lane >> 3));
      if (slot >= 0) weights_out[slot] = old + w;
      stage = stage == ring + (C::STAGES - 1) * C::STAGE ? ring : stage + C::STAGE;
    }
    cp_async_wait<0>();
    __syncwarp();
  }
}

// The same for many rows of a sequence.  What a group of eight rows costs is its queries: read from L2, scaled, its ranges and sums looked up, one behind
// the other.  So the four warps of a CTA, each with 32 tokens as operands (D = 256: 16), take the same groups: each makes one of four ready in shared
// memory, the loads for the next four in flight, and all go through the four.  Blocks of tokens that no row of a group sees are passed over.  48 rows of 4
// heads over 3 sequences of up to 3000 tokens, 8 key/value heads: 22.9 us, of which the longest chain of a CTA is most; 70.5 by single warps.
template <int FMT_, int D_>
struct KvRowWeightsCfg {
  static constexpr int FMT = FMT_, D = D_, WARPS = 4, THREADS = 128, CH = D / 32, SB = D / kv_block(FMT), CTAS = D == 256 ? 2 : 3;
  static constexpr int TILES = D == 256 ? 1 : 2, OWN = 16 * TILES, TOK = WARPS * OWN;      // tokens of a warp, of a CTA
  static constexpr int K_BYTES = OWN * D / 2, S_BYTES = 32 * SB, STAGE = K_BYTES + S_BYTES, ROOM = KvScaleRoom<FMT, D>::KEYS;
  static constexpr int QUERIES = CH * 512, GROUP = QUERIES + 8 * 24 + 64;                  // a group: operand; per row factor, offset, slope, place, range; limits
  static constexpr int GROUPS_AT = WARPS * (2 * STAGE + ROOM), SMEM = GROUPS_AT + 2 * WARPS * GROUP;
};

template <class C>
__global__ void __launch_bounds__(C::THREADS, C::CTAS) kv_row_weights_kernel(const KvView c, const KvScoring a, const __nv_bfloat16* Q, int64_t q_stride,
                                                                             int heads, const float* lse, const float* weights, float* weights_out) {
  constexpr int FMT = C::FMT, D = C::D, CH = C::CH, SB = C::SB, TILES = C::TILES, OWN = C::OWN;
  extern __shared__ __align__(128) uint8_t smem[];
  griddep_wait_and_launch();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3, group = heads / c.heads;
  KvItem it;
  int groups, cost, per;                                                   // groups of rows; what a block of TOK tokens counts; blocks of a head
  auto units_of = [&](int b) -> long long {
    if (b >= c.batch) return 0;
    it.b = b;
    kv_new_tokens(c, b, it.first_token, it.count);
    it.length = kv_length(c, b);
    groups = (it.count * group + 7) / 8;
    cost = 1 + (groups + 3) / 4;
    per = (it.length + C::TOK - 1) / C::TOK;
    const int p0 = it.length - it.count;
    it.lo = a.window > 0 && p0 - a.window + 1 > 0 ? p0 - a.window + 1 : 0;
    return (long long)cost * c.heads * per;
  };
  const long long mine = units_of(lane);
  long long units = mine;
#pragma unroll 4
  for (int b0 = 32; b0 < c.batch; b0 += 32) units += units_of(b0 + lane);
#pragma unroll
  for (int o = 16; o; o >>= 1) units += __shfl_xor_sync(0xFFFFFFFFu, units, o);
  const long long begin = kv_range_begin(units, blockIdx.x, gridDim.x), end = kv_range_begin(units, blockIdx.x + 1, gridDim.x);
  if (begin >= end) return;                                                // the same for all warps, as is what follows from it
  int b = 0;
  long long sequence_begin = 0;
  for (int b0 = 0;; b0 += 32) {                                            // ends, since begin < units
    const long long v = b0 ? units_of(b0 + lane) : mine, sum = warp_scan(v, lane);
    const uint32_t here = __ballot_sync(0xFFFFFFFFu, begin < sequence_begin + sum);
    if (here) {
      const int first = __ffs(here) - 1;
      b = b0 + first;
      sequence_begin += __shfl_sync(0xFFFFFFFFu, sum - v, first);
      break;
    }
    sequence_begin += __shfl_sync(0xFFFFFFFFu, sum, 31);
  }
  long long sequence_units = units_of(b);
  long long at = (begin - sequence_begin + cost - 1) / cost * cost + sequence_begin;       // the first block that begins in the range

  uint8_t *ring_p = smem + warp * 2 * C::STAGE, *room = smem + C::WARPS * 2 * C::STAGE + warp * C::ROOM, *shared_groups = smem + C::GROUPS_AT;
  const uint32_t ring = smem_u32(ring_p);
  const int row_of = lane & 15, chunk_of = lane >> 4, mask = (1 << c.page_shift) - 1;
  constexpr int PER_GROUP = CH / 2, PIECES = SB;                           // copies of a lane for the codes of 16 tokens; 16-byte pieces of their scale bytes
  uint32_t to_chunk[CH == 8 ? 2 : 1];
#pragma unroll
  for (int i = 0; i < (CH == 8 ? 2 : 1); ++i) to_chunk[i] = 16 * kv_swizzled<D>((32 * i + lane) / CH, lane % CH) - 512 * i;
  const bool special = a.softcap > 0.f || a.slopes;

  while (at < end) {
    while (at >= sequence_begin + sequence_units) {
      sequence_begin += sequence_units;
      sequence_units = units_of(++b);
    }
    const long long block_of = (at - sequence_begin) / cost;
    it.head = (int)(block_of / per);
    const int block0 = (int)(block_of - (long long)it.head * per);
    kv_first_seen(a, lane, it);
    const long long left = (end - at + cost - 1) / cost;                   // blocks that begin in the range
    const int blocks = (int)(left < per - block0 ? left : per - block0);
    at += (long long)blocks * cost;

    const int32_t* table = c.table + (int64_t)b * c.width;
    const uint8_t* head_pages = c.pages + (int64_t)it.head * c.head_bytes;
    auto fetch = [&](int k) {                                              // this warp's tokens of block k
      const int j0 = (block0 + k) * C::TOK + warp * OWN;
      const uint32_t dst = ring + (k & 1) * C::STAGE;
#pragma unroll
      for (int i = 0; i < TILES; ++i) {
        const int j = j0 + 16 * i;
        bool there = k < blocks && groups > 0 && j < it.length && j + 16 > it.lo;
        const int p = there ? table[j >> c.page_shift] : 0;
        if (there && (unsigned)p >= (unsigned)c.num_pages) {
          kv_bad_page(c);
          there = false;
        }
        const uint8_t* page = head_pages + (there ? p * c.page_bytes : 0);
        const int slot = j & mask;
#pragma unroll
        for (int x = 0; x < PER_GROUP; ++x) {
          const int y = i * PER_GROUP + x;
          cp_async_16(dst + to_chunk[CH == 8 ? y & 1 : 0] + 512 * y, page + slot * (D / 2) + lane * 16 + 512 * x, there ? 16 : 0);
        }
        if (lane < PIECES) cp_async_16(dst + C::K_BYTES + (i * PIECES + lane) * 16, page + c.k_scales + slot * SB + lane * 16, there ? 16 : 0);
      }
      cp_async_commit();
    };
    // group n of eight rows: lane (g, t) has row g
    uint4 raw[CH];
    float row_lse = -INFINITY, row_slope = 0.f;
    int row_place = 0, row_lo = 0, row_hi = 0;
    auto load_group = [&](int n) {
      const int r = 8 * n + g;
      const bool have = r < it.count * group;
      const int i = it.first_token + r / group, h = it.head * group + r % group;
      row_lse = have ? lse[(int64_t)i * heads + h] : -INFINITY;
      const __nv_bfloat16* q = Q + i * q_stride + h * D + 8 * t;
#pragma unroll
      for (int x = 0; x < CH; ++x) raw[x] = have ? *reinterpret_cast<const uint4*>(q + 32 * x) : make_uint4(0, 0, 0, 0);
      row_slope = have && a.slopes ? kv_slope(a, h) : 0.f;
      row_place = it.length - it.count + r / group;
      row_lo = row_hi = 0;
      if (have) kv_range(a, it.b, i, row_place, it.length, row_lo, row_hi);
    };
    auto store_group = [&](int n) {
      if (8 * n >= it.count * group) return;                               // the same for the whole warp
      uint8_t* to = shared_groups + (n / 4 & 1) * (4 * C::GROUP) + (n & 3) * C::GROUP;
      if (row_lse == -INFINITY) {                                          // saw nothing: its queries may be no numbers
        row_lo = row_hi = 0;
#pragma unroll
        for (int x = 0; x < CH; ++x) raw[x] = make_uint4(0, 0, 0, 0);
      }
      KvQuery<D> q;
      const float back = kv_scale_query<FMT, D>(raw, q);
#pragma unroll
      for (int x = 0; x < CH; ++x) reinterpret_cast<uint4*>(to)[32 * x + lane] = make_uint4(q.q[x][0], q.q[x][1], q.q[x][2], q.q[x][3]);
      const int in_all_lo = __reduce_max_sync(0xFFFFFFFFu, row_lo), in_all_hi = __reduce_min_sync(0xFFFFFFFFu, row_hi);
      const int in_any_lo = __reduce_min_sync(0xFFFFFFFFu, row_hi > 0 ? row_lo : INT32_MAX), in_any_hi = __reduce_max_sync(0xFFFFFFFFu, row_hi);
      if (t == 0) {
        reinterpret_cast<float4*>(to + C::QUERIES)[g] = make_float4(back, -row_lse * kLog2e, row_slope, __int_as_float(row_place));
        reinterpret_cast<int2*>(to + C::QUERIES + 128)[g] = make_int2(row_lo, row_hi);
      }
      if (lane == 0) *reinterpret_cast<int4*>(to + C::QUERIES + 192) = make_int4(in_all_lo, in_all_hi, in_any_lo, in_any_hi);
    };

    fetch(0);
    for (int k = 0; k < blocks; ++k) {
      if (groups > 0) load_group(warp);
      fetch(k + 1);                                                        // into the stage that the last block has left
      const int j0 = (block0 + k) * C::TOK + warp * OWN, mine_j = j0 + lane;
      int64_t slot = -1;                                                   // of this lane's token in the account
      float old = 0.f;
      if (lane < OWN && mine_j < it.length) {
        const int p = table[mine_j >> c.page_shift];
        if ((unsigned)p < (unsigned)c.num_pages) {
          slot = (((int64_t)p * c.heads + it.head) << c.page_shift) + (mine_j & mask);
          if (mine_j < it.length - it.count) old = weights[slot];
        }
      }
      if (groups > 0) store_group(warp);
      cp_async_wait<1>();
      __syncwarp();
      const uint32_t stage = ring + (k & 1) * C::STAGE;
      const int token = lane % OWN;                                        // D = 256: two lanes to a token
      const float now = a.scale * (FMT == FMT_NVFP4 ? c.k_ts : 1.f) * kLog2e *
                        kv_ready_key_scales<FMT, D>(ring_p + (k & 1) * C::STAGE + C::K_BYTES, token, j0 + token >= it.lo && j0 + token < it.length, room);
      __syncwarp();
      uint32_t keys[TILES][CH][2][4], scale[TILES][2][CH];
      float part[TILES][2] = {};
#pragma unroll
      for (int u = 0; u < TILES; ++u) {
        kv_key_scales<FMT, D>(room, 16 * u + g, t, scale[u][0]);
        kv_key_scales<FMT, D>(room, 16 * u + g + 8, t, scale[u][1]);
#pragma unroll
        for (int c2 = 0; c2 < CH; c2 += 2) {
          uint32_t codes[4];
          ldmatrix_x4(stage + 16 * kv_swizzled<D>(16 * u + row_of, c2 + chunk_of), codes);
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            kv_key_pairs<FMT>(codes[x], keys[u][c2 + x / 2][x & 1]);
            if constexpr (FMT == FMT_NVFP4) {
#pragma unroll
              for (int i = 0; i < 4; ++i) keys[u][c2 + x / 2][x & 1][i] = mul_f16x2(keys[u][c2 + x / 2][x & 1][i], scale[u][x & 1][c2 + x / 2]);
            }
          }
        }
      }
      __syncthreads();
#pragma unroll 1
      for (int n0 = 0; n0 < groups; n0 += 4) {
        const bool more = n0 + 4 < groups;
        if (more) load_group(n0 + 4 + warp);
        const uint8_t* from = shared_groups + (n0 / 4 & 1) * (4 * C::GROUP);
#pragma unroll 1
        for (int n = n0; n < n0 + 4 && n < groups; ++n, from += C::GROUP) {
          const int4 limits = *reinterpret_cast<const int4*>(from + C::QUERIES + 192);
          if (j0 >= limits.w || j0 + OWN <= limits.z) continue;            // no row of the group sees any of these tokens
          const bool border = j0 < limits.x || j0 + OWN > limits.y;
          float4 f[2] = {reinterpret_cast<const float4*>(from + C::QUERIES)[2 * t], reinterpret_cast<const float4*>(from + C::QUERIES)[2 * t + 1]};
          f[0].x *= now;
          f[1].x *= now;
          float s[TILES][4] = {};
#pragma unroll
          for (int ch = 0; ch < CH; ++ch) {
            const uint4 q = reinterpret_cast<const uint4*>(from)[32 * ch + lane];
#pragma unroll
            for (int u = 0; u < TILES; ++u) {
              const uint32_t(&x)[2][4] = keys[u][ch];
              if constexpr (FMT == FMT_NVFP4) {
                mma_f16(s[u], x[0][0], x[1][0], x[0][1], x[1][1], q.x, q.y, s[u]);
                mma_f16(s[u], x[0][2], x[1][2], x[0][3], x[1][3], q.z, q.w, s[u]);
              } else {
                const float zero[4] = {};
                float y[4];
                mma_f16(y, x[0][0], x[1][0], x[0][1], x[1][1], q.x, q.y, zero);
                mma_f16(y, x[0][2], x[1][2], x[0][3], x[1][3], q.z, q.w, y);
#pragma unroll
                for (int i = 0; i < 4; ++i) s[u][i] = fmaf(y[i], __uint_as_float(scale[u][i >> 1][ch]), s[u][i]);
              }
            }
          }
          if (special || border) {
            const int4 range = *reinterpret_cast<const int4*>(from + C::QUERIES + 128 + 16 * t);
            const int lo[2] = {range.x, range.z}, hi[2] = {range.y, range.w};
#pragma unroll
            for (int u = 0; u < TILES; ++u)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int e = i & 1, j = j0 + 16 * u + g + 8 * (i >> 1);
                float x = s[u][i] * f[e].x;
                if (special) x = kv_score(x, a, f[e].z, abs(__float_as_int(f[e].w) - j));
                part[u][i >> 1] += j >= lo[e] && j < hi[e] ? ex2(x + f[e].y) : 0.f;
              }
          } else {
#pragma unroll
            for (int u = 0; u < TILES; ++u)
#pragma unroll
              for (int i = 0; i < 4; ++i) part[u][i >> 1] += ex2(fmaf(s[u][i], f[i & 1].x, f[i & 1].y));
          }
        }
        if (more) store_group(n0 + 4 + warp);
        __syncthreads();                                                   // all have left this buffer, the next one is written
      }
#pragma unroll
      for (int o = 1; o < 4; o <<= 1)
#pragma unroll
        for (int i = 0; i < 2 * TILES; ++i) part[i >> 1][i & 1] += __shfl_xor_sync(0xFFFFFFFFu, part[i >> 1][i & 1], o);
      const float low = t & 1 ? part[0][1] : part[0][0], high = t & 1 ? part[TILES - 1][1] : part[TILES - 1][0];
      const float own = TILES == 2 && (t & 2) ? high : low;                // token g + 8 t
      const float w = __shfl_sync(0xFFFFFFFFu, own, (lane & 7) * 4 + (lane >> 3));
      if (slot >= 0) weights_out[slot] = old + w;
    }
    cp_async_wait<0>();
    __syncwarp();
  }
}

}  // namespace torq
