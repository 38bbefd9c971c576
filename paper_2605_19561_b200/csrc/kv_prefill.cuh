// Attention of many new tokens per sequence over the 4-bit cache, on tcgen05: rows (tokens times the query heads of a group) in tiles of 128, two tiles
// to a CTA (D = 256: one), cached tokens in tiles of TOK.
//   S = Q K^T        float16 operands in shared memory, float32 in tensor memory
//   P = exp2(...)    from tensor memory and back into it as float16, in the place of S
//   O += P V         P from tensor memory, V from shared memory
// Keys and values are widened to float16 once per CTA and tile, whatever the number of rows: codes are exact there, with the scales as follows.
// NVFP4: code times E4M3 scale, exact.  MXFP4, MXINT4: code times 2^(e - E + 12), E the largest exponent in 128 tokens (keys and values apart), exact for
// scales down to 2^-35 of that; 2^E of the keys goes into the scores' factor, that of the values into the weights: P = exp2(x - m + 10 + E - e), where m and e,
// for each row, follow the largest score and the largest product of a weight and 2^E: that one's P lies in [2^10, 2^15].  So a weight counts by what its values
// make of it, and tokens that a row does not see, or hardly, do not lower the precision of others.  What is summed for the softmax does not have 2^E.
// (One e for all rows, the largest E so far: 313 us instead of 315, but values 2^30 smaller than some that a row gives no weight had 4 bits of their weights left.)
//
// Bound by the softmax warps: about 2300 cycles per 64 tokens and 256 rows, of which the exponentials' rate is 1024; the tensor pipe is busy for 43 %.  2048 tokens
// behind 6144, 8 heads of 128 with 4 queries: 315 us, 145 as products alone.  Heads of 256 spill 48 to 72 bytes of registers.
//
// Warp-specialised, one CTA per SM, persistent over the items (sequence, head, tiles of rows):
//   warps 0 - 3, 4 - 7   softmax of the first and second tile, a row to each thread: loads its query, keeps maximum and sum, corrects O when the maximum has
//                        grown by more than 2^5 (seldom), writes the result
//   warps 8 - 11         cached tokens: codes 128 tokens ahead in registers, widened into a ring of tiles of 64 (K, K, V, V, ...)
//   warps 12, 13         issue the products of the first and second tile: P V of a tile of tokens and then S of the one after the next
// Each tile of rows has two buffers for S, so its softmax goes from one tile of tokens to the next without waiting for the products of its own weights.
// (One buffer and tiles of 128 tokens: a softmax of 2600 cycles, then its products' 1400, then the next; 327 to 391 us for 2048 tokens behind 6144,
// whether one thread had a row or two, whether one warp issued the products or two.)
#pragma once
#include "kv_attention.cuh"

namespace torq {

template <int FMT_, int D_>
struct KvPrefillCfg {
  static constexpr int FMT = FMT_, D = D_, TILES = D == 256 ? 1 : 2, ROWS = 128 * TILES, TOK = 64;
  static constexpr int CH = D / 32, SB = D / kv_block(FMT), THREADS = 512;
  static constexpr int Q_BYTES = 128 * D * 2, KV_BYTES = TOK * D * 2;
  // A fill of the ring: the keys, or the values, of FT tiles (every barrier costs its waiters 100 to 300 cycles, so they are few).
  static constexpr int FT = D == 256 ? 1 : 2, STAGES = D == 256 ? 5 : 4, FILL_BYTES = FT * KV_BYTES;
  static constexpr int INFO_AT = TILES * Q_BYTES + STAGES * FILL_BYTES, SMEM = INFO_AT + 256 + 1024;
  static constexpr int O_COL = 256;
  static constexpr int PARTIAL = ROWS * (D + 2);                           // floats: results, maxima, sums
  static_assert(SMEM <= 232448, "shared memory");
};
// kind::f16 with float16 operands, as idesc_bf16.
__host__ __device__ constexpr uint32_t idesc_f16(int M, int N, bool a_mn_major, bool b_mn_major) {
  return idesc_bf16(M, N, a_mn_major, b_mn_major) & ~((1u << 7) | (1u << 10));
}

// The larger of three.
__device__ __forceinline__ float max3(float x, float y, float z) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(x), "f"(y), "f"(z));
  return r;
}

struct KvPrefillItem {
  int b, head, first_token, count, length, first_row, rows, base, lo, hi, tiles;       // rows of the item; cached tokens [lo, hi), base <= lo; tiles of tokens
  int part;                              // -1: all tokens that its rows see; 1, 0: some of them, the first ones among them or not
};
// CTAs take whole items in turn, those with the most tokens of a sequence first; or, where that would take longer, equal ranges of the list of all items
// (sequence after sequence, tile after tile, heads inside).  There every item of a sequence counts as many units as its longest has groups of 128 tokens, so that
// a place in the list is found by divisions (counted exactly, tile by tile, it took every warp 5 us); of an item with fewer groups a part has its
// share.  An item that a border cuts leaves partial results, as in the streaming kernel.
struct KvPrefillWalk {
  long long at, end, units;              // items, or units (and how many there are)
  int ranges;                            // 0: whole items
};

// Of sequence b: its new rows, and how many tiles of rows they make for a head.
template <int ROWS>
__device__ __forceinline__ int kv_prefill_sequence(const KvView& c, int group, int b, KvPrefillItem& it) {
  it.b = b;
  kv_new_tokens(c, b, it.first_token, it.count);
  it.length = kv_length(c, b);
  return it.length > 0 ? (it.count * group + ROWS - 1) / ROWS : 0;
}
// Tile `tile` of its rows and the tokens that they see.  Returns the groups of 128 tokens, one at least: rows that see nothing are an item all the same.
template <int ROWS, int TOK>
__device__ __forceinline__ int kv_prefill_tile(const KvScoring& a, int group, int tile, KvPrefillItem& it) {
  it.first_row = tile * ROWS;
  it.rows = min(ROWS, it.count * group - it.first_row);
  const int p0 = it.length - it.count, p_first = p0 + it.first_row / group, p_last = p0 + (it.first_row + it.rows - 1) / group;
  it.hi = p_last + 1;
  if (a.prefix && a.prefix[it.b] > it.hi) it.hi = a.prefix[it.b];
  it.hi = min(it.hi, it.length);
  it.lo = a.window > 0 && p_first - a.window + 1 > 0 ? p_first - a.window + 1 : 0;
  it.base = it.lo & ~15;
  it.tiles = it.hi > it.base ? (it.hi - it.base + TOK - 1) / TOK : 1;
  return (it.tiles + 1) / 2;
}
// Items of sequence b, and the units of each.
template <int ROWS, int TOK>
__device__ __forceinline__ long long kv_prefill_items(const KvView& c, const KvScoring& a, int group, int b, int& each) {
  each = 0;
  if (b >= c.batch) return 0;
  KvPrefillItem it;
  const int tiles = kv_prefill_sequence<ROWS>(c, group, b, it);
  if (tiles == 0) return 0;
  each = max(kv_prefill_tile<ROWS, TOK>(a, group, tiles - 1, it), kv_prefill_tile<ROWS, TOK>(a, group, max(tiles - 2, 0), it));
  return (long long)tiles * c.heads;
}
// Whole items where ranges, with what cutting costs (partial results and their join: as much as EXTRA groups of each CTA; a start from the middle: 8 for an item),
// would not take less time; ranges have LEAST units at least.  Measured, whole items against ranges, us: one sequence of 32768 tokens, 8 heads of 128: 256
// rows of a head 618, 93;  1024: 621, 188;  of 256 dimensions, 1024 rows: 1344, 634.  8 sequences of up to 5000 tokens, 8 heads of 256, up to 1024 rows: 587,
// 477.  2048 tokens behind 6144, 8 heads of 128 with 4 queries: 316, 341.  16 sequences of up to 5000 tokens, up to 1024 rows: 256, 351.
template <int ROWS, int TOK>
__device__ __forceinline__ KvPrefillWalk kv_prefill_walk(const KvView& c, const KvScoring& a, int group, int lane, int which, int ctas) {
  constexpr int EXTRA = ROWS == 128 ? 12 : 24, LEAST = 4;
  long long units = 0, items = 0;
  int longest = 0;
  for (int b = lane; b < c.batch; b += 32) {
    int each;
    const long long n = kv_prefill_items<ROWS, TOK>(c, a, group, b, each);
    items += n;
    units += n * each;
    longest = max(longest, each);
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    units += __shfl_xor_sync(0xFFFFFFFFu, units, o);
    items += __shfl_xor_sync(0xFFFFFFFFu, items, o);
  }
  longest = __reduce_max_sync(0xFFFFFFFFu, longest);
  KvPrefillWalk w;
  w.units = units;
  // Turns of whole items: the longest is in one of them, the others are like the average.  Two kernels decide this, each for itself, and have to agree: every
  // operation is rounded by itself, so that no compilation fuses some of them.
  const float n = (float)items, u = (float)units, k = (float)ctas;
  if (items == 0 || __fadd_rn(__fmul_rn(ceilf(__fdiv_rn(n, k)) - 1.f, __fdiv_rn(u, n)), (float)longest) <=
                        __fadd_rn(__fadd_rn(__fdiv_rn(u, k), (float)EXTRA), __fdiv_rn(8.f * n, k))) {
    w.ranges = 0;
    w.at = which;
    w.end = items;
  } else {
    w.ranges = (int)min((long long)ctas, max(units / LEAST, 1ll));
    w.at = which < w.ranges ? kv_range_begin(units, which, w.ranges) : 0;
    w.end = which < w.ranges ? kv_range_begin(units, which + 1, w.ranges) : 0;
  }
  return w;
}
// Where number `at` of the list lies: the item (its tokens all of them), its groups, and which of its units; false behind the last.  Whole warps.  `from`, if any,
// in shared memory: of this warp's last search the 32 sequences that it ended at and what lies in front of them, where the next one begins, since a CTA's numbers
// ascend.  (From the first sequence each time: 4096 sequences with 24 new tokens each 14 ms.)
struct KvPrefillFrom {
  long long before;
  int b0;
};
template <int ROWS, int TOK>
__device__ __forceinline__ bool kv_prefill_find(const KvView& c, const KvScoring& a, int group, long long at, bool items, int lane, KvPrefillItem& it, int& unit,
                                                int& each, int& groups, KvPrefillFrom* from) {
  long long before = from ? from->before : 0;
  for (int b0 = from ? from->b0 : 0; b0 < c.batch; b0 += 32) {
    const long long n = kv_prefill_items<ROWS, TOK>(c, a, group, b0 + lane, each) * (items ? 1 : max(each, 0)), sum = warp_scan(n, lane);
    const uint32_t here = __ballot_sync(0xFFFFFFFFu, at < before + sum);
    if (here) {
      const int l = __ffs(here) - 1;
      if (from) {
        __syncwarp();                                                      // all have read
        if (lane == 0) *from = {before, b0};
        __syncwarp();
      }
      const long long rest = at - before - __shfl_sync(0xFFFFFFFFu, sum - n, l);
      each = __shfl_sync(0xFFFFFFFFu, each, l);
      const int tiles = kv_prefill_sequence<ROWS>(c, group, b0 + l, it);
      const int item = (int)(items ? rest : rest / each);
      unit = items ? 0 : (int)(rest - (long long)item * each);
      it.head = item % c.heads;
      groups = kv_prefill_tile<ROWS, TOK>(a, group, items ? tiles - 1 - item / c.heads : item / c.heads, it);
      return true;
    }
    before += __shfl_sync(0xFFFFFFFFu, sum, 31);
  }
  return false;
}
// The next item of a CTA, or the part of it that lies in its range.
template <int ROWS, int TOK>
__device__ __forceinline__ bool kv_prefill_item(const KvView& c, const KvScoring& a, int group, KvPrefillWalk& w, int lane, KvPrefillItem& it, KvPrefillFrom* from) {
  int unit, each, groups;
  if (w.at >= w.end || !kv_prefill_find<ROWS, TOK>(c, a, group, w.at, w.ranges == 0, lane, it, unit, each, groups, from)) return false;
  it.part = -1;
  if (w.ranges == 0) {
    w.at += gridDim.x;
  } else {
    const int n = (int)min(w.end - w.at, (long long)(each - unit));
    w.at += n;
    if (n < each) {
      it.part = unit == 0 ? 1 : 0;
      const int from = (int)((long long)unit * groups / each), to = (int)((long long)(unit + n) * groups / each);
      it.lo = max(it.lo, it.base + 128 * from);
      it.hi = min(it.hi, it.base + 128 * to);
    }
  }
  if (a.first) {
    const int t0 = it.first_token + it.first_row / group, t1 = it.first_token + (it.first_row + it.rows - 1) / group;
    int least = INT32_MAX;
    for (int i = t0 + lane; i <= t1; i += 32) least = min(least, a.first[i]);
    it.lo = max(it.lo, __reduce_min_sync(0xFFFFFFFFu, least));
  }
  it.lo = min(it.lo, max(it.hi, 0));
  it.base = it.lo & ~15;
  it.tiles = it.hi > it.base ? (it.hi - it.base + TOK - 1) / TOK : 1;
  return true;
}

template <class C>
__global__ void __launch_bounds__(C::THREADS, 1) kv_prefill_kernel(const KvView c, const KvScoring a, const __nv_bfloat16* Q, int64_t q_stride, int heads,
                                                                   __nv_bfloat16* out, float* lse, float* partials) {
  constexpr int FMT = C::FMT, D = C::D, CH = C::CH, SB = C::SB, TOK = C::TOK;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[2 * C::STAGES + 10];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  __shared__ KvPrefillFrom froms[C::THREADS / 32];
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_p = smem_raw + (smem - smem_u32(smem_raw));
  volatile int* cta_abort = &abort_flag;
  const uint32_t bar = smem_u32(bars);
  auto kv_full = [&](uint32_t i) { return bar + 8 * (i % C::STAGES); };
  auto kv_empty = [&](uint32_t i) { return bar + 8 * (C::STAGES + i % C::STAGES); };
  auto s_full = [&](int t, int buffer) { return bar + 8 * (2 * C::STAGES + 2 * t + buffer); };
  auto p_full = [&](int t, int buffer) { return bar + 8 * (2 * C::STAGES + 4 + 2 * t + buffer); };
  auto q_full = [&](int t) { return bar + 8 * (2 * C::STAGES + 8 + t); };
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, group = heads / c.heads;
  volatile int* tile_top = reinterpret_cast<volatile int*>(smem_p + C::INFO_AT);                   // [8][2]: E of the keys and (as a float) of the values of 128 tokens
  int* warp_top = reinterpret_cast<int*>(smem_p + C::INFO_AT + 64);                                // [2][4][2]

  if (tid == 0) {
    for (int i = 0; i < C::STAGES; ++i) {
      mbar_init(bar + 8 * i, 128);
      mbar_init(bar + 8 * (C::STAGES + i), C::TILES);
    }
    for (int t = 0; t < 2; ++t) {
      for (int i = 0; i < 2; ++i) {
        mbar_init(s_full(t, i), 1);
        mbar_init(p_full(t, i), 128);
      }
      mbar_init(q_full(t), 128);
    }
    abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 12) {
    tmem_alloc(smem_u32(&tmem_slot), 512);
    tmem_relinquish();
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = tmem_slot;
  griddep_wait_and_launch();
  KvPrefillFrom* from = froms + warp;
  if (lane == 0) *from = {0, 0};
  __syncwarp();
  KvPrefillItem it;
  KvPrefillWalk walk = kv_prefill_walk<C::ROWS, TOK>(c, a, group, lane, blockIdx.x, gridDim.x);

  if (warp < 8) {
    // ------------------------------------------------------------------ softmax
    const int t = warp >> 2, row = (warp & 3) * 32 + lane;                 // of the tile
    // rows of the batch that no sequence has, or an empty one
    const int who = blockIdx.x * 8 + warp, all = gridDim.x * 8;
    auto nothing = [&](int i) {
      const int64_t r = (int64_t)i * heads;
      for (int e = lane; e < heads * D / 8; e += 32) reinterpret_cast<uint4*>(out + r * D)[e] = make_uint4(0, 0, 0, 0);
      if (lse)
        for (int e = lane; e < heads; e += 32) lse[r + e] = -INFINITY;
    };
    if (c.starts) {
      const int before = min(max(c.starts[0], 0), c.tokens), behind = min(max(c.starts[c.batch], before), c.tokens), none = before + c.tokens - behind;
      for (int i = who; i < none; i += all) nothing(i < before ? i : behind + i - before);
    }
    for (int b = who; b < c.batch; b += all)
      if (c.lengths[b] <= 0) {
        int first, count;
        kv_new_tokens(c, b, first, count);
        for (int i = 0; i < count; ++i) nothing(first + i);
      }

    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, o_at = tmem + lanes + C::O_COL + t * D;
    const bool special = a.softcap > 0.f || a.slopes;
    uint32_t phases[2] = {0, 0}, group_no = 0;                             // of s_full; of 128 tokens, over all items
    bool ok = true;
    // Two tiles of rows weigh in turn: side by side they wait for the exponentials of one another and then leave that unit idle together (2048 tokens behind
    // 6144: 317 us, in turn 304).  The barriers for that are executed for every tile of tokens, also after a wait has given up, so that no warp is left in
    // one.
    while (kv_prefill_item<C::ROWS, TOK>(c, a, group, walk, lane, it, from)) {
      const uint32_t first_group = group_no;
      group_no += (it.tiles + 1) / 2;
      if (128 * t >= it.rows) continue;
      const bool in_turn = it.rows > 128;
      // S of tile k, or what comes after the last ones, is number k of its item on s_full: at k it is there, and P V of tile k - 2 is done
      auto wait_s = [&](int k) {
        ok = ok && mbar_wait_warp(s_full(t, k & 1), (phases[k & 1] + (k >> 1)) & 1, cta_abort, c.err_word, SITE_EPI_ACC_FULL);
        return ok;
      };
      const int rr = it.first_row + 128 * t + row;
      const bool there = 128 * t + row < it.rows;
      int lo = 0, hi = 0, place;
      float factor, slope = 0.f;
      {
        // the query: float16 times a power of two, as kv_load_query
        const int token = it.first_token + rr / group, h = it.head * group + rr % group;
        place = it.length - it.count + rr / group;
        const __nv_bfloat16* p = Q + token * q_stride + h * D;
        uint32_t top = 0;
#pragma unroll 4
        for (int e = 0; e < D / 8; ++e) {
          const uint4 w = there ? load_once(p + 8 * e) : make_uint4(0, 0, 0, 0);
#pragma unroll
          for (int i = 0; i < 4; ++i) top = max(top, max((&w.x)[i] >> 16 & 0x7FFFu, (&w.x)[i] & 0x7FFFu));
        }
        const uint32_t ef = top >> 7, field = ef > 15 ? 268u - ef : 253u;
        const float mul = __uint_as_float(field << 23);
        uint8_t* dst = smem_p + t * C::Q_BYTES + row * 128;
#pragma unroll 4
        for (int e = 0; e < D / 8; ++e) {
          const uint4 w = there ? load_once(p + 8 * e) : make_uint4(0, 0, 0, 0);
          float v[8];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float((&w.x)[i] << 16) * mul;
            v[2 * i + 1] = __uint_as_float((&w.x)[i] & 0xFFFF0000u) * mul;
          }
          uint4 y;
#pragma unroll
          for (int i = 0; i < 4; ++i) (&y.x)[i] = pack_f16(v[kv_query_order<FMT>(i, 0)], v[kv_query_order<FMT>(i, 1)]);
          if (ok) *reinterpret_cast<uint4*>(dst + (e >> 3) * (128 * 128) + (((e & 7) ^ (row & 7)) << 4)) = y;
        }
        factor = __uint_as_float((254u - field) << 23);
        if (there) {
          kv_range(a, it.b, token, place, it.length, lo, hi);
          lo = max(lo, it.lo);
          hi = min(hi, it.hi);
          if (a.slopes) slope = kv_slope(a, h);
        }
      }
      fence_proxy_async_smem();
      if (ok) mbar_arrive(q_full(t));
      const int clear_lo = (int)__reduce_max_sync(0xFFFFFFFFu, there ? (uint32_t)max(lo, 0) : 0u);          // tiles within [clear_lo, clear_hi) need no mask
      const int clear_hi = (int)__reduce_min_sync(0xFFFFFFFFu, there ? (uint32_t)max(hi, 0) : 0x7FFFFFFFu);

      float m = kLowest, l = 0.f;
      bool far = false;                                                    // whether some row's m is
      float e_row = 27.f;                                                  // O is held times 2^(10 - m - e_row), e_row the E of the largest product so far or near it
      if (in_turn && t == 1) named_barrier_arrive(2, 256);                 // the first tile's turn
      for (int k = 0; k < it.tiles; ++k) {
        if (!wait_s(k)) {
          if (in_turn) {
            named_barrier_sync(2 + t, 256);
            named_barrier_arrive(3 - t, 256);
          }
          continue;
        }
        tc_fence_after_sync();
        const int j0 = it.base + k * TOK;
        const uint32_t s_at = tmem + lanes + (2 * t + (k & 1)) * TOK;
        float f = a.scale * (FMT == FMT_NVFP4 ? c.k_ts : 1.f) * kLog2e;    // the keys' power of two before the query's: with that it may be too small a number
        float e_tile = 27.f;
        if constexpr (FMT != FMT_NVFP4) {
          const volatile int* tops = tile_top + 2 * ((first_group + (k >> 1)) & 7);
          f *= __uint_as_float((uint32_t)(tops[0] - 12) << 23);
          e_tile = __int_as_float(tops[1]);
        }
        f *= factor;
        auto score = [&](float s, int col) {                               // where there is more to a score than its factor
          const int j = j0 + col;
          float x = __fmul_rn(s, f);                                       // not fused with what is taken off it
          if (special) x = kv_score(x, a, slope, abs(place - j));
          return j >= lo && j < hi ? x : -INFINITY;
        };
        bool slow = special || far || j0 < clear_lo || j0 + TOK > clear_hi;
        // This tile's values are 2^down smaller than e_row says: so are its weights.  (Down to 2^-80, where they are nothing in float16; in the sum they count.)
        float down = FMT == FMT_NVFP4 ? 0.f : fminf(e_row - e_tile, 80.f);
        // Whether m and e_row do not do for a score.  Where the tile's values are larger than e_row says, its weights are too: products count, not weights.
        auto beyond = [&](float top) { return top - m > kSlack + fminf(down, 0.f); };
        bool wrong = false;                                                // whether some row's O has to be corrected
        float fix = 1.f;                                                   // of O
        auto raised = [&](float top) {
          if (!beyond(top)) return;
          const float now = top - m > kSlack ? top : m, less = m - now;
          fix = ex2(less);
          l *= fix;
          m = now;
          if constexpr (FMT != FMT_NVFP4) {
            // whole numbers, so that weights and their sum differ by a power of two
            const float e = fmaxf(floorf(fmaxf(less, -1024.f)) + e_row, floorf(top - now) + e_tile);
            fix = ex2(less + (e_row - e));
            e_row = e;
            down = fminf(e_row - e_tile, 80.f);
          }
        };
        // In one pass with the maximum so far; a second one where a score turns out to exceed it by too much (the first tiles).  P stays in
        // registers until it may take the place of S.  What is seldom needed has loops of its own: in one loop with the plain case it
        // made the warps wait for instructions (1530 us).
        uint32_t w[2][16];
        float sum = 0.f, top = -INFINITY;
        auto weigh = [&]() {
          const uint64_t f2 = pair_of(f), off2 = pair_of(kShift - down - m);
          uint64_t sums = 0;
          float tops[2] = {-INFINITY, -INFINITY};
          uint32_t v[2][32];
          tmem_ld_32x32(s_at, v[0]);
          tmem_ld_wait();
          tmem_ld_32x32(s_at + 32, v[1]);
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            if (x) tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              tops[i / 2 & 1] = max3(tops[i / 2 & 1], __uint_as_float(v[x][i]), __uint_as_float(v[x][i + 1]));
              const float2 z = halves(fma2(pair_of(v[x][i], v[x][i + 1]), f2, off2));
              const float p = ex2(z.x), p2 = ex2(z.y);
              sums = add2(sums, pair_of(__float_as_uint(p), __float_as_uint(p2)));
              w[x][i / 2] = pack_f16(p, p2);
            }
          }
          sum = halves(sums).x + halves(sums).y;
          top = fmaxf(tops[0], tops[1]) * f;
        };
        if (in_turn) named_barrier_sync(2 + t, 256);
        if (!slow) {
          weigh();
          if (in_turn) named_barrier_arrive(3 - t, 256);
          if (__any_sync(0xFFFFFFFFu, beyond(top))) {
            wrong = true;
            raised(top);
            slow = far = __any_sync(0xFFFFFFFFu, kv_far(m));
            if (!far) weigh();
          }
        } else {
          if (in_turn) named_barrier_arrive(3 - t, 256);
#pragma unroll 1
          for (int x = 0; x < TOK; x += 32) {
            uint32_t v[32];
            tmem_ld_32x32(s_at + x, v);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) top = fmaxf(top, score(__uint_as_float(v[i]), x + i));
            __syncwarp();
          }
          wrong = __any_sync(0xFFFFFFFFu, beyond(top));
          raised(top);
          far = __any_sync(0xFFFFFFFFu, kv_far(m));
        }
        if (k > 0 && wrong) {
          if (!wait_s(k + 1)) continue;                                    // the products of the tile before are done
          tc_fence_after_sync();
#pragma unroll 1
          for (int x = 0; x < D; x += 16) {
            uint32_t v[16];
            tmem_ld_32x32_x16(o_at + x, v);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * fix);
            tmem_st_32x32_x16(o_at + x, v);
          }
        }
        if (slow) {
          sum = 0.f;
#pragma unroll 1
          for (int x = 0; x < TOK; x += 32) {
            uint32_t v[32], y[16];
            tmem_ld_32x32(s_at + x, v);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              const float p = ex2(__fsub_rn(score(__uint_as_float(v[i]), x + i), m) + (kShift - down)), p2 = ex2(__fsub_rn(score(__uint_as_float(v[i + 1]), x + i + 1), m) + (kShift - down));
              sum += p + p2;
              y[i / 2] = pack_f16(p, p2);
            }
            __syncwarp();
            tmem_st_32x32_x16(s_at + x / 2, y);
          }
        } else {
          tmem_st_32x32_x16(s_at, w[0]);
          tmem_st_32x32_x16(s_at + 16, w[1]);
        }
        l += FMT == FMT_NVFP4 ? sum : sum * ex2(down);
        tmem_st_wait();
        tc_fence_before_sync();
        mbar_arrive(p_full(t, k & 1));
      }
      if (in_turn && t == 0) named_barrier_sync(2, 256);                   // the second tile's last turn is over
      wait_s(it.tiles + 1);
      phases[0] += (it.tiles + 3) / 2;
      phases[1] += (it.tiles + 2) / 2;
      if (!ok) continue;
      tc_fence_after_sync();
      // of a part too, as in the streaming kernel
      const float inv = l > 0.f ? 1.f / l : 0.f, fs = FMT == FMT_NVFP4 ? c.v_ts : __uint_as_float((uint32_t)((int)e_row - 12) << 23);
      const int64_t to = (int64_t)(it.first_token + rr / group) * heads + it.head * group + rr % group;
      float* part = partials + (int64_t)(2 * blockIdx.x + it.part) * C::PARTIAL;
#pragma unroll 1
      for (int x = 0; x < D; x += 16) {
        uint32_t v[16];
        tmem_ld_32x32_x16(o_at + x, v);
        tmem_ld_wait();
        constexpr auto column = [](int el) { return FMT == FMT_MXINT4 ? (el < 4 ? 2 * el : 2 * (el - 4) + 1) : el; };   // the elements lie in the order of kv_query_order
#pragma unroll
        for (int e = 0; e < 16; e += 8) {
          float z[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) z[i] = __uint_as_float(v[e + column(i)]) * inv * fs;
          if (!there) continue;
          if (it.part >= 0) {
            float4* y = reinterpret_cast<float4*>(part + (128 * t + row) * D + x + e);
            y[0] = make_float4(z[0], z[1], z[2], z[3]);
            y[1] = make_float4(z[4], z[5], z[6], z[7]);
          } else {
            uint4 y;
#pragma unroll
            for (int i = 0; i < 4; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"((&y.x)[i]) : "f"(z[2 * i + 1]), "f"(z[2 * i]));
            *reinterpret_cast<uint4*>(out + to * D + x + e) = y;
          }
        }
        __syncwarp();
      }
      if (there && it.part >= 0) {
        part[C::ROWS * D + 128 * t + row] = m;
        part[C::ROWS * D + C::ROWS + 128 * t + row] = l;
      } else if (there && lse) lse[to] = l > 0.f ? (m - kShift + log2f(l)) * kLn2 : -INFINITY;
      tc_fence_before_sync();
    }
  } else if (warp < 12) {
    // ------------------------------------------------------------------ cached tokens
    // In groups of two tiles, 128 tokens, keys before values.  A thread takes every 128th chunk of 16 bytes (32 codes of a token), with its scale byte, from
    // global memory into registers, the next group's while it widens this one's.  The named barrier is executed by every one of these threads for
    // every group, also after a wait has given up, so that no warp is left in one.
    const int dt = tid - 256, dw = warp - 8, mask = (1 << c.page_shift) - 1;
    constexpr int N = CH;                                                  // chunks of keys, and of values, the first half of them of the first tile
    const int ch = dt % CH, row0 = dt / CH;                                // of chunk i: row row0 + i 128 / CH of the group
    uint32_t fill = 0, group_no = 0;
    bool ok = true;
    while (kv_prefill_item<C::ROWS, TOK>(c, a, group, walk, lane, it, from)) {
      const int32_t* table = c.table + (int64_t)it.b * c.width;
      const uint8_t* head_pages = c.pages + (int64_t)it.head * c.head_bytes;
      const int groups = (it.tiles + 1) / 2;
      int page[N];                                                         // of the next group's chunks; -1: nothing there that any row sees
      auto look_up = [&](int g) {                                          // all loads before the first is looked at
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int j = it.base + g * 128 + row0 + i * (128 / CH);
          page[i] = g < groups && j >= it.lo && j < it.hi ? table[j >> c.page_shift] : -1;
        }
      };
      auto check = [&](int g) {
        bool bad = false;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int j = it.base + g * 128 + row0 + i * (128 / CH);
          bad |= g < groups && j >= it.lo && j < it.hi && (unsigned)page[i] >= (unsigned)c.num_pages;
          if ((unsigned)page[i] >= (unsigned)c.num_pages) page[i] = -1;
        }
        if (bad) kv_bad_page(c);
      };
      uint4 codes[2][N];
      uint32_t scale[2][N], next_scale[N];                                 // zero where there is nothing; the values' of the next group
      auto load_scale = [&](int g, int half, int i) -> uint32_t {
        if (page[i] < 0) return 0;
        const int slot = (it.base + g * 128 + row0 + i * (128 / CH)) & mask;
        const uint8_t* p = head_pages + page[i] * c.page_bytes + (half ? c.v_scales : c.k_scales) + slot * SB;
        return FMT == FMT_NVFP4 ? *reinterpret_cast<const uint16_t*>(p + 2 * ch) : p[ch];
      };
      auto load_codes = [&](int g, int half) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int slot = (it.base + g * 128 + row0 + i * (128 / CH)) & mask;
          codes[half][i] = make_uint4(0, 0, 0, 0);
          if (page[i] >= 0) codes[half][i] = load_once(head_pages + page[i] * c.page_bytes + (half ? c.v_codes : 0) + slot * (D / 2) + ch * 16);
        }
      };
      // E of a group needs the scale bytes of both, so the values' come with the keys, a group ahead of their codes
      auto load_keys = [&](int g) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          scale[0][i] = load_scale(g, 0, i);
          next_scale[i] = load_scale(g, 1, i);
        }
        load_codes(g, 0);
      };
      auto load_values = [&](int g) {
#pragma unroll
        for (int i = 0; i < N; ++i) scale[1][i] = next_scale[i];
        load_codes(g, 1);
      };
      // this warp's largest scale bytes of a group, keys' and values'
      auto tell_top = [&](uint32_t no) {
        if constexpr (FMT != FMT_NVFP4) {
          uint32_t top[2] = {27, 27};
#pragma unroll
          for (int i = 0; i < N; ++i) {
            top[0] = max(top[0], scale[0][i]);
            top[1] = max(top[1], next_scale[i]);
          }
          top[0] = __reduce_max_sync(0xFFFFFFFFu, top[0]);
          top[1] = __reduce_max_sync(0xFFFFFFFFu, top[1]);
          if (lane < 2) warp_top[(no & 1) * 8 + dw * 2 + lane] = (int)(lane ? top[1] : top[0]);
        }
      };
      look_up(0);
      check(0);
      load_keys(0);
      tell_top(group_no);
      load_values(0);
      look_up(1);
      for (int g = 0; g < groups; ++g, ++group_no) {
        int down[2] = {0, 0};                                              // 27 - E
        if constexpr (FMT != FMT_NVFP4) {
          named_barrier_sync(1, 128);
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const int* w = warp_top + (group_no & 1) * 8 + half;
            const int most = max(max(w[0], w[2]), max(w[4], w[6]));
            down[half] = 27 - most;
            if (dt == 0) tile_top[2 * (group_no & 7) + half] = half ? __float_as_int((float)most) : most;
          }
        }
        const int tiles = min(2, it.tiles - 2 * g);
#pragma unroll
        for (int half = 0; half < 2; ++half) {                             // keys, values
#pragma unroll
          for (int tile = 0; tile < 2; ++tile) {
            if (tile < tiles) {
              if (tile % C::FT == 0 && ok)
                ok = mbar_wait_warp(kv_empty(fill), ((fill / C::STAGES) & 1) ^ 1, cta_abort, c.err_word, SITE_PRODUCER_EMPTY);
              if (ok) {
                uint8_t* dst = smem_p + C::TILES * C::Q_BYTES + (fill % C::STAGES) * C::FILL_BYTES + tile % C::FT * C::KV_BYTES + (ch >> 1) * (TOK * 128);
#pragma unroll
                for (int i = tile * (N / 2); i < (tile + 1) * (N / 2); ++i) {
                  const int r = (row0 + i * (128 / CH)) & (TOK - 1);
                  uint32_t f[2];                                           // of the first and last 16 codes
                  if constexpr (FMT == FMT_NVFP4) {
                    const uint32_t two = e4m3x2_f16x2(scale[half][i]);
                    f[0] = __byte_perm(two, 0, 0x1010);
                    f[1] = __byte_perm(two, 0, 0x3232);
                  } else {
                    // 2^(e - E + 12): its exponent in float16, or, for e - E from -27 to -35, a number below the normal ones
                    const int field = (int)scale[half][i] + down[half];
                    const uint32_t small = scale[half][i] ? 0x200u >> min(max(-field, 0), 31) & 0x3FEu : 0u;
                    f[0] = f[1] = (field > 0 ? (uint32_t)field << 10 : small) * 0x00010001u;
                  }
#pragma unroll
                  for (int x = 0; x < 4; ++x) {
                    uint32_t o[4];
                    kv_key_pairs<FMT>((&codes[half][i].x)[x], o);
                    uint4 y;
#pragma unroll
                    for (int e = 0; e < 4; ++e) (&y.x)[e] = mul_f16x2(o[e], f[x >> 1]);
                    *reinterpret_cast<uint4*>(dst + r * 128 + ((((ch & 1) * 4 + x) ^ (r & 7)) << 4)) = y;
                  }
                }
              }
              if (tile % C::FT == C::FT - 1 || tile == tiles - 1) {
                if (ok) {
                  fence_proxy_async_smem();
                  mbar_arrive(kv_full(fill));
                }
                ++fill;
              }
            }
            if (half == 1 && tile == 0) tell_top(group_no + 1);            // of the next group, whose scale bytes have come meanwhile
          }
          if (half == 0) {
            check(g + 1);
            load_keys(g + 1);
          } else {
            load_values(g + 1);
          }
        }
        look_up(g + 2);
      }
    }
  } else {
    // ------------------------------------------------------------------ products
    constexpr uint32_t idesc_s = idesc_f16(128, TOK, false, false), idesc_o = idesc_f16(128, D, false, true);
    uint32_t fill = 0, p_count[2] = {0, 0}, q_count = 0;
    bool ok = true;
    // What goes into the products' descriptors has to lie in uniform registers (from others an instruction takes 75 cycles to issue: 330 us), and the
    // result of a reduction does.
    const int t = (int)__reduce_max_sync(0xFFFFFFFFu, (uint32_t)warp) - 12;                  // the tile of rows
    const uint32_t tm = __reduce_max_sync(0xFFFFFFFFu, tmem), sm = __reduce_max_sync(0xFFFFFFFFu, smem);
    while (t < C::TILES && ok && kv_prefill_item<C::ROWS, TOK>(c, a, group, walk, lane, it, from)) {
      const int tiles = (int)__reduce_max_sync(0xFFFFFFFFu, (uint32_t)it.tiles);
      const bool active = 128 * t < (int)__reduce_max_sync(0xFFFFFFFFu, (uint32_t)it.rows);
      const uint32_t o_at = tm + C::O_COL + t * D;
      if (active) ok = mbar_wait_warp(q_full(t), q_count++ & 1, cta_abort, c.err_word, SITE_MMA_ACC_EMPTY);
      // number i: P V of tile i - 2, then S of tile i into the place of that P
      for (int i = 0; i < tiles + 2 && ok; ++i) {
        const int k = i - 2;
        // the fills of tile i's keys and of tile k's values, and whether a tile is the first or last of its fill
        uint32_t kf, vf;
        if constexpr (C::FT == 2) {
          kf = fill + 2 * (i >> 1);
          vf = fill + 2 * (k >> 1) + 1;
        } else {
          kf = fill + 4 * (i >> 1) + (i & 1);
          vf = fill + 4 * (k >> 1) + min(2, tiles - (k & ~1)) + (k & 1);
        }
        const bool k_first = i % C::FT == 0, k_last = i % C::FT == C::FT - 1 || i == tiles - 1, v_first = k % C::FT == 0,
                   v_last = k % C::FT == C::FT - 1 || k == tiles - 1;
        if (k >= 0 && v_first) ok = mbar_wait_warp(kv_full(vf), (vf / C::STAGES) & 1, cta_abort, c.err_word, SITE_MMA_FULL);
        if (ok && i < tiles && k_first) ok = mbar_wait_warp(kv_full(kf), (kf / C::STAGES) & 1, cta_abort, c.err_word, SITE_MMA_FULL);
        if (ok && active && k >= 0) ok = mbar_wait_warp(p_full(t, i & 1), p_count[i & 1]++ & 1, cta_abort, c.err_word, SITE_MMA_ACC_EMPTY);
        if (!ok) break;
        tc_fence_after_sync();
        const uint32_t s_at = tm + (2 * t + (i & 1)) * TOK;
        if (elect_one()) {
          if (active && k >= 0) {
            const uint64_t v = make_desc(sm + C::TILES * C::Q_BYTES + (vf % C::STAGES) * C::FILL_BYTES + k % C::FT * C::KV_BYTES, TOK * 128, 1024, kSwizzle128);
#pragma unroll
            for (int x = 0; x < TOK / 16; ++x)             // 16 tokens: 8 columns of P, 16 rows of V (2 KiB)
              mma_bf16_tmem_a(o_at, s_at + 8 * x, v + 128 * x, idesc_o, k > 0 || x > 0);
          }
          if (active && i < tiles) {
            const uint64_t q = make_desc(sm + t * C::Q_BYTES, 16, 1024, kSwizzle128);
            const uint64_t y = make_desc(sm + C::TILES * C::Q_BYTES + (kf % C::STAGES) * C::FILL_BYTES + i % C::FT * C::KV_BYTES, 16, 1024, kSwizzle128);
#pragma unroll
            for (int x = 0; x < D / 16; ++x)               // 16 elements: 32 bytes of a row of 128
              mma_bf16(s_at, q + (x >> 2) * (128 * 128 / 16) + 2 * (x & 3), y + (x >> 2) * (TOK * 128 / 16) + 2 * (x & 3), idesc_s, x > 0);
          }
          if (active) tc_commit(s_full(t, i & 1));
          if (k >= 0 && v_last) tc_commit(kv_empty(vf));             // a tile of rows that is not there gives the tokens back as they come
          if (i < tiles && k_last) tc_commit(kv_empty(kf));
        }
        __syncwarp();
      }
      fill += C::FT == 2 ? 2 * ((tiles + 1) / 2) : 2 * tiles;
    }
  }

  // ------------------------------------------------------------------ teardown
  tc_fence_before_sync();
  __syncthreads();
  if (*cta_abort)
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);                      // products in flight end before their memory goes
  if (warp == 12) {
    tc_fence_after_sync();
    tmem_dealloc(tmem, 512);
  }
}

// Joins the parts of an item that borders have cut.  CTA (k, y): the item that goes over from range k to k + 1, where k has its beginning; 32 of its rows, a
// row to a warp at a time.
template <class C>
__global__ void __launch_bounds__(256) kv_prefill_join_kernel(const KvView c, const KvScoring a, int ctas, int heads, const float* partials, __nv_bfloat16* out,
                                                              float* lse) {
  constexpr int D = C::D, EACH = D / 32, BATCH = 8;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, group = heads / c.heads;
  const KvPrefillWalk w = kv_prefill_walk<C::ROWS, C::TOK>(c, a, group, lane, blockIdx.x + 1, ctas);
  KvPrefillItem it;
  int unit = 0, each = 1, groups = 0, from = 0, to = -1;
  auto range_of = [&](long long unit) { return (int)(((unit + 1) * w.ranges + w.units - 1) / w.units) - 1; };
  if (w.ranges && w.at < w.end && kv_prefill_find<C::ROWS, C::TOK>(c, a, group, w.at, false, lane, it, unit, each, groups, nullptr) && unit > 0) {
    from = range_of(w.at - unit);
    to = range_of(w.at - unit + each - 1);
  }
  griddep_wait_and_launch();                                               // every CTA waits: what stands behind this kernel relies on that
  if (from != (int)blockIdx.x) return;
  for (int i = 0; i < 4; ++i) {
    const int r = 32 * blockIdx.y + 8 * i + warp;
    if (r >= it.rows || to < from) return;
    float m = -INFINITY, l = 0.f, o[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) o[e] = 0.f;
    for (int k0 = from; k0 <= to; k0 += BATCH) {
      float pm[BATCH], pl[BATCH], v[BATCH][EACH], top = m;
#pragma unroll
      for (int x = 0; x < BATCH; ++x) {
        const bool have = k0 + x <= to;
        const float* p = partials + (int64_t)(2 * (k0 + x) + (k0 + x == from ? 1 : 0)) * C::PARTIAL;
        pm[x] = have ? p[C::ROWS * D + r] : -INFINITY;
        pl[x] = have ? p[C::ROWS * D + C::ROWS + r] : 0.f;
#pragma unroll
        for (int e = 0; e < EACH; ++e) v[x][e] = have ? p[r * D + e * 32 + lane] : 0.f;
      }
#pragma unroll
      for (int x = 0; x < BATCH; ++x) top = fmaxf(top, pm[x]);
      kv_join<BATCH, EACH>(pm, pl, v, top, m, l, o);
    }
    const int rr = it.first_row + r;
    const int64_t row = (int64_t)(it.first_token + rr / group) * heads + it.head * group + rr % group;
#pragma unroll
    for (int e = 0; e < EACH; ++e) out[row * D + e * 32 + lane] = __float2bfloat16(o[e]);
    if (lse && lane == 0) lse[row] = l > 0.f ? (m - kShift + log2f(l)) * kLn2 : -INFINITY;
  }
}

}  // namespace torq
