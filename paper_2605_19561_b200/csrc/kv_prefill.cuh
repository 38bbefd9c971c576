// Attention of many new tokens per sequence over the 4-bit cache, on tcgen05: rows (tokens times the query heads of a group) in tiles of 128, two tiles
// to a CTA (D = 256: one), cached tokens in tiles of TOK.
//   S = Q K^T        float16 operands in shared memory, float32 in tensor memory
//   P = exp2(...)    from tensor memory and back into it as float16, in the place of S
//   O += P V         P from tensor memory, V from shared memory
// Keys and values are widened to float16 once per CTA and tile, whatever the number of rows: codes are exact there, with the scales as follows.
// NVFP4: code times E4M3 scale, exact.  MXFP4, MXINT4: code times 2^(e - E + 12), E the largest exponent in the tile (keys and values apart), exact for
// scales down to 2^-35 of that; 2^E of the keys goes into the scores' factor, that of the values into the weights: P = exp2(x - m + 12 + E - E_max), E_max the
// largest E so far, so a tile with smaller values has smaller weights.  What is summed for the softmax does not have it.
//
// Warp-specialised, one CTA per SM, persistent over the items (sequence, head, tiles of rows):
//   warps 0 - 3, 4 - 7   softmax of the first and second tile, a row to each thread: loads its query, keeps maximum and sum, corrects O when the maximum has
//                        grown by more than 2^3 (seldom), writes the result
//   warps 8 - 11         cached tokens: cp.async of the codes one tile ahead, widening into a ring of three tiles (K, V, K, ...)
//   warp 12              issues the products: for every tile of tokens P V of the one before and then the next S, of the first tile of rows, then of the
//                        second, so that one tile's softmax runs beside the other's products
#pragma once
#include "kv_attention.cuh"

namespace torq {

template <int FMT_, int D_>
struct KvPrefillCfg {
  static constexpr int FMT = FMT_, D = D_, TILES = D == 256 ? 1 : 2, ROWS = 128 * TILES, TOK = D == 256 ? 64 : 128;
  static constexpr int CH = D / 32, SB = D / kv_block(FMT), THREADS = 416, GROUPS = TOK / 16;
  static constexpr int Q_BYTES = 128 * D * 2, KV_BYTES = TOK * D * 2, STAGES = 3;
  static constexpr int CODES = TOK * D / 2, SCALES = TOK * SB, RAW = 2 * (CODES + SCALES);
  static constexpr int RAW_AT = TILES * Q_BYTES + STAGES * KV_BYTES, INFO_AT = RAW_AT + 2 * RAW, SMEM = INFO_AT + 512 + 1024;
  static constexpr int O_COL = 256;
  static_assert(SMEM <= 232448, "shared memory");
};
// kind::f16 with float16 operands, as idesc_bf16.
__host__ __device__ constexpr uint32_t idesc_f16(int M, int N, bool a_mn_major, bool b_mn_major) {
  return idesc_bf16(M, N, a_mn_major, b_mn_major) & ~((1u << 7) | (1u << 10));
}

struct KvPrefillItem {
  int b, head, first_token, count, length, first_row, rows, base, lo, hi, tiles;       // rows of the item; cached tokens [lo, hi), base <= lo; tiles of tokens
};

// Item `index` of the list (sequence after sequence, the tiles with the most tokens first, heads inside); false behind the last.  Whole warps.
template <int ROWS, int TOK>
__device__ __forceinline__ bool kv_prefill_item(const KvView& c, const KvScoring& a, int group, long long index, int lane, KvPrefillItem& it) {
  long long before = 0;
  for (int b0 = 0; b0 < c.batch; b0 += 32) {
    int first = 0, count = 0, tiles = 0;
    if (b0 + lane < c.batch) {
      kv_new_tokens(c, b0 + lane, first, count);
      tiles = kv_length(c, b0 + lane) > 0 ? (count * group + ROWS - 1) / ROWS : 0;
    }
    const long long items = (long long)tiles * c.heads, sum = warp_scan(items, lane);
    const uint32_t here = __ballot_sync(0xFFFFFFFFu, index < before + sum);
    if (here) {
      const int l = __ffs(here) - 1;
      const int local = (int)(index - before - __shfl_sync(0xFFFFFFFFu, sum - items, l));
      tiles = __shfl_sync(0xFFFFFFFFu, tiles, l);
      it.b = b0 + l;
      kv_new_tokens(c, it.b, it.first_token, it.count);
      it.length = kv_length(c, it.b);
      it.head = local % c.heads;
      it.first_row = (tiles - 1 - local / c.heads) * ROWS;
      it.rows = min(ROWS, it.count * group - it.first_row);
      const int p0 = it.length - it.count, p_first = p0 + it.first_row / group, p_last = p0 + (it.first_row + it.rows - 1) / group;
      it.hi = p_last + 1;
      if (a.prefix && a.prefix[it.b] > it.hi) it.hi = a.prefix[it.b];
      it.hi = min(it.hi, it.length);
      it.lo = a.window > 0 && p_first - a.window + 1 > 0 ? p_first - a.window + 1 : 0;
      it.base = it.lo & ~15;
      it.tiles = it.hi > it.base ? (it.hi - it.base + TOK - 1) / TOK : 1;  // rows that see nothing are an item all the same
      return true;
    }
    before += __shfl_sync(0xFFFFFFFFu, sum, 31);
  }
  return false;
}

template <class C>
__global__ void __launch_bounds__(C::THREADS, 1) kv_prefill_kernel(const KvView c, const KvScoring a, const __nv_bfloat16* Q, int64_t q_stride, int heads,
                                                                   __nv_bfloat16* out, float* lse) {
  constexpr int FMT = C::FMT, D = C::D, CH = C::CH, SB = C::SB, TOK = C::TOK;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t bars[16];
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag;
  const uint32_t smem = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_p = smem_raw + (smem - smem_u32(smem_raw));
  volatile int* cta_abort = &abort_flag;
  const uint32_t bar = smem_u32(bars);
  auto kv_full = [&](uint32_t i) { return bar + 8 * (i % C::STAGES); };
  auto kv_empty = [&](uint32_t i) { return bar + 24 + 8 * (i % C::STAGES); };
  auto s_full = [&](int t) { return bar + 48 + 8 * t; };
  auto p_full = [&](int t) { return bar + 64 + 8 * t; };
  auto q_full = [&](int t) { return bar + 80 + 8 * t; };
  auto o_full = [&](int t) { return bar + 96 + 8 * t; };
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, group = heads / c.heads;
  volatile int* tile_top = reinterpret_cast<volatile int*>(smem_p + C::INFO_AT);                   // [4][2]: E of the keys and of the values
  int64_t* page_at = reinterpret_cast<int64_t*>(smem_p + C::INFO_AT + 64);                         // [2][GROUPS], -1: nothing there
  int* warp_top = reinterpret_cast<int*>(smem_p + C::INFO_AT + 64 + 2 * 8 * C::GROUPS);            // [2][4][2]

  if (tid == 0) {
    for (int i = 0; i < C::STAGES; ++i) {
      mbar_init(bar + 8 * i, 128);
      mbar_init(bar + 24 + 8 * i, 1);
    }
    for (int t = 0; t < 2; ++t) {
      mbar_init(s_full(t), 1);
      mbar_init(p_full(t), 128);
      mbar_init(q_full(t), 128);
      mbar_init(o_full(t), 1);
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
  KvPrefillItem it;

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

    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, s_at = tmem + lanes + t * TOK, o_at = tmem + lanes + C::O_COL + t * D;
    const bool special = a.softcap > 0.f || a.slopes;
    uint32_t s_count = 0, o_count = 0, tile_no = 0;
    bool ok = true;
    for (long long index = blockIdx.x; ok && kv_prefill_item<C::ROWS, TOK>(c, a, group, index, lane, it); index += gridDim.x) {
      const uint32_t first_tile = tile_no;
      tile_no += it.tiles;
      if (128 * t >= it.rows) continue;
      const int rr = it.first_row + 128 * t + row;
      const bool there = 128 * t + row < it.rows;
      const int token = it.first_token + rr / group, h = it.head * group + rr % group, place = it.length - it.count + rr / group;
      int lo = 0, hi = 0;
      float factor, slope = 0.f;
      {
        // the query: float16 times a power of two, as kv_load_query
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
          *reinterpret_cast<uint4*>(dst + (e >> 3) * (128 * 128) + (((e & 7) ^ (row & 7)) << 4)) = y;
        }
        factor = __uint_as_float((254u - field) << 23) * (a.scale * (FMT == FMT_NVFP4 ? c.k_ts : 1.f) * kLog2e);
        if (there) {
          kv_range(a, it.b, token, place, it.length, lo, hi);
          if (a.slopes) slope = a.slopes[h];
        }
      }
      fence_proxy_async_smem();
      mbar_arrive(q_full(t));

      float m = -1e30f, l = 0.f;
      int e_max = 27;
      for (int k = 0; k < it.tiles; ++k, ++s_count) {
        ok = __all_sync(0xFFFFFFFFu, mbar_wait(s_full(t), s_count & 1, cta_abort, c.err_word, SITE_EPI_ACC_FULL));
        if (!ok) break;
        tc_fence_after_sync();
        const int j0 = it.base + k * TOK;
        const bool masked = __any_sync(0xFFFFFFFFu, there && (j0 < lo || j0 + TOK > hi));
        float f = factor;
        int e_tile = 27;
        if constexpr (FMT != FMT_NVFP4) {
          f *= __uint_as_float((uint32_t)(tile_top[2 * ((first_tile + k) & 3)] - 12) << 23);
          e_tile = tile_top[2 * ((first_tile + k) & 3) + 1];
        }
        auto score = [&](float s, int col) {                               // where there is more to a score than its factor
          const int j = j0 + col;
          float x = s * f;
          if (special) x = kv_score(x * kLn2, a.softcap, slope, abs(place - j));
          return j >= lo && j < hi ? x : -INFINITY;
        };
        const bool slow = masked || special;
        // Two buffers, so that a load from tensor memory runs beside the work on the one before.  What is seldom needed has loops of its own: in
        // one loop with the plain case it made the warps wait for instructions (2048 tokens behind 6144: 1530 us).
        uint32_t va[32], vb[32];
        float top = -INFINITY;
        if (!slow) {
          float top2 = -INFINITY;
          tmem_ld_32x32(s_at, va);
#pragma unroll 1
          for (int x = 0; x < TOK; x += 64) {
            tmem_ld_wait();
            tmem_ld_32x32(s_at + x + 32, vb);
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              top = fmaxf(top, __uint_as_float(va[i]));
              top2 = fmaxf(top2, __uint_as_float(va[i + 1]));
            }
            tmem_ld_wait();
            if (x + 64 < TOK) tmem_ld_32x32(s_at + x + 64, va);
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              top = fmaxf(top, __uint_as_float(vb[i]));
              top2 = fmaxf(top2, __uint_as_float(vb[i + 1]));
            }
          }
          top = fmaxf(top, top2) * f;
        } else {
#pragma unroll 1
          for (int x = 0; x < TOK; x += 32) {
            tmem_ld_32x32(s_at + x, va);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 32; ++i) top = fmaxf(top, score(__uint_as_float(va[i]), x + i));
          }
        }
        float fix = 1.f;
        __syncwarp();
        if (top > m + 3.f) {
          fix = ex2(m - top);
          m = top;
          l *= fix;
        }
        if (e_tile > e_max) {
          fix *= e_tile - e_max > 126 ? 0.f : __uint_as_float((uint32_t)(127 - (e_tile - e_max)) << 23);
          e_max = e_tile;
        }
        if (k > 0 && __any_sync(0xFFFFFFFFu, fix != 1.f)) {
#pragma unroll 1
          for (int x = 0; x < D; x += 16) {
            uint32_t w[16];
            tmem_ld_32x32_x16(o_at + x, w);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) w[i] = __float_as_uint(__uint_as_float(w[i]) * fix);
            tmem_st_32x32_x16(o_at + x, w);
          }
        }
        const int down = e_max - e_tile;                                   // this tile's values are smaller: so are its weights
        const bool faint = down > 40;                                      // too small to matter, but they count in the sum
        const float off = 12.f - m - (faint ? 0.f : (float)down);
        float sum = 0.f, sum2 = 0.f;
        if (!slow) {
          auto weigh = [&](const uint32_t (&v)[32], int x) {
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              const float p = ex2(fmaf(__uint_as_float(v[i]), f, off)), p2 = ex2(fmaf(__uint_as_float(v[i + 1]), f, off));
              sum += p;
              sum2 += p2;
              w[i / 2] = pack_f16(p, p2);
            }
            if (faint) {
#pragma unroll
              for (int i = 0; i < 16; ++i) w[i] = 0;
            }
            tmem_st_32x32_x16(s_at + x / 2, w);
          };
          tmem_ld_32x32(s_at, va);
#pragma unroll 1
          for (int x = 0; x < TOK; x += 64) {
            tmem_ld_wait();
            tmem_ld_32x32(s_at + x + 32, vb);
            weigh(va, x);
            tmem_ld_wait();
            if (x + 64 < TOK) tmem_ld_32x32(s_at + x + 64, va);
            weigh(vb, x + 32);
          }
        } else {
#pragma unroll 1
          for (int x = 0; x < TOK; x += 32) {
            tmem_ld_32x32(s_at + x, va);
            tmem_ld_wait();
            uint32_t w[16];
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
              const float p = ex2(score(__uint_as_float(va[i]), x + i) + off), p2 = ex2(score(__uint_as_float(va[i + 1]), x + i + 1) + off);
              sum += p;
              sum2 += p2;
              w[i / 2] = faint ? 0u : pack_f16(p, p2);
            }
            __syncwarp();
            tmem_st_32x32_x16(s_at + x / 2, w);
          }
        }
        sum += sum2;
        l += sum * (faint ? 1.f : __uint_as_float((uint32_t)(127 + down) << 23));
        tmem_st_wait();
        tc_fence_before_sync();
        mbar_arrive(p_full(t));
      }
      if (!ok) break;
      ok = __all_sync(0xFFFFFFFFu, mbar_wait(o_full(t), o_count & 1, cta_abort, c.err_word, SITE_EPI_ACC_FULL));
      ++o_count;
      if (!ok) break;
      tc_fence_after_sync();
      const float inv = (l > 0.f ? 1.f / l : 0.f) * (FMT == FMT_NVFP4 ? c.v_ts : __uint_as_float((uint32_t)(e_max - 12) << 23));
      const int64_t to = (int64_t)token * heads + h;
#pragma unroll 1
      for (int x = 0; x < D; x += 16) {
        uint32_t w[16];
        tmem_ld_32x32_x16(o_at + x, w);
        tmem_ld_wait();
#pragma unroll
        for (int e = 0; e < 16; e += 8) {
          uint4 y;
#pragma unroll
          for (int i = 0; i < 4; ++i) {                                    // MXINT4: the elements lie in the order of kv_query_order
            constexpr auto column = [](int el) { return FMT == FMT_MXINT4 ? (el < 4 ? 2 * el : 2 * (el - 4) + 1) : el; };
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"((&y.x)[i]) : "f"(__uint_as_float(w[e + column(2 * i + 1)]) * inv),
                "f"(__uint_as_float(w[e + column(2 * i)]) * inv));
          }
          if (there) *reinterpret_cast<uint4*>(out + to * D + x + e) = y;
        }
        __syncwarp();
      }
      if (there && lse) lse[to] = l > 0.f ? (m - 12.f + log2f(l)) * kLn2 : -INFINITY;
      tc_fence_before_sync();
    }
  } else if (warp < 12) {
    // ------------------------------------------------------------------ cached tokens
    // The named barriers are executed by every one of these threads for every tile, also after a wait has given up, so that no warp is left in one.
    const int dt = tid - 256, dw = warp - 8, mask = (1 << c.page_shift) - 1;
    uint32_t fill = 0, tile_no = 0;
    bool ok = true;
    for (long long index = blockIdx.x; kv_prefill_item<C::ROWS, TOK>(c, a, group, index, lane, it); index += gridDim.x) {
      const int32_t* table = c.table + (int64_t)it.b * c.width;
      const uint8_t* head_pages = c.pages + (int64_t)it.head * c.head_bytes;
      auto look_up = [&](int k) {                                          // where the pages of tile k's groups of 16 tokens begin
        if (dt < C::GROUPS) {
          const int j = it.base + k * TOK + 16 * dt;
          int64_t at = -1;
          if (k < it.tiles && j < it.hi) {
            const int p = table[j >> c.page_shift];
            if ((unsigned)p < (unsigned)c.num_pages) at = p * c.page_bytes;
            else kv_bad_page(c);
          }
          page_at[(k & 1) * C::GROUPS + dt] = at;
        }
      };
      auto fetch = [&](int k) {
        if (ok && k < it.tiles) {
          const uint32_t dst = smem + C::RAW_AT + (k & 1) * C::RAW;
          constexpr int PER = TOK * CH / 128;                              // chunks of codes of a thread, of keys and of values
#pragma unroll
          for (int i = 0; i < PER; ++i) {
            const int id = i * 128 + dt, r = id / CH;
            const int64_t at = page_at[(k & 1) * C::GROUPS + r / 16];
            const uint8_t* src = head_pages + (at < 0 ? 0 : at) + ((it.base + k * TOK + r) & mask) * (D / 2) + (id % CH) * 16;
            cp_async_16(dst + id * 16, src, at < 0 ? 0 : 16);
            cp_async_16(dst + C::CODES + id * 16, src + c.v_codes, at < 0 ? 0 : 16);
          }
          constexpr int PIECES = TOK * SB / 16;                            // of scale bytes
#pragma unroll
          for (int i = 0; i < (PIECES + 127) / 128; ++i) {
            const int id = i * 128 + dt;
            if (id < PIECES) {
              const int g16 = id / SB;
              const int64_t at = page_at[(k & 1) * C::GROUPS + g16];
              const uint8_t* src = head_pages + (at < 0 ? 0 : at) + c.k_scales + ((it.base + k * TOK + 16 * g16) & mask) * SB + (id % SB) * 16;
              cp_async_16(dst + 2 * C::CODES + id * 16, src, at < 0 ? 0 : 16);
              cp_async_16(dst + 2 * C::CODES + C::SCALES + id * 16, src + (c.v_scales - c.k_scales), at < 0 ? 0 : 16);
            }
          }
        }
        cp_async_commit();
      };
      named_barrier_sync(1, 128);                                          // the item before has been read
      look_up(0);
      named_barrier_sync(1, 128);
      fetch(0);
      look_up(1);
      for (int k = 0; k < it.tiles; ++k, ++tile_no) {
        cp_async_wait<0>();
        named_barrier_sync(1, 128);                                        // the tile is there, and the next one's pages; the one before has been read
        fetch(k + 1);
        const int j0 = it.base + k * TOK;
        const uint8_t* raw = smem_p + C::RAW_AT + (k & 1) * C::RAW;
        const uint8_t *k_scales = raw + 2 * C::CODES, *v_scales = k_scales + C::SCALES;
        int down[2] = {0, 0};                                              // 27 - E
        if constexpr (FMT != FMT_NVFP4) {
          int top[2] = {27, 27};
          if (dt < TOK && j0 + dt < it.hi) {
#pragma unroll
            for (int i = 0; i < SB; ++i) {
              top[0] = max(top[0], (int)k_scales[dt * SB + i]);
              top[1] = max(top[1], (int)v_scales[dt * SB + i]);
            }
          }
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            top[i] = __reduce_max_sync(0xFFFFFFFFu, top[i]);
            if (lane == 0) warp_top[(k & 1) * 8 + dw * 2 + i] = top[i];
          }
          named_barrier_sync(1, 128);
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int* w = warp_top + (k & 1) * 8 + i;
            const int most = max(max(w[0], w[2]), max(w[4], w[6]));
            down[i] = 27 - most;
            if (dt == 0) tile_top[2 * (tile_no & 3) + i] = most;
          }
        }
        look_up(k + 2);
#pragma unroll 1
        for (int half = 0; half < 2; ++half, ++fill) {                     // keys, values
          if (ok) ok = mbar_wait_warp(kv_empty(fill), ((fill / C::STAGES) & 1) ^ 1, cta_abort, c.err_word, SITE_PRODUCER_EMPTY);
          if (!ok) continue;
          uint8_t* dst = smem_p + C::TILES * C::Q_BYTES + (fill % C::STAGES) * C::KV_BYTES;
          const uint8_t *codes = raw + half * C::CODES, *scales = half ? v_scales : k_scales;
#pragma unroll 2
          for (int i = 0; i < TOK * CH / 128; ++i) {
            const int id = i * 128 + dt, r = id / CH, ch = id % CH;
            const uint4 w = *reinterpret_cast<const uint4*>(codes + id * 16);
            uint32_t f[2];                                                 // of the first and last 16 codes
            if constexpr (FMT == FMT_NVFP4) {
              const uint32_t two = e4m3x2_f16x2(*reinterpret_cast<const uint16_t*>(scales + r * SB + 2 * ch));
              f[0] = __byte_perm(two, 0, 0x1010);
              f[1] = __byte_perm(two, 0, 0x3232);
            } else {
              f[0] = f[1] = (uint32_t)max((int)scales[r * SB + ch] + (half ? down[1] : down[0]), 0) * 0x04000400u;
            }
            if (j0 + r >= it.hi) f[0] = f[1] = 0;                          // what lies there may be no number
            uint8_t* to = dst + (ch >> 1) * (TOK * 128) + r * 128;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              uint32_t o[4];
              kv_key_pairs<FMT>((&w.x)[x], o);
              uint4 y;
#pragma unroll
              for (int e = 0; e < 4; ++e) (&y.x)[e] = mul_f16x2(o[e], f[x >> 1]);
              *reinterpret_cast<uint4*>(to + ((((ch & 1) * 4 + x) ^ (r & 7)) << 4)) = y;
            }
          }
          fence_proxy_async_smem();
          mbar_arrive(kv_full(fill));
        }
      }
      cp_async_wait<0>();
    }
  } else {
    // ------------------------------------------------------------------ products
    constexpr uint32_t idesc_s = idesc_f16(128, TOK, false, false), idesc_o = idesc_f16(128, D, false, true);
    uint32_t fill = 0, p_count[2] = {0, 0}, q_count[2] = {0, 0};
    bool ok = true;
    for (long long index = blockIdx.x; ok && kv_prefill_item<C::ROWS, TOK>(c, a, group, index, lane, it); index += gridDim.x) {
      const int active = it.rows > 128 ? 2 : 1;
      for (int k = 0; k <= it.tiles && ok; ++k) {
        const uint32_t kf = fill + 2 * k, vf = kf - 1;
        if (k > 0) ok = mbar_wait_warp(kv_full(vf), (vf / C::STAGES) & 1, cta_abort, c.err_word, SITE_MMA_FULL);
        if (ok && k < it.tiles) ok = mbar_wait_warp(kv_full(kf), (kf / C::STAGES) & 1, cta_abort, c.err_word, SITE_MMA_FULL);
        for (int t = 0; t < active && ok; ++t) {
          if (k == 0) {
            ok = mbar_wait_warp(q_full(t), q_count[t] & 1, cta_abort, c.err_word, SITE_MMA_ACC_EMPTY);
            ++q_count[t];
          } else {
            ok = mbar_wait_warp(p_full(t), p_count[t] & 1, cta_abort, c.err_word, SITE_MMA_ACC_EMPTY);
            ++p_count[t];
          }
          if (!ok) break;
          tc_fence_after_sync();
          const uint32_t s_at = tmem + t * TOK, o_at = tmem + C::O_COL + t * D;
          if (elect_one()) {
            if (k > 0) {
              const uint64_t v = make_desc(smem + C::TILES * C::Q_BYTES + (vf % C::STAGES) * C::KV_BYTES, TOK * 128, 1024, kSwizzle128);
#pragma unroll
              for (int i = 0; i < TOK / 16; ++i)           // 16 tokens: 8 columns of P, 16 rows of V (2 KiB)
                mma_bf16_tmem_a(o_at, s_at + 8 * i, v + 128 * i, idesc_o, k > 1 || i > 0);
            }
            if (k < it.tiles) {
              const uint64_t q = make_desc(smem + t * C::Q_BYTES, 16, 1024, kSwizzle128);
              const uint64_t x = make_desc(smem + C::TILES * C::Q_BYTES + (kf % C::STAGES) * C::KV_BYTES, 16, 1024, kSwizzle128);
#pragma unroll
              for (int i = 0; i < D / 16; ++i)             // 16 elements: 32 bytes of a row of 128
                mma_bf16(s_at, q + (i >> 2) * (128 * 128 / 16) + 2 * (i & 3), x + (i >> 2) * (TOK * 128 / 16) + 2 * (i & 3), idesc_s, i > 0);
              tc_commit(s_full(t));
            } else {
              tc_commit(o_full(t));
            }
          }
          __syncwarp();
        }
        if (!ok) break;
        if (elect_one()) {
          if (k > 0) tc_commit(kv_empty(vf));
          if (k < it.tiles) tc_commit(kv_empty(kf));
        }
        __syncwarp();
      }
      fill += 2 * it.tiles;
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

}  // namespace torq
