// Attention of the new tokens of every sequence over its cached tokens:
//   x_j = cap(f q k_j) - slope |p - j|,   out = sum_j softmax(x)_j v_j,   lse = log sum_j exp(x_j)
// over the tokens j that a query at place p may see:  p - window < j <= max(p, prefix - 1),  first <= j < length.
// cap(x) = c tanh(x / c).  A query that sees nothing gets zeros and -inf.
#pragma once
#include "kv_cache.cuh"
#include "kv_fragments.cuh"

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


// ---- few queries per sequence -----------------------------------------------------------------------------------------------------------------
// The cache is streamed once, by all SMs alike: the work is a list of units of UNIT cached tokens (sequence after sequence, key/value head after head,
// group of 8 NT rows after group), cut into as many equal ranges as there are CTAs, whatever the lengths are.  Lengths are known on the device
// alone, so every CTA counts the units itself.  An item (sequence, head, group) that lies in one range is finished by its CTA; of one that crosses a
// border each CTA leaves sums, maximum and a partial result, and a second kernel joins them in the order of the ranges.
//
// Inside a CTA each of four warps takes 32 tokens of a unit by itself, through a ring of its own filled by cp.async: no barrier until the item ends.
// A warp keeps a maximum m of its scores in powers of two that is raised only when a score exceeds it by 3, so weights are exp2(x - m + 12) <= 2^15 in
// float16; they keep 11 bits down to 2^-26 of the largest.  The same goes for the values' scales (see kv_fragments.cuh).
template <int FMT_, int D_, int NT_>
struct KvDecodeCfg {
  static constexpr int FMT = FMT_, D = D_, NT = NT_;
  static constexpr int WARPS = 4, THREADS = 32 * WARPS, STEP = 32, UNIT = WARPS * STEP, ROWS = 8 * NT;
  static constexpr int CH = D / 32, SB = D / kv_block(FMT);
  static constexpr int K_BYTES = STEP * D / 2, S_BYTES = STEP * SB, STAGE = 2 * (K_BYTES + S_BYTES);      // keys, values, their scales
  static constexpr int CTAS = D == 256 || NT == 2 ? 2 : 3;                 // per SM
  static constexpr int STAGES = D == 256 ? 3 : (D == 128 ? 4 : 6);
  static constexpr int RING = WARPS * STAGES * STAGE;
  static constexpr int JOIN = WARPS * ROWS * D * 4;                        // the warps' results, in the ring's place
  static constexpr int SMEM = (RING > JOIN ? RING : JOIN) + 1024;
  static constexpr int PARTIAL = ROWS * (D + 2);                           // floats: results, maxima, sums
};
struct KvOwner {                         // written by every CTA: the item that it begins and does not finish
  int32_t rows, first_row, first_token, head;                              // of the group (0: none), its first of its sequence's, of the batch; key/value head
  long long end, units;                                                    // of the item's units, one behind the last; units in all
};

// What one warp's rows are, for its columns 2t and 2t + 1 of each group of eight.
struct KvItem {
  int b, head, first_token, count, length, first_row, rows;                // of the sequence; of the group: its first row among count * group, how many
  int lo, base, hi;                                                        // cached tokens [lo, hi) that any row of the sequence sees; base = lo / 32 * 32
};

__device__ __forceinline__ long long kv_range_begin(long long units, int cta, int ctas) { return units * cta / ctas; }

// Of sequence b: groups of ROWS rows, units per group and head.
template <int ROWS, int UNIT>
__device__ __forceinline__ void kv_sequence_units(const KvView& c, const KvScoring& a, int b, int group, KvItem& it, int& groups, int& units) {
  it.b = b;
  kv_new_tokens(c, b, it.first_token, it.count);
  it.length = kv_length(c, b);
  groups = (it.count * group + ROWS - 1) / ROWS;
  const int p0 = it.length - it.count;
  int lo = 0, hi = it.length;
  if (a.window > 0 && p0 - a.window + 1 > 0) lo = p0 - a.window + 1;
  it.lo = lo;
  it.base = lo & ~31;
  it.hi = hi;
  units = hi > it.base ? (hi - it.base + UNIT - 1) / UNIT : 1;             // rows that see nothing are an item all the same
}

template <class C>
__global__ void __launch_bounds__(C::THREADS, C::CTAS) kv_decode_kernel(const KvView c, const KvScoring a, const __nv_bfloat16* Q, int64_t q_stride, int heads,
                                                                        __nv_bfloat16* out, float* lse, KvOwner* owners, float* partials) {
  constexpr int FMT = C::FMT, D = C::D, NT = C::NT, CH = C::CH, SB = C::SB, ROWS = C::ROWS;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ long long scan[C::WARPS + 1];
  __shared__ float row_m[C::WARPS][ROWS], row_l[C::WARPS][ROWS];
  griddep_wait_and_launch();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3, group = heads / c.heads;
  const int cta = blockIdx.x, ctas = gridDim.x;

  // rows of the batch that no sequence has
  if (c.starts) {
    const int before = min(max(c.starts[0], 0), c.tokens), behind = min(max(c.starts[c.batch], before), c.tokens), none = before + c.tokens - behind;
    for (int i = cta; i < none; i += ctas) {
      const int64_t row = (int64_t)(i < before ? i : behind + i - before) * heads;
      for (int e = tid; e < heads * D / 8; e += C::THREADS) reinterpret_cast<uint4*>(out + row * D)[e] = make_uint4(0, 0, 0, 0);
      if (lse)
        for (int e = tid; e < heads; e += C::THREADS) lse[row + e] = -INFINITY;
    }
  }

  // units in all, then where this CTA's range begins
  KvItem it;
  int groups, per;
  auto units_of = [&](int b) -> long long {
    if (b >= c.batch) return 0;
    kv_sequence_units<ROWS, C::UNIT>(c, a, b, group, it, groups, per);
    return (long long)groups * c.heads * per;
  };
  auto block_scan = [&](long long v, long long& total) {                   // exclusive
    long long s = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long x = __shfl_up_sync(0xFFFFFFFFu, s, o);
      if (lane >= o) s += x;
    }
    __syncthreads();
    if (lane == 31) scan[warp] = s;
    __syncthreads();
    long long before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < C::WARPS; ++w) {
      if (w < warp) before += scan[w];
      total += scan[w];
    }
    return before + s - v;
  };
  long long units = 0, total;
  __shared__ long long found[2];
  const long long mine = units_of(tid), mine_before = block_scan(mine, units);
  for (int b = C::THREADS; b < c.batch; b += C::THREADS) {
    block_scan(units_of(b + tid), total);
    units += total;
  }
  const long long begin = kv_range_begin(units, cta, ctas), end = kv_range_begin(units, cta + 1, ctas);
  if (tid == 0) owners[cta].rows = 0;
  if (begin >= end) return;
  {
    long long before = mine_before, v = mine, base = 0;
    for (int b = 0;; b += C::THREADS) {                                    // ends: begin < units
      if (b) {
        v = units_of(b + tid);
        before = base + block_scan(v, total);
      } else {
        total = 0;
        for (int w = 0; w < C::WARPS; ++w) total += scan[w];
        if (c.batch > C::THREADS) block_scan(mine, total);                 // `scan` has been overwritten
      }
      if (before <= begin && begin < before + v) {
        found[0] = b + tid;
        found[1] = before;
      }
      base += total;
      if (begin < base) break;
    }
    __syncthreads();
  }
  int b = (int)found[0];
  long long at = begin, sequence_begin = found[1], sequence_units = units_of(b);

  const uint32_t ring = smem_u32(smem) + warp * C::STAGES * C::STAGE;
  uint8_t* ring_p = smem + warp * C::STAGES * C::STAGE;
  const int row_of = lane & 15, chunk_of = lane >> 4;

  while (at < end) {
    while (at >= sequence_begin + sequence_units) {                        // sequences without rows have no units
      sequence_begin += sequence_units;
      sequence_units = units_of(++b);
    }
    const int local = (int)((at - sequence_begin) / per), unit0 = (int)((at - sequence_begin) % per);   // (head, group) of the sequence; its unit
    const long long left = end - at;
    const int unit1 = (int)(left < per - unit0 ? unit0 + left : per);
    it.head = local / groups;
    it.first_row = local % groups * ROWS;
    it.rows = min(ROWS, it.count * group - it.first_row);
    at += unit1 - unit0;

    // the queries, and what each row sees
    KvQuery<D> q[NT];
    float factor[NT][2], slope[NT][2], m[NT][2], l[NT][2];
    int place[NT][2], lo[NT][2], hi[NT][2], all_lo = 0, all_hi = INT32_MAX;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int r = it.first_row + 8 * n + g;
      const int i = it.first_token + r / group, h = it.head * group + r % group;
      const float back = kv_load_query<FMT, D>(8 * n + g < it.rows ? Q + i * q_stride + h * D : nullptr, t, q[n]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int col = 8 * n + 2 * t + e, rr = it.first_row + col;
        factor[n][e] = __shfl_sync(0xFFFFFFFFu, back, 8 * t + 4 * e) * (a.scale * (FMT == FMT_NVFP4 ? c.k_ts : 1.f) * kLog2e);
        lo[n][e] = hi[n][e] = place[n][e] = 0;
        slope[n][e] = 0.f;
        if (col < it.rows) {
          const int token = rr / group;
          place[n][e] = it.length - it.count + token;
          kv_range(a, it.b, it.first_token + token, place[n][e], it.length, lo[n][e], hi[n][e]);
          if (a.slopes) slope[n][e] = a.slopes[it.head * group + rr % group];
          all_lo = max(all_lo, lo[n][e]);
          all_hi = min(all_hi, hi[n][e]);
        }
        m[n][e] = -1e30f;
        l[n][e] = 0.f;
      }
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
      all_lo = max(all_lo, __shfl_xor_sync(0xFFFFFFFFu, all_lo, o));
      all_hi = min(all_hi, __shfl_xor_sync(0xFFFFFFFFu, all_hi, o));
    }
    const bool special = a.softcap > 0.f || a.slopes;
    float o[NT][CH][2][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int i = 0; i < CH * 8; ++i) o[n][i / 8][i / 4 % 2][i % 4] = 0.f;
    int top_scale[CH];                                                     // MXFP4, MXINT4: E of each chunk
    uint32_t top_pair[CH / 2], shift[CH];                                  // the same, chunks i and i + 2 (bytes apart) in halves; 27 - E twice
#pragma unroll
    for (int i = 0; i < CH; ++i) {
      top_scale[i] = 27;
      shift[i] = 0;
      top_pair[i / 2] = 0x001B001Bu;
    }

    const int steps = unit1 - unit0, first = it.base + unit0 * C::UNIT + warp * C::STEP;
    const int32_t* table = c.table + (int64_t)b * c.width;
    int page[2];
    auto look_up = [&](int k) {                                            // pages of step k's two groups of 16 tokens; -1: nothing there
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int j = first + k * C::UNIT + 16 * i;
        page[i] = -1;
        if (k < steps && j < it.hi && j + 16 > it.lo) {
          page[i] = table[j >> c.page_shift];
          if ((unsigned)page[i] >= (unsigned)c.num_pages) {
            kv_bad_page(c);
            page[i] = -1;
          }
        }
      }
    };
    auto fetch = [&](int k) {
      const int j0 = first + k * C::UNIT, mask = (1 << c.page_shift) - 1;
      const uint32_t dst = ring + (k % C::STAGES) * C::STAGE;
      if (k < steps) {
#pragma unroll
        for (int i = 0; i < 2 * CH; ++i) {                                 // chunks of keys, then of values
          const int id = i % CH * 32 + lane, row = id / CH, chunk = id % CH, p = page[row >> 4];
          const uint8_t* src = kv_head_page(c, p < 0 ? 0 : p, it.head) + (i < CH ? 0 : c.v_codes) + ((j0 + row) & mask) * (D / 2) + chunk * 16;
          cp_async_16(dst + (i < CH ? 0 : C::K_BYTES) + 16 * kv_swizzled<D>(row, chunk), src, p < 0 ? 0 : 16);
        }
        constexpr int PIECES = C::S_BYTES / 16;                            // of the keys' scales, and of the values'
#pragma unroll
        for (int i = 0; i < (2 * PIECES + 31) / 32; ++i) {
          const int id = i * 32 + lane, piece = id % PIECES;
          if (id < 2 * PIECES) {
            const int row = piece * 16 / SB, p = page[row >> 4];
            const uint8_t* src = kv_head_page(c, p < 0 ? 0 : p, it.head) + (id < PIECES ? c.k_scales : c.v_scales) + ((j0 + row) & mask) * SB +
                                 (piece * 16 - row * SB);
            cp_async_16(dst + 2 * C::K_BYTES + id * 16, src, p < 0 ? 0 : 16);
          }
        }
      }
      cp_async_commit();
    };
    look_up(0);
#pragma unroll
    for (int k = 0; k < C::STAGES - 1; ++k) {
      fetch(k);
      look_up(k + 1);
    }

    for (int k = 0; k < steps; ++k) {
      cp_async_wait<C::STAGES - 2>();
      __syncwarp();
      fetch(k + C::STAGES - 1);                                            // into the stage that the last step has left
      look_up(k + C::STAGES);
      const int j0 = first + k * C::UNIT;
      if (j0 >= it.hi) continue;
      const uint32_t stage = ring + (k % C::STAGES) * C::STAGE;
      uint8_t* stage_p = ring_p + (k % C::STAGES) * C::STAGE;
      uint8_t* v_scales = stage_p + 2 * C::K_BYTES + C::S_BYTES;
      const bool border = j0 < all_lo || j0 + C::STEP > all_hi;
      if (border && (j0 + lane >= it.hi || j0 + lane < it.base)) {         // what lies there may be no numbers
#pragma unroll
        for (int i = 0; i < SB; i += 2) *reinterpret_cast<uint16_t*>(v_scales + lane * SB + i) = 0;
      }
      if (border) __syncwarp();

      // scores, weights
      uint32_t p[NT][2][2];
      float s[2][NT][4];
#pragma unroll
      for (int u = 0; u < 2; ++u) kv_tile_scores<FMT, D, NT>(stage, stage_p + 2 * C::K_BYTES, 16 * u, lane, q, s[u]);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float f[2] = {factor[n][0], factor[n][1]};
        if (special || border) {
#pragma unroll
          for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int e = i & 1, j = j0 + 16 * u + g + 8 * (i >> 1);
              float x = s[u][n][i] * factor[n][e];
              if (special) x = kv_score(x * kLn2, a.softcap, slope[n][e], abs(place[n][e] - j));
              s[u][n][i] = j >= lo[n][e] && j < hi[n][e] ? x : -INFINITY;
            }
          f[0] = f[1] = 1.f;
        }
        bool raise = false;
        float most[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          most[e] = fmaxf(fmaxf(s[0][n][e], s[0][n][e + 2]), fmaxf(s[1][n][e], s[1][n][e + 2])) * f[e];
          raise |= most[e] > m[n][e] + 3.f;
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
        }
        const float off[2] = {12.f - m[n][0], 12.f - m[n][1]};
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
      if constexpr (FMT != FMT_NVFP4) {
        uint32_t w[(SB + 3) / 4], pair[CH / 2];
        kv_scale_words<SB>(v_scales + lane * SB, w);                       // a token's each
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
            shift[i] = (uint32_t)(27 - top) & 0xFFFFu;
            shift[i] |= shift[i] << 16;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int x = 0; x < 8; ++x) o[n][i][x / 4][x % 4] *= old;
          }
        }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        uint32_t w[4][(SB + 3) / 4];                                       // scales of tokens 2t, 2t + 1, 2t + 8, 2t + 9
#pragma unroll
        for (int i = 0; i < 4; ++i) kv_scale_words<SB>(v_scales + (16 * u + 2 * t + (i & 1) + 8 * (i >> 1)) * SB, w[i]);
#pragma unroll
        for (int c2 = 0; c2 < CH; c2 += 2) {
          uint32_t raw[4];
          ldmatrix_x4_t(stage + C::K_BYTES + 16 * kv_swizzled<D>(16 * u + row_of, c2 + chunk_of), raw);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int ch = c2 + e;
            uint32_t v[2][4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              uint32_t f;
              if constexpr (FMT == FMT_NVFP4) {
                const uint32_t at_byte = 2 * (ch & 1) + (g >> 2);
                f = e4m3x2_f16x2(__byte_perm(w[2 * i][ch / 2], w[2 * i + 1][ch / 2], at_byte | (at_byte + 4) << 4));
              } else {
                const uint32_t x = __byte_perm(w[2 * i][ch / 4], w[2 * i + 1][ch / 4], (ch % 4) | (ch % 4 + 4) << 8) & 0x00FF00FFu;
                f = __viaddmax_s16x2_relu(x, shift[ch], 0u) << 10;
              }
              kv_value_pairs<FMT>(raw[2 * e + i], v[i]);
#pragma unroll
              for (int x = 0; x < 4; ++x) v[i][x] = mul_f16x2(v[i][x], f);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              mma_f16(o[n][ch][0], v[0][0], v[0][1], v[1][0], v[1][1], p[n][u][0], p[n][u][1], o[n][ch][0]);
              mma_f16(o[n][ch][1], v[0][2], v[0][3], v[1][2], v[1][3], p[n][u][0], p[n][u][1], o[n][ch][1]);
            }
          }
        }
      }
    }
    cp_async_wait<0>();

    // the warps' results together
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l[n][e] += __shfl_xor_sync(0xFFFFFFFFu, l[n][e], x);
        if (g == 0) {
          row_m[warp][8 * n + 2 * t + e] = m[n][e];
          row_l[warp][8 * n + 2 * t + e] = l[n][e];
        }
      }
    __syncthreads();                                                       // and the ring is free
    float* join = reinterpret_cast<float*>(smem);
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = 8 * n + 2 * t + e;
        float top = row_m[0][r];
#pragma unroll
        for (int w = 1; w < C::WARPS; ++w) top = fmaxf(top, row_m[w][r]);
        const float f = ex2(m[n][e] - top);
#pragma unroll
        for (int ch = 0; ch < CH; ++ch) {
          const float fs = FMT == FMT_NVFP4 ? f * c.v_ts : f * __uint_as_float((uint32_t)(top_scale[ch] - 12) << 23);
          *reinterpret_cast<float4*>(join + (warp * ROWS + r) * D + 32 * ch + 4 * g) =
              make_float4(o[n][ch][0][e] * fs, o[n][ch][0][e + 2] * fs, o[n][ch][1][e] * fs, o[n][ch][1][e + 2] * fs);
        }
      }
    __syncthreads();
    const bool begins = unit0 == 0, whole = begins && unit1 == per;
    float* part = partials + (int64_t)(2 * cta + (begins ? 1 : 0)) * C::PARTIAL;
    for (int i = tid; i < ROWS * D / 4; i += C::THREADS) {
      const int r = i / (D / 4), d = i % (D / 4) * 4;
      float4 v = make_float4(0, 0, 0, 0);
      float top = row_m[0][r], sum = 0.f;
#pragma unroll
      for (int w = 1; w < C::WARPS; ++w) top = fmaxf(top, row_m[w][r]);
#pragma unroll
      for (int w = 0; w < C::WARPS; ++w) {
        const float4 x = *reinterpret_cast<const float4*>(join + (w * ROWS + r) * D + d);
        v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
        sum += row_l[w][r] * ex2(row_m[w][r] - top);
      }
      if (whole) {
        if (r < it.rows) {
          const float inv = sum > 0.f ? 1.f / sum : 0.f;
          const int rr = it.first_row + r;
          const int64_t row = (int64_t)(it.first_token + rr / group) * heads + it.head * group + rr % group;
          uint2 y;
          asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y.x) : "f"(v.y * inv), "f"(v.x * inv));
          asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y.y) : "f"(v.w * inv), "f"(v.z * inv));
          *reinterpret_cast<uint2*>(out + row * D + d) = y;
          if (lse && d == 0) lse[row] = sum > 0.f ? (top - 12.f + log2f(sum)) * kLn2 : -INFINITY;
        }
      } else {
        *reinterpret_cast<float4*>(part + r * D + d) = v;
        if (d == 0) {
          part[ROWS * D + r] = top;
          part[ROWS * D + ROWS + r] = sum;
        }
      }
    }
    if (begins && !whole && tid == 0) {
      KvOwner w;
      w.rows = it.rows;
      w.first_row = it.first_row;
      w.first_token = it.first_token;
      w.head = it.head;
      w.end = sequence_begin + (long long)local * per + per;
      w.units = units;
      owners[cta] = w;
    }
    __syncthreads();                                                       // before the ring is filled again
  }
}

// The CTA of an item's first range joins the ranges' results; SPLIT warps to a row, each with its share of the ranges.
template <int D, int NT>
struct KvJoinCfg {
  static constexpr int ROWS = 8 * NT, SPLIT = NT == 1 ? 4 : 2, THREADS = 32 * ROWS * SPLIT, EACH = D / 32;       // elements per lane
  static constexpr int PARTIAL = ROWS * (D + 2);
};
template <int D, int NT>
__global__ void __launch_bounds__(KvJoinCfg<D, NT>::THREADS) kv_join_kernel(int ctas, int heads, int group, const KvOwner* owners, const float* partials,
                                                                         __nv_bfloat16* out, float* lse) {
  using J = KvJoinCfg<D, NT>;
  constexpr int ROWS = J::ROWS;
  __shared__ float parts[J::SPLIT][ROWS][D + 2];
  griddep_wait_and_launch();
  const int cta = blockIdx.x, lane = threadIdx.x & 31, r = (threadIdx.x >> 5) / J::SPLIT, which = (threadIdx.x >> 5) % J::SPLIT;
  const KvOwner w = owners[cta];
  if (w.rows == 0) return;
  int last = cta;                        // the CTA of unit end - 1: the last whose range begins before `end`
  {
    long long x = (w.end * ctas - 1) / w.units;                            // about there
    if (x > ctas - 1) x = ctas - 1;
    while (kv_range_begin(w.units, (int)x, ctas) >= w.end) --x;
    while (x + 1 < ctas && kv_range_begin(w.units, (int)x + 1, ctas) < w.end) ++x;
    last = (int)x;
  }
  float m = -1e30f, l = 0.f, o[J::EACH] = {};
  auto part_of = [&](int i) { return partials + (int64_t)(2 * i + (i == cta ? 1 : 0)) * J::PARTIAL; };
  constexpr int BATCH = 4;
  for (int i = cta + which; i <= last; i += J::SPLIT * BATCH) {
    float pm[BATCH], pl[BATCH], v[BATCH][J::EACH];
#pragma unroll
    for (int x = 0; x < BATCH; ++x) {
      const int at = i + x * J::SPLIT;
      pm[x] = -1e30f;
      pl[x] = 0.f;
#pragma unroll
      for (int e = 0; e < J::EACH; ++e) v[x][e] = 0.f;
      if (at <= last && kv_range_begin(w.units, at, ctas) < kv_range_begin(w.units, at + 1, ctas)) {       // CTAs without units left nothing
        const float* p = part_of(at);
        pm[x] = p[ROWS * D + r];
        pl[x] = p[ROWS * D + ROWS + r];
#pragma unroll
        for (int e = 0; e < J::EACH; ++e) v[x][e] = p[r * D + e * 32 + lane];
      }
    }
    float top = m;
#pragma unroll
    for (int x = 0; x < BATCH; ++x) top = fmaxf(top, pm[x]);
    const float old = ex2(m - top);
    l *= old;
#pragma unroll
    for (int e = 0; e < J::EACH; ++e) o[e] *= old;
#pragma unroll
    for (int x = 0; x < BATCH; ++x) {
      const float f = ex2(pm[x] - top);
      l += pl[x] * f;
#pragma unroll
      for (int e = 0; e < J::EACH; ++e) o[e] += v[x][e] * f;
    }
    m = top;
  }
#pragma unroll
  for (int e = 0; e < J::EACH; ++e) parts[which][r][e * 32 + lane] = o[e];
  if (lane == 0) {
    parts[which][r][D] = m;
    parts[which][r][D + 1] = l;
  }
  __syncthreads();
  if (which || r >= w.rows) return;
  float top = m;
#pragma unroll
  for (int x = 1; x < J::SPLIT; ++x) top = fmaxf(top, parts[x][r][D]);
  l = 0.f;
#pragma unroll
  for (int e = 0; e < J::EACH; ++e) o[e] = 0.f;
#pragma unroll
  for (int x = 0; x < J::SPLIT; ++x) {
    const float f = ex2(parts[x][r][D] - top);
    l += parts[x][r][D + 1] * f;
#pragma unroll
    for (int e = 0; e < J::EACH; ++e) o[e] += parts[x][r][e * 32 + lane] * f;
  }
  const int rr = w.first_row + r;
  const int64_t row = (int64_t)(w.first_token + rr / group) * heads + w.head * group + rr % group;
  const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
  for (int e = 0; e < J::EACH; ++e) out[row * D + e * 32 + lane] = __float2bfloat16(o[e] * inv);
  if (lse && lane == 0) lse[row] = l > 0.f ? (top - 12.f + log2f(l)) * kLn2 : -INFINITY;
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
