// Products of a few tokens with 4-bit weights, the activations in bfloat16 (not quantized):
//   y[m, n] = alpha sum_k x[m, k] w^[n, k],   w^ = code * block scale
// and the gated pair of projections, both stacked in one weight matrix [2 N, K]:
//   y[m, n] = silu(g) u,  g / u = the product with row n / N + n.
// Streaming the weights from HBM once is the work (K / 2 bytes and K / 32 or K / 16 scale bytes per row).  They go to the block-scaled
// FP4 instruction as they are: widened to float16 in registers for warp-level instructions, they took 146 instructions per
// 16 x 128 weights and the kernel was bound by those (1 x 5120 -> 5120 7.0 us, now 5.1; 16 tokens 11.5, now 7.0; 32 x 5120 -> 51200 107, 42 in this kernel).
//
// What the instruction cannot take is a bfloat16 activation, so x is written as a sum of numbers that it can.  Per block of 32 (NVFP4: 16)
// with largest magnitude in [2^E, 2^(E+1)), v = rint(x 2^(21-E)) is an integer of at most 22 bits and a sign; in base 8 with digits
// -4 ... 3,
//   v = sum_t d_t 8^(7-t), t = 0 ... 7,   x = sum_t d_t 2^(E-3t),
// every digit is an e2m1 number and 2^(E-3t) a block scale: a token becomes eight rows of an MXFP4 operand, whose products with a
// feature add up to the token's.  bfloat16's 8 bits are kept exactly down to 2^-14 of the block's largest magnitude, and nothing is off by more than
// 2^-22 of it: half a unit of the sum that a float32 accumulator would make of the block, if the large element enters it.  Where its weight is
// zero the sum is small and the error is not (beside an element of 2^16 up to 2^-6).  (NVFP4 scales reach from 2^-9 to 2^8: the scale
// of a block is taken relative to the token's largest one in this CTA's range of K, 2^(E-R+8), not below 2^(R-17), and the powers 8^-t
// and 2^(R-8) are multiplied in when the eight sums are added.)
// The digits cost some 200 instructions per eight elements of x.  Up to FEW_TOK tokens every CTA writes those of its own range of K, once
// per 128 features, which saves a launch; more tokens have them written once, by a kernel of its own, into the caller's workspace.
// From 17 tokens on (gated: 9) the GEMM on CTA pairs may take the digits instead, where it has enough tiles for them.
//
// MXINT4: a two's-complement nibble n is no e2m1 number, but n = 2 (l + 4 h) with l the e2m1 value of the code n & 3 (0, 1/2, 1, 3/2) and h that of
// its upper half (0, 4, -8, -4 over 8: codes 0, 1, 10, 9): two operands from one, six logical instructions per eight weights, in shared
// memory.  Both are multiplied with the same digits, h with scales two powers higher, into one accumulator.
//
// Swapped operands as in the few-token GEMM: the instruction's 128 rows are features, its columns the rows of digits.  A CTA has 128
// features (gated: the 128 gates and the 128 ups of the same features, two accumulators) and a range of K; a CLUSTER of S CTAs shares the
// features.  Roles: warp 0 fetches W and its scales, warp 1 issues the instructions, warps 2..5 write the digits of every stage (a token
// each, other ones at the next stage, so that few tokens still keep all four busy) and add up and store at the end.  The partial sums
// go from registers to the CTA that owns a quarter of the features and 4 tokens (gated: 2), which adds them in the order of their ranks.
#pragma once
#include <cuda_bf16.h>
#include "activation.cuh"
#include "sm100_ptx.cuh"

namespace torq {

// Where the rows of the second operand come from: digits that warps 2..5 write; digits that were written before, into a workspace; or
// no digits, the caller's quantized activations, a row per token (the gated GEMM of few tokens).
enum : int { ROWS_HERE = 0, ROWS_AHEAD = 1, ROWS_QUANTIZED = 2 };

template <int FMT, bool GATED, int ROWS = ROWS_HERE>
struct DigitsCfg {
  // MXINT4: two operands from one in front of digits; beside quantized activations operand bytes, a byte per element (kind::mxf8f6f4)
  static constexpr bool BYTES = FMT == FMT_MXINT4 && ROWS == ROWS_QUANTIZED, PLANES = FMT == FMT_MXINT4 && !BYTES;
  static constexpr int BF = 128;                       // features per tile
  static constexpr int BK = BYTES ? 128 : 256;         // elements of K per stage (128 bytes per row)
  static constexpr int DIGITS = ROWS == ROWS_QUANTIZED ? 1 : 8;   // rows per token
  // tokens of a CTA (quantized: as many as two CTAs have room on an SM for, with their partial sums; gated MXINT4: one CTA has an SM's tensor
  // memory to itself: 4096 -> 14336 45.9 us for 16 tokens in two groups of 8, 28.8 in one)
  static constexpr int MAX_TOK = ROWS == ROWS_QUANTIZED ? (FMT == FMT_NVFP4 ? 24 : 32) : (GATED && !PLANES ? 8 : 16);
  static constexpr int FEW_TOK = 4;                    // up to here the product's CTAs may write the digits themselves
  static constexpr int PER_UNIT = GATED ? 2 : 4;       // tokens of what an epilogue warp adds up at a time
  static constexpr int TILES = GATED ? 2 : 1;          // of W per stage
  static constexpr int TILE_BYTES = (PLANES ? 2 : 1) * BF * 128;
  static constexpr int W_BYTES = TILES * TILE_BYTES;
  static constexpr int CH = FMT == FMT_NVFP4 ? 4 : (BYTES ? 1 : 2);   // scale chunks per stage and 128 rows
  static constexpr int SF_BYTES = CH * 512;
  static constexpr int SF_SETS = TILES + (PLANES ? 2 : 1);   // of W's tiles and of the digits
  static constexpr int MAX_STAGES = 4;
  static constexpr int CTAS_PER_SM = PLANES && GATED ? 1 : 2;
  static constexpr int MAX_SMEM = CTAS_PER_SM == 2 ? 113 * 1024 : 232448;
  static constexpr int THREADS = 192;
  static constexpr int MAX_CLUSTER = 8;
  static constexpr int BAR_BYTES = 256;
  static constexpr int PART_BYTES = 32 * 16;           // a unit's partial sums from one CTA: 16 bytes per feature
  __host__ __device__ static constexpr int rows(int tokens) { return (DIGITS * tokens + 15) / 16 * 16; }
  __host__ __device__ static constexpr int stage_bytes(int r) { return (W_BYTES + r * 128 + SF_SETS * SF_BYTES + 1023) / 1024 * 1024; }
  __host__ __device__ static constexpr int units(int tokens) { return 4 * ((tokens + PER_UNIT - 1) / PER_UNIT); }
  __host__ __device__ static constexpr int push_bytes(int tokens, int S) { return S > 1 ? (units(tokens) + S - 1) / S * S * PART_BYTES : 0; }
  __host__ __device__ static constexpr int smem_bytes(int tokens, int stages, int S) {
    return 1024 + stages * stage_bytes(rows(tokens)) + push_bytes(tokens, S) + BAR_BYTES;
  }
  // accumulators, then the scale chunks of W and of the digits (4 columns each)
  __host__ __device__ static constexpr int tmem_cols(int r) {
    const int n = TILES * r + SF_SETS * 4 * CH;
    return n <= 32 ? 32 : (n <= 64 ? 64 : (n <= 128 ? 128 : (n <= 256 ? 256 : 512)));
  }
  static_assert(TILES * rows(MAX_TOK) + SF_SETS * 4 * CH <= 512 / CTAS_PER_SM, "the CTAs of an SM share its tensor memory");
  static_assert(smem_bytes(MAX_TOK, 2, 1) <= MAX_SMEM, "two stages at least");
};

// u_j = v_j + 44444444 (octal) in 24 bits: field t is d_t + 4.  Eight numbers -> eight words, word t the e2m1 codes of the digits t.
__device__ __forceinline__ void digit_words(const uint32_t (&u)[8], uint32_t (&word)[8]) {
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    uint32_t even = 0, odd = 0;                          // fields of elements 0, 2, 4, 6 and 1, 3, 5, 7, a nibble each
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int from = 21 - 3 * t, to = 4 * (j >> 1);
      const uint32_t f = (from >= to ? u[j] >> (from - to) : u[j] << (to - from)) & (7u << to);
      if (j & 1) odd |= f;
      else even |= f;
    }
    // e2m1 codes of -4 ... 3: 14 13 12 10 0 2 4 5
    word[t] = __byte_perm(0x0A0C0D0Eu, 0x05040200u, even) | __byte_perm(0xA0C0D0E0u, 0x50402000u, odd);
  }
}

// The largest of eight magnitudes, as bits of bfloat16 (what is not a number is larger than all others).
__device__ __forceinline__ uint32_t largest8(const uint4& x) {
  const uint32_t a = __vmaxu2(__vmaxu2(x.x & 0x7FFF7FFFu, x.y & 0x7FFF7FFFu), __vmaxu2(x.z & 0x7FFF7FFFu, x.w & 0x7FFF7FFFu));
  return max(a & 0xFFFFu, a >> 16);
}
constexpr uint32_t kLeastExponent = 21;                  // field of the smallest E: 2^(E - 21) is the smallest E8M0 scale
constexpr uint32_t kScaleBinades = 17;                   // NVFP4: from the largest scale down to 2^-9

// The digits of 256 elements of K of a token, eight per lane (x): word[t] has the eight codes of digit t.  Returns the scale bytes of the
// four blocks that this lane's chunk of scales has (32 lanes share two chunks, NVFP4: four), of digit 0.  `ref`, NVFP4: the exponent field
// that block scales are relative to.  A whole warp calls this.
template <int FMT>
__device__ __forceinline__ uint32_t digits_of_256(const uint4& x, uint32_t ref, int lane, uint32_t (&word)[8]) {
  // exponent field of the block's largest magnitude: of 32 elements in four lanes, or of 16 in two
  uint32_t ef = largest8(x);
  ef = max(ef, __shfl_xor_sync(0xFFFFFFFFu, ef, 1));
  if constexpr (FMT != FMT_NVFP4) ef = max(ef, __shfl_xor_sync(0xFFFFFFFFu, ef, 2));
  ef >>= 7;
  uint32_t four;                                         // this lane's block's scale byte, then those of the chunk
  if constexpr (FMT == FMT_NVFP4) {
    ef = max(ef, ref - kScaleBinades);
    const int q = (int)ef - (int)ref + 8;                // -9 ... 8
    four = (q >= -6 ? (uint32_t)(q + 7) << 3 : 1u << (q + 9)) << (8 * ((lane >> 1) & 3));
    four |= __shfl_xor_sync(0xFFFFFFFFu, four, 2);
    four |= __shfl_xor_sync(0xFFFFFFFFu, four, 4);
  } else {
    ef = max(ef, kLeastExponent);
    four = ef << (8 * ((lane >> 2) & 3));                // 255 where something is not a number: so is the scale, and the sum
    four |= __shfl_xor_sync(0xFFFFFFFFu, four, 4);
    four |= __shfl_xor_sync(0xFFFFFFFFu, four, 8);
  }
  const float f = __uint_as_float((275u - ef) << 23);    // 2^(21 - E)
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
  uint32_t u[8];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    // 1.5 2^23 + x 2^(21-E): rounded to an integer by the addition, the bits of 1.5 2^23 + v
    constexpr uint32_t bias = 044444444u - 0x4B400000u;
    u[2 * i] = __float_as_uint(fmaf(__uint_as_float(w[i] << 16), f, 12582912.f)) + bias;
    u[2 * i + 1] = __float_as_uint(fmaf(__uint_as_float(w[i] & 0xFFFF0000u), f, 12582912.f)) + bias;
  }
  digit_words(u, word);
  return four;
}
// Where this lane stores the word of scale bytes it has of its chunk, if it does: lane t of those that share a chunk has row t of the
// token's eight.  `token`: in its 128-row scale tile.
template <int FMT>
__device__ __forceinline__ bool digit_scales(uint32_t four, int token, int lane, uint32_t& word, uint32_t& chunk, uint32_t& offset) {
  constexpr int LANES = FMT == FMT_NVFP4 ? 8 : 16;       // that share a chunk
  const int t = lane & 7;
  chunk = lane / LANES;
  offset = ((token & 3) * 8 + t) * 16 + (token >> 2) * 4;
  word = FMT == FMT_NVFP4 ? four : four - 0x03030303u * t;   // E8M0: 2^(E - 3t); every byte is 21 at least
  return LANES == 8 || (lane & 8) == 0;
}

// The digits of all tokens, ahead of the product: codes [8 M, K / 2], scales tiled, and for NVFP4 the exponent field of each token's
// largest magnitude.  grid = M ceil(K / 2048): a warp has 256 elements of a token.
template <int FMT>
__global__ void __launch_bounds__(256)
matvec_split_kernel(const __nv_bfloat16* __restrict__ X, int K, uint8_t* __restrict__ codes, uint8_t* __restrict__ scales,
                    uint32_t* __restrict__ exponents) {
  __shared__ uint32_t top_of[8];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int parts = (K + 2047) / 2048;
  const int64_t m = blockIdx.x / parts;
  const int k0 = (int)(blockIdx.x % parts) * 2048 + warp * 256, k = k0 + 8 * lane;
  const uint4* row = reinterpret_cast<const uint4*>(X + m * K);
  // Into the L2 ahead of the product's W, which would stand before it in memory's queue.  Only that: the kernel before may still be writing x.
  if (k < K) asm volatile("prefetch.global.L2 [%0];" ::"l"(row + k / 8));
  griddep_launch_and_wait();
  uint32_t ref = 0;
  uint4 own = make_uint4(0, 0, 0, 0);
  if constexpr (FMT == FMT_NVFP4) {
    uint32_t top = 0;
    for (int p0 = 0; p0 < K / 8; p0 += 8 * 256) {        // eight loads under way: each takes microseconds behind the next kernel's W
      uint4 x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (p0 + 256 * j < K / 8) x[j] = load_once(row + min(p0 + 256 * j + (int)threadIdx.x, K / 8 - 1));
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (p0 + 256 * j < K / 8) {
          top = max(top, largest8(x[j]));
          if (p0 / 256 + j == (int)(blockIdx.x % parts)) own = x[j];   // piece k / 8
        }
    }
    top = __reduce_max_sync(0xFFFFFFFFu, top);
    if (lane == 0) top_of[warp] = top;
    __syncthreads();
    for (int i = 0; i < 8; ++i) top = max(top, top_of[i]);
    ref = max(top >> 7, kLeastExponent + kScaleBinades);
    if (blockIdx.x % parts == 0 && threadIdx.x == 0) exponents[m] = ref;
  } else if (k < K) {
    own = load_once(row + k / 8);
  }
  if (k0 >= K) return;
  uint32_t word[8], w, chunk, offset;
  const uint32_t four = digits_of_256<FMT>(own, ref, lane, word);
  if (k < K) {
#pragma unroll
    for (int t = 0; t < 8; ++t) *reinterpret_cast<uint32_t*>(codes + (8 * m + t) * (K / 2) + k / 2) = word[t];
  }
  const int kb4 = K / (FMT == FMT_NVFP4 ? 64 : 128);
  const bool mine = digit_scales<FMT>(four, (int)(m & 15), lane, w, chunk, offset);
  const int c = k0 / (FMT == FMT_NVFP4 ? 64 : 128) + (int)chunk;
  if (mine && c < kb4) *reinterpret_cast<uint32_t*>(scales + ((m >> 4) * kb4 + c) * 512 + offset) = w;
}

// grid: feature tiles x groups of MAX_TOK tokens (the groups of a tile next to one another: W comes from the L2 for all but the first) x S, in
// clusters of S.  tmW: Wq, box [128 rows x 128 B].  tmD, Ds, exponents: the rows where they are there already (codes [8 M or M, K / 2], box
// [rows x 128 B]; tiled scales); X otherwise.
template <int FMT, bool GATED, int ROWS>
__global__ void __launch_bounds__(192, DigitsCfg<FMT, GATED, ROWS>::CTAS_PER_SM)
matvec_digits_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmD, const __nv_bfloat16* __restrict__ X,
                     const uint8_t* __restrict__ Ws, const uint8_t* __restrict__ Ds, const uint32_t* token_exponents,
                     void* __restrict__ Y, int y_is_bf16, int M, int N, int K, int S, int groups, int nst, float alpha, int* err_word) {
  using C = DigitsCfg<FMT, GATED, ROWS>;
  constexpr bool SPLIT = ROWS != ROWS_HERE;
  constexpr int CH = C::CH, PER = C::PER_UNIT;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_gen = smem_raw + (smem_base - smem_u32(smem_raw));
  const int rank = blockIdx.x % S, nt = blockIdx.x / S / groups, group = blockIdx.x / S % groups;
  const int m0 = group * C::MAX_TOK;
  const int mt = M - m0 < C::MAX_TOK ? M - m0 : C::MAX_TOK;   // tokens of this CTA
  const int rows = C::rows(M < C::MAX_TOK ? M : C::MAX_TOK);
  const int stage_bytes = C::stage_bytes(rows);
  constexpr bool PLANES = C::PLANES;
  const uint32_t b_off = C::W_BYTES, sfw_off = b_off + rows * 128, sfb_off = sfw_off + C::TILES * C::SF_BYTES;
  const uint32_t bar_off = nst * stage_bytes;
  const uint32_t bar_base = smem_base + bar_off;
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (C::MAX_STAGES + s); };
  const uint32_t accf_bar = bar_base + 8u * (2 * C::MAX_STAGES);
  auto recv_bar = [&](int w) { return accf_bar + 8u + 8u * w; };   // all partials of the units of epilogue warp w are here
  const uint32_t recv_base = bar_base + C::BAR_BYTES;
  auto ready_bar = [&](int s) { return bar_base + 208u + 8u * s; };   // MXINT4: W has been taken apart (and the digits written)
  volatile uint32_t* exponents = reinterpret_cast<volatile uint32_t*>(smem_gen + bar_off + 112);   // NVFP4: of each token's largest magnitude
  volatile uint32_t* tmem_slot = reinterpret_cast<volatile uint32_t*>(smem_gen + bar_off + 192);
  volatile int* cta_abort = reinterpret_cast<volatile int*>(smem_gen + bar_off + 200);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int k_tiles = (K + C::BK - 1) / C::BK;           // K % 128 == 0: the last stage may be half
  const int kb4 = K / (C::BK / CH);                      // scale chunks per row tile
  const int kt0 = (int)((long long)k_tiles * rank / S), kt1 = (int)((long long)k_tiles * (rank + 1) / S);
  const int steps = kt1 - kt0;                           // one at least
  const uint32_t tmem_cols = C::tmem_cols(rows);
  // unit u = q + 4 c is quarter q of the tile's features and tokens PER c ...; CTA u % S owns it, its epilogue warp u / S % 4
  // adds and stores it
  const int units = C::units(mt);

  auto fetch = [&](int it, int s) {
    const int kt = kt0 + it;
    const uint32_t st = smem_base + s * stage_bytes;
    const uint32_t sf = 512u * (uint32_t)min(CH, kb4 - CH * kt);
    mbar_arrive_expect_tx(full_bar(s), (uint32_t)(C::TILES * C::BF * 128) + C::TILES * sf + (SPLIT ? (uint32_t)rows * 128u + sf : 0u));
#pragma unroll
    for (int w = 0; w < C::TILES; ++w) {
      const int row_tile = nt + w * (N >> 7);            // gated: N % 128 == 0
      tma_load_2d(st + w * C::TILE_BYTES, &tmW, kt * 128, row_tile * C::BF, full_bar(s));
      bulk_load_1d(st + sfw_off + w * C::SF_BYTES, Ws + ((size_t)row_tile * kb4 + CH * kt) * 512, sf, full_bar(s));
    }
  };
  auto fetch_digits = [&](int it, int s) {
    const int kt = kt0 + it;
    const uint32_t st = smem_base + s * stage_bytes;
    tma_load_2d(st + b_off, &tmD, kt * 128, C::DIGITS * m0, full_bar(s));
    bulk_load_1d(st + sfb_off, Ds + ((size_t)(C::DIGITS * m0 >> 7) * kb4 + CH * kt) * 512, 512u * (uint32_t)min(CH, kb4 - CH * kt), full_bar(s));
  };
  // The weights are constants of the layer: their first stages are asked for before anything else.
  const int pre = steps < nst ? steps : nst;
  if (threadIdx.x == 0) {
    for (int s = 0; s < nst; ++s) { mbar_init(full_bar(s), SPLIT || PLANES ? 1 : 1 + 4); mbar_init(empty_bar(s), 1); mbar_init(ready_bar(s), 4); }
    mbar_init(accf_bar, 1);
    for (int w = 0; w < 4; ++w) mbar_init(recv_bar(w), 1);
    *cta_abort = 0;
    fence_mbar_init();
    fence_proxy_async_smem();                            // the copy engine sees the initialised barriers
    for (int it = 0; it < pre; ++it) fetch(it, it);
    if (S > 1)
      for (int w = 0; w < 4 && rank + S * w < units; ++w)
        mbar_arrive_expect_tx(recv_bar(w), (uint32_t)((units - rank - S * w + 4 * S - 1) / (4 * S) * S * C::PART_BYTES));
  }
  if (warp == 1) { tmem_alloc(smem_u32(const_cast<uint32_t*>(tmem_slot)), tmem_cols); tmem_relinquish(); }
  tc_fence_before_sync();
  __syncthreads();
  if (S > 1) cluster_arrive_relaxed();                   // the wait stands before the first access to another CTA
  tc_fence_after_sync();
  const uint32_t tmem_base = *tmem_slot;
  griddep_launch_dependents();

  if (warp == 0) {
    // ------------------------------------------------------------------ W
    griddep_wait();                                      // the stages are freed behind products that wait for the kernel before
    if constexpr (SPLIT) {
      if (elect_one())
        for (int it = 0; it < pre; ++it) fetch_digits(it, it);
      __syncwarp();
    }
    uint32_t s = 0, phase = 0;
    for (int it = pre; it < steps; ++it) {
      if (!mbar_wait_warp(empty_bar(s), phase, cta_abort, err_word, SITE_PRODUCER_EMPTY)) break;
      if (elect_one()) {
        fetch(it, s);
        if constexpr (SPLIT) fetch_digits(it, s);
      }
      __syncwarp();
      if ((int)++s == nst) { s = 0; phase ^= 1; }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer
    griddep_wait();                                      // the waits below count the digits, which wait for the kernel before
    bool ok = true;
    const uint32_t idesc0 = FMT == FMT_NVFP4 ? idesc_nvf4(128, rows) : idesc_mxf4(128, rows, 0, 0);
    const uint32_t idesc2 = FMT == FMT_NVFP4 ? idesc_nvf4(128, rows) : idesc_mxf4(128, rows, 2, 2);
    const uint32_t sfb_t = tmem_base + C::TILES * rows, sfw_t = sfb_t + (PLANES ? 2 : 1) * 4 * CH;   // 4 columns per chunk
    // a group of 64 rows may have the second half of its scale tile: columns 2 and 3 of each chunk
    const uint32_t sfb_m = sfb_t + (SPLIT && (C::DIGITS * m0 & 64) ? 2u : 0u);
    uint32_t s = 0, phase = 0;
    for (int it = 0; it < steps; ++it) {
      if (!mbar_wait_warp(full_bar(s), phase, cta_abort, err_word, SITE_MMA_FULL)) { ok = false; break; }
      if (PLANES && !mbar_wait_warp(ready_bar(s), phase, cta_abort, err_word, SITE_MMA_FULL)) { ok = false; break; }
      tc_fence_after_sync();
      const bool two = kb4 - CH * (kt0 + it) >= CH;        // K % 256 == 128: the last stage is half
      const uint32_t st = smem_base + s * stage_bytes;
      const uint64_t bdesc = make_desc(st + b_off, 16, 1024, kSwizzle128);
      const uint64_t sfw_d = make_desc(st + sfw_off, 0, 128, 0), sfb_d = make_desc(st + sfb_off, 0, 128, 0);
      if (elect_one()) {
#pragma unroll
        for (int c = 0; c < CH; ++c) {
          if (c < CH / 2 || two) {
            tmem_cp_32x128b_warpx4(sfb_t + 4 * c, sfb_d + 32 * c);
            if constexpr (PLANES) tmem_cp_32x128b_warpx4(sfb_t + 4 * (CH + c), sfb_d + 32 * (CH + c));
#pragma unroll
            for (int w = 0; w < C::TILES; ++w) tmem_cp_32x128b_warpx4(sfw_t + 4 * (w * CH + c), sfw_d + 32 * (w * CH + c));
          }
        }
#pragma unroll
        for (int w = 0; w < C::TILES; ++w) {
          const uint32_t acc = tmem_base + w * rows, sfw = sfw_t + 4 * CH * w;
#pragma unroll
          for (int plane = 0; plane < (PLANES ? 2 : 1); ++plane) {
            const uint64_t adesc = make_desc(st + w * C::TILE_BYTES + plane * C::BF * 128, 16, 1024, kSwizzle128);
            const uint32_t sfb = sfb_m + 4 * CH * plane, more = (uint32_t)(it | plane) != 0 ? 1u : 0u;
            if constexpr (FMT == FMT_NVFP4) {            // one chunk per instruction
#pragma unroll
              for (int j = 0; j < 4; ++j)
                if (j < 2 || two) mma_nvf4(acc, adesc + 2 * j, bdesc + 2 * j, idesc0, sfw + 4 * j, sfb + 4 * j, (it | j) != 0);
            } else if constexpr (C::BYTES) {                // a scale byte per instruction
#pragma unroll
              for (int j = 0; j < 4; ++j) mma_mxf8(acc, adesc + 2 * j, bdesc + 2 * j, idesc_mxf8(128, rows, j), sfw, sfb, (it | j) != 0);
            } else {                                     // half a chunk (two scale bytes) per instruction
              mma_mxf4(acc, adesc, bdesc, idesc0, sfw, sfb, more);
              mma_mxf4(acc, adesc + 2, bdesc + 2, idesc2, sfw, sfb, 1);
              if (two) {
                mma_mxf4(acc, adesc + 4, bdesc + 4, idesc0, sfw + 4, sfb + 4, 1);
                mma_mxf4(acc, adesc + 6, bdesc + 6, idesc2, sfw + 4, sfb + 4, 1);
              }
            }
          }
        }
        tc_commit(empty_bar(s));
      }
      __syncwarp();
      if ((int)++s == nst) { s = 0; phase ^= 1; }
    }
    if (ok && elect_one()) tc_commit(accf_bar);
    __syncwarp();
  } else {
    // ------------------------------------------------------------------ digits, then the sums (warps 2..5)
    const int ew = warp - 2;
    griddep_wait();
    bool ok = true;
    // MXINT4: the nibbles of a stage's W -> the two operands, in place and behind it, 16 bytes per thread at a time
    auto take_apart = [&](uint32_t st) {
#pragma unroll
      for (int w = 0; w < C::TILES; ++w)
#pragma unroll
        for (int i = 0; i < C::BF * 128 / (16 * 128); ++i) {
          const uint32_t a = st + w * C::TILE_BYTES + i * 2048 + (threadIdx.x - 64) * 16;
          uint32_t n[4], h[4];
          asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(n[0]), "=r"(n[1]), "=r"(n[2]), "=r"(n[3]) : "r"(a));
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            // bits b3 b2 of a nibble -> sign b3, magnitude code 1 if b2, else 2 if b3
            const uint32_t up2 = n[e] >> 2, up1 = n[e] >> 1;
            h[e] = (n[e] & 0x88888888u) | (up2 & 0x11111111u) | (up2 & ~up1 & 0x22222222u);
            n[e] &= 0x33333333u;
          }
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(n[0]), "r"(n[1]), "r"(n[2]), "r"(n[3]) : "memory");
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a + C::BF * 128), "r"(h[0]), "r"(h[1]), "r"(h[2]), "r"(h[3]) : "memory");
        }
    };
    if constexpr (SPLIT && PLANES) {
      uint32_t s = 0, phase = 0;
      for (int it = 0; it < steps; ++it) {
        if (!mbar_wait_warp(full_bar(s), phase, cta_abort, err_word, SITE_MMA_FULL)) { ok = false; break; }
        const uint32_t st = smem_base + s * stage_bytes;
        take_apart(st);
#pragma unroll
        for (int i = 0; i < C::SF_BYTES / 512; ++i) {    // the digits' scales for the upper halves: two powers higher
          const uint32_t a = st + sfb_off + i * 512 + (threadIdx.x - 64) * 4;
          uint32_t v;
          asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a));
          asm volatile("st.shared.b32 [%0], %1;" ::"r"(a + C::SF_BYTES), "r"(__vaddus4(v, 0x02020202u)) : "memory");
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(ready_bar(s));
        if ((int)++s == nst) { s = 0; phase ^= 1; }
      }
    } else if constexpr (SPLIT) {
      if (FMT == FMT_NVFP4 && ROWS == ROWS_AHEAD) {
        if (warp == 2 && lane < mt) exponents[lane] = token_exponents[m0 + lane];
        named_barrier_sync(1, 128);
      }
    } else {
      // a warp takes 256 of K of a token, a lane eight elements (16 bytes)
      auto load = [&](int m, int it) {
        const int k = (kt0 + it) * C::BK + 8 * lane;
        return m < mt && k < K ? load_once(X + (int64_t)(m0 + m) * K + k) : make_uint4(0, 0, 0, 0);
      };
      if constexpr (FMT == FMT_NVFP4) {
        for (int m = ew; m < mt; m += 4) {
          uint32_t top = 0;
          for (int it = 0; it < steps; it += 8) {
            uint4 x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = it + j < steps ? load(m, it + j) : make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int j = 0; j < 8; ++j) top = max(top, largest8(x[j]));
          }
          top = __reduce_max_sync(0xFFFFFFFFu, top);
          if (lane == 0) exponents[m] = max(top >> 7, kLeastExponent + kScaleBinades);
        }
        named_barrier_sync(1, 128);
      }
      constexpr int SLOTS = C::FEW_TOK / 4;
      uint4 next[SLOTS];
#pragma unroll
      for (int j = 0; j < SLOTS; ++j) next[j] = load(4 * j + ew, 0);
      uint32_t s = 0, phase = PLANES ? 0 : 1;
      for (int it = 0; it < steps; ++it) {
        uint4 xr[SLOTS];
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) {
          xr[j] = next[j];
          if (it + 1 < steps) next[j] = load(4 * j + ((ew - it - 1) & 3), it + 1);
        }
        // MXINT4: until W is there, and with it the stage free; else until the stage is free (the first time round the barrier's phase
        // before its first counts as completed)
        if (!mbar_wait_warp(PLANES ? full_bar(s) : empty_bar(s), phase, cta_abort, err_word,
                            PLANES ? SITE_MMA_FULL : SITE_PRODUCER_EMPTY)) { ok = false; break; }
        const uint32_t st = smem_base + s * stage_bytes;
#pragma unroll
        for (int j = 0; j < SLOTS; ++j) {
          const int m = 4 * j + ((ew - it) & 3);
          if (m < mt) {                                  // the same for the whole warp
            uint32_t word[8], w, chunk, offset;
            const uint32_t four = digits_of_256<FMT>(xr[j], FMT == FMT_NVFP4 ? exponents[m] : 0u, lane, word);
            // row 8 m + t of the operand: 128 bytes in the 128-byte swizzle (8 m + t = t modulo 8)
            const uint32_t row0 = st + b_off + m * 1024 + (lane & 3) * 4;
#pragma unroll
            for (int t = 0; t < 8; ++t)
              asm volatile("st.shared.b32 [%0], %1;" ::"r"(row0 + t * 128 + (((lane >> 2) ^ t) << 4)), "r"(word[t]) : "memory");
            if (digit_scales<FMT>(four, m, lane, w, chunk, offset)) {
              asm volatile("st.shared.b32 [%0], %1;" ::"r"(st + sfb_off + chunk * 512 + offset), "r"(w) : "memory");
              if constexpr (PLANES)
                asm volatile("st.shared.b32 [%0], %1;" ::"r"(st + sfb_off + C::SF_BYTES + chunk * 512 + offset), "r"(__vaddus4(w, 0x02020202u)) : "memory");
            }
          }
        }
        if constexpr (PLANES) take_apart(st);
        fence_proxy_async_smem();                        // the tensor cores see what has been stored
        __syncwarp();
        if (lane == 0) mbar_arrive(PLANES ? ready_bar(s) : full_bar(s));
        if ((int)++s == nst) { s = 0; phase ^= 1; }
      }
    }

    // ---- sums: the accumulator's columns 8 m ... 8 m + 7 are the digits of token m
    const int q = warp & 3;                              // quarter of the features that this warp can read
    const uint32_t tacc = tmem_base + ((uint32_t)(q * 32) << 16);
    ok = ok && __all_sync(0xFFFFFFFFu, mbar_wait(accf_bar, 0, cta_abort, err_word, SITE_EPI_ACC_FULL));
    tc_fence_after_sync();
    auto add8 = [&](const uint32_t* d, int m) {
      float y = __uint_as_float(d[7]);                   // from the smallest digit on
      if constexpr (FMT == FMT_NVFP4) {
#pragma unroll
        for (int t = 6; t >= 0; --t) y = fmaf(y, 0.125f, __uint_as_float(d[t]));
        const uint32_t ref = exponents[m < mt ? m : 0];
        return y * __uint_as_float(ref == 255u ? 0x7FC00000u : (ref - 8u) << 23);
      } else {
#pragma unroll
        for (int t = 6; t >= 0; --t) y += __uint_as_float(d[t]);
        return y;
      }
    };
    // calls f(c, the four values of this lane's feature in unit q + 4 c) for every c
    auto units_of_quarter = [&](auto f) {
      if constexpr (ROWS == ROWS_QUANTIZED) {
        static_assert(GATED, "the GEMM of one projection has kernels of its own");
        for (int c0 = 0; 4 * c0 < units; c0 += 16 / PER) {
          uint32_t d[2][16];
#pragma unroll
          for (int w = 0; w < 2; ++w) tmem_ld_32x32_x16(tacc + w * rows + PER * c0, d[w]);
          tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 16 / PER; ++i) {
            const float p[4] = {__uint_as_float(d[0][2 * i]), __uint_as_float(d[1][2 * i]), __uint_as_float(d[0][2 * i + 1]), __uint_as_float(d[1][2 * i + 1])};
            if (4 * (c0 + i) < units) f(c0 + i, p);
          }
        }
      } else {
        for (int c = 0; 4 * c < units; ++c) {
          uint32_t d[32];
          float p[4];
          if constexpr (GATED) {
            tmem_ld_32x32_x16(tacc + 16 * c, *reinterpret_cast<uint32_t(*)[16]>(d));
            tmem_ld_32x32_x16(tacc + rows + 16 * c, *reinterpret_cast<uint32_t(*)[16]>(d + 16));
            tmem_ld_wait();
            p[0] = add8(d, 2 * c); p[1] = add8(d + 16, 2 * c);
            p[2] = add8(d + 8, 2 * c + 1); p[3] = add8(d + 24, 2 * c + 1);
          } else {
            tmem_ld_32x32(tacc + 32 * c, d);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 4; ++i) p[i] = add8(d + 8 * i, 4 * c + i);
          }
          f(c, p);
        }
      }
    };
    auto put = [&](int m, int64_t n, float y) {
      if (m < mt && n < N) {
        const int64_t o = (int64_t)(m0 + m) * N + n;
        if (y_is_bf16) static_cast<__nv_bfloat16*>(Y)[o] = __float2bfloat16_rn(y);
        else static_cast<float*>(Y)[o] = y;
      }
    };
    auto store = [&](int c, int quarter, const float (&v)[4]) {
      const int64_t n = (int64_t)nt * C::BF + quarter * 32 + lane;
      if constexpr (GATED) {
        put(2 * c, n, silu(v[0] * alpha) * (v[1] * alpha));
        put(2 * c + 1, n, silu(v[2] * alpha) * (v[3] * alpha));
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) put(4 * c + i, n, v[i] * alpha);
      }
    };
    if (S == 1) {
      if (ok) units_of_quarter([&](int c, const float (&p)[4]) { store(c, q, p); });
    } else {
      cluster_wait();
      if (ok)
        units_of_quarter([&](int c, const float (&p)[4]) {
          const int u = q + 4 * c, ui = u / S, owner = u - ui * S;
          st_async_v4(map_to_cta(recv_base + (uint32_t)((ui * S + rank) * C::PART_BYTES + lane * 16), (uint32_t)owner), __float_as_uint(p[0]),
                      __float_as_uint(p[1]), __float_as_uint(p[2]), __float_as_uint(p[3]), map_to_cta(recv_bar(ui & 3), (uint32_t)owner));
        });
      if (ok && rank + S * ew < units) {
        ok = __all_sync(0xFFFFFFFFu, mbar_wait_cluster(recv_bar(ew), 0, cta_abort, err_word, SITE_EPI_ACC_FULL));
        for (int u = rank + S * ew, ui = ew; u < units && ok; u += 4 * S, ui += 4) {
          float v[4] = {0.f, 0.f, 0.f, 0.f};             // rank order: the result does not depend on timing
#pragma unroll
          for (int r = 0; r < C::MAX_CLUSTER; ++r)
            if (r < S) {
              float4 p;
              asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(p.x), "=f"(p.y), "=f"(p.z), "=f"(p.w)
                           : "r"(recv_base + (uint32_t)((ui * S + r) * C::PART_BYTES + lane * 16)));
              v[0] += p.x; v[1] += p.y; v[2] += p.z; v[3] += p.w;
            }
          store(u >> 2, u & 3, v);
        }
      }
    }
    tc_fence_before_sync();
  }
  if (S > 1 && warp < 2) cluster_wait();                 // the epilogue warps have waited above

  // ------------------------------------------------------------------ teardown
  __syncthreads();
  if (S > 1 && *cta_abort) cluster_sync_all();           // others may still push to this CTA, see the few-token rotation
  if (warp == 1) {
    tc_fence_after_sync();
    tmem_dealloc(tmem_base, tmem_cols);
  }
}

}  // namespace torq
