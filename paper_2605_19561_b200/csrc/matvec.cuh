// Products of a few tokens with 4-bit weights, the activations in bfloat16 (not quantized):
//   y[m, n] = alpha sum_k x[m, k] w^[n, k],   w^ = code * block scale
// and the gated pair of projections, both stacked in one weight matrix [2 N, K]:
//   y[m, n] = silu(g) u,  g / u = the product with row n / N + n,  silu(g) = g / (1 + exp(-g)).
// Streaming the weights from HBM once is the work (K / 2 bytes and K / 32 or K / 16 scale bytes per row).
//
// The tensor cores' block-scaled instructions want both operands in few bits, so the codes are widened here: to float16,
// exactly (e2m1 by the conversion instruction, 41 pairs per clock and SM measured against 22 by masks and shifts; integers by
// a mask and a subtraction), and contracted by the warp-level mma.m16n8k16 with float32 accumulators: 16 features x 8 tokens.
// Its rate (1013 multiply-adds per clock and SM measured) is 2.7 times what the weights' stream asks for at 8 tokens.
//  * x becomes float16 as well, per token and 128 of K scaled by a power of two that puts the largest magnitude into [2^14, 2^15):
//    bfloat16's 8 bits are kept exactly down to 2^-31 of that magnitude, and what is smaller than 2^-39 of it is lost.  The
//    power of two comes back in float32 when the 128 products have been added.
//  * MXFP4 and MXINT4: the sum over one block of 32 is multiplied by the block's power of two in float32.  NVFP4: the E4M3 scale
//    goes into the codes (e2m1 x e4m3 has 6 significant bits and lies in [2^-10, 2688]: exact in float16).
//
// A CTA has 128 rows of W (gated: 64 of the gate and the 64 of the up projection that belong to them) and a range of K; a CLUSTER of S
// CTAs shares the rows.  The x of its range is widened ahead of the contraction, by all warps (one of nine doing it stage by stage for
// the others was what the kernel waited for: 8 tokens, 5120 x 51200, 55.9 us against 39.9).  Then warp 8 fetches W by TMA (256 of K per
// stage: 128 bytes per row in the 128-byte swizzle, and the scales' 512-byte chunks) and warps 0..7 contract.  Up to 16 tokens such a
// warp has two instructions' rows (32) and half of the stage's K, which halves what it reads of x; above, 16 rows and all of it.
// Gated: rows 0..7 of an instruction are gates, 8..15 the ups of the same features, so that both sums of a feature meet in one lane.
// ldmatrix gives lane (g, t) = (lane / 4, lane % 4) word t of a block of rows g and g + 8: eight elements that stay in their order,
// so that x is read in its own order, 16 bytes per block.
// Every warp stores its partial sums straight into the shared memory of the CTA that owns its rows (st.async in a cluster), which adds
// them in the order of their ranks.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <type_traits>
#include "activation.cuh"
#include "sm100_ptx.cuh"

namespace torq {

template <int FMT, int NT>
struct MatvecCfg {
  static constexpr int ROWS = 128;
  static constexpr int BK = 256;                       // elements of K per stage (128 bytes per row)
  static constexpr int W_BYTES = ROWS * 128;
  static constexpr int CH = FMT == FMT_NVFP4 ? 4 : 2;  // scale chunks per stage and 128-row tile
  static constexpr int STAGES = 3;
  static constexpr int MAX_CLUSTER = 8;
  static constexpr int WARPS = 8;                      // that contract
  static constexpr int RT = NT > 2 ? 1 : 2;            // instructions' rows per warp: the warps split a stage's K RT ways
  static constexpr int THREADS = 32 * (WARPS + 1);
  static constexpr int BAR_BYTES = 128;
  // what arrives at the owner of 8 / S instructions' rows: 16 bytes per lane and eight tokens from RT warps of S CTAs
  static constexpr int RECV_BYTES = WARPS * RT * 512 * NT;
  static constexpr int CTAS_PER_SM = NT == 1 ? 3 : 2;
  __host__ __device__ static constexpr int stage_bytes(bool gated) { return W_BYTES + (gated ? 2 : 1) * CH * 512; }
  // float16 row of a token (eight lanes that read 16 bytes of two rows hit all banks), and the powers of two of 8 NT tokens per 128 of K
  __host__ __device__ static constexpr int x_row(int steps) { return steps * BK * 2 + 64; }
  __host__ __device__ static constexpr int x_bytes(int tokens, int steps) { return tokens * x_row(steps) + steps * 2 * 32 * NT; }
  // `tokens` of a group, `steps`: the longest range of K, in stages
  __host__ __device__ static constexpr int smem_bytes(int tokens, int steps, bool gated) {
    return 1024 + STAGES * stage_bytes(gated) + x_bytes(tokens, steps) + RECV_BYTES + BAR_BYTES;
  }
};

__device__ __forceinline__ void mma_16816_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Four 8 x 8 matrices of 16-bit pairs: lane l gives the address of row l % 8 of matrix l / 8 and gets word l % 4 of row l / 4 of each.
__device__ __forceinline__ void ldmatrix_x4(uint32_t a, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a));
}
// The same with nothing to add to.
__device__ __forceinline__ void mma_16816_f16_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}

// Eight codes of one word -> four float16 pairs.  e2m1: elements (0,1) (2,3) (4,5) (6,7); integers: (0,4) (1,5) (2,6) (3,7), the
// order in which a mask finds them (x is stored in the same one).
template <int FMT>
__device__ __forceinline__ void widen8(uint32_t w, uint32_t (&p)[4]) {
  if constexpr (FMT == FMT_MXINT4) {
    // nibble n of [-8, 8) into float16's mantissa: the bits of 1024 + (n + 8), or of 1024 + 16 (n + 8)
    auto low = [](uint32_t v) {
      const uint32_t b = (v & 0x000F000Fu) ^ 0x64086408u;
      const __half2 h = __hsub2(*reinterpret_cast<const __half2*>(&b), __half2half2(__ushort_as_half(0x6408)));          // 1032
      return *reinterpret_cast<const uint32_t*>(&h);
    };
    auto high = [](uint32_t v) {
      const uint32_t b = (v & 0x00F000F0u) ^ 0x64806480u;
      const __half2 h = __hfma2(*reinterpret_cast<const __half2*>(&b), __half2half2(__ushort_as_half(0x2C00)),           // 1 / 16
                                __half2half2(__ushort_as_half(0xD480)));                                                 // -72
      return *reinterpret_cast<const uint32_t*>(&h);
    };
    p[0] = low(w); p[1] = high(w); p[2] = low(w >> 8); p[3] = high(w >> 8);
  } else {
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(p[0]), "=r"(p[1]), "=r"(p[2]), "=r"(p[3]) : "r"(w));
  }
}
// Byte `sel & 3` of a word of E4M3 scales, as a float16 pair (sel: the byte's number twice, as __byte_perm takes it).
__device__ __forceinline__ uint32_t e4m3_pair(uint32_t word, uint32_t sel) {
  const uint32_t b = __byte_perm(word, 0, sel);
  uint32_t r;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}" : "=r"(r) : "r"(b));
  return r;
}
// The four E8M0 bytes of a word as float32 (by way of bfloat16, which has their range: byte 0 is 2^-127).
__device__ __forceinline__ void e8m0_values(uint32_t word, float (&v)[4]) {
  uint32_t a, b;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %2;\n\tcvt.rn.bf16x2.ue8m0x2 %0, lo;\n\tcvt.rn.bf16x2.ue8m0x2 %1, hi;\n\t}"
      : "=r"(a), "=r"(b) : "r"(word));
  v[0] = __uint_as_float(a << 16); v[1] = __uint_as_float(a & 0xFFFF0000u);
  v[2] = __uint_as_float(b << 16); v[3] = __uint_as_float(b & 0xFFFF0000u);
}
__device__ __forceinline__ uint32_t hmul2_bits(uint32_t a, uint32_t b) {
  const __half2 v = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&v);
}

// grid = (row tiles * S in clusters of S along x, groups of 8 NT tokens).  tmW: Wq [rows, K / 2 bytes], box [64 x 128 B].
template <int FMT, int NT, bool GATED>
__global__ void __launch_bounds__(MatvecCfg<FMT, NT>::THREADS, MatvecCfg<FMT, NT>::CTAS_PER_SM)
matvec_kernel(const __grid_constant__ CUtensorMap tmW, const __nv_bfloat16* __restrict__ X, const uint8_t* __restrict__ Ws,
              void* __restrict__ Y, int y_is_bf16, int M, int N, int K, int S, float alpha, int* err_word) {
  using C = MatvecCfg<FMT, NT>;
  constexpr int CH = C::CH, STAGES = C::STAGES, RT = C::RT;
  constexpr int STAGE_BYTES = C::stage_bytes(GATED);
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const int rank = blockIdx.x % S, tile = blockIdx.x / S;
  const int m0 = blockIdx.y * 8 * NT;
  const int mt = M - m0 < 8 * NT ? M - m0 : 8 * NT;      // tokens of this CTA
  const int k_tiles = (K + C::BK - 1) / C::BK;           // K % 128 == 0: the last stage may be half
  const int kb4 = K / (CH == 4 ? 64 : 128);              // scale chunks per row tile
  const int kt0 = (int)((long long)k_tiles * rank / S), kt1 = (int)((long long)k_tiles * (rank + 1) / S);
  const int steps = kt1 - kt0;                           // one at least
  const int x_row = C::x_row((k_tiles + S - 1) / S);
  const uint32_t x_base = base + STAGES * STAGE_BYTES;
  const uint32_t sx_base = x_base + (uint32_t)((M < 8 * NT ? M : 8 * NT) * x_row);
  const uint32_t recv_base = sx_base + (uint32_t)((k_tiles + S - 1) / S * 2 * 32 * NT);
  const uint32_t bar_base = recv_base + C::RECV_BYTES;
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (STAGES + s); };
  const uint32_t recv_bar = bar_base + 8u * (2 * STAGES);   // all partial sums that this CTA owns are here
  volatile int* cta_abort = reinterpret_cast<volatile int*>(smem_raw + (bar_base + 8u * (2 * STAGES + 1) - smem_u32(smem_raw)));
  const int n0 = tile * (GATED ? 64 : 128), row1 = GATED ? N + n0 : n0 + 64;   // first rows of the two halves of the tile

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  auto fetch = [&](int it, int s) {
    const int kt = kt0 + it;
    const uint32_t st = base + s * STAGE_BYTES;
    const uint32_t sf = 512u * (uint32_t)min(CH, kb4 - CH * kt);
    mbar_arrive_expect_tx(full_bar(s), (uint32_t)C::W_BYTES + (GATED ? 2u : 1u) * sf);
    tma_load_2d(st, &tmW, kt * 128, n0, full_bar(s));
    tma_load_2d(st + C::W_BYTES / 2, &tmW, kt * 128, row1, full_bar(s));
    bulk_load_1d(st + C::W_BYTES, Ws + ((size_t)(n0 >> 7) * kb4 + CH * kt) * 512, sf, full_bar(s));
    if constexpr (GATED) bulk_load_1d(st + C::W_BYTES + CH * 512, Ws + ((size_t)(row1 >> 7) * kb4 + CH * kt) * 512, sf, full_bar(s));
  };
  // The weights are constants of the layer: their first stages are asked for before anything else.
  const int pre = steps < STAGES ? steps : STAGES;
  if (threadIdx.x == 32 * C::WARPS) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), C::WARPS); }
    mbar_init(recv_bar, 1);
    *cta_abort = 0;
    fence_mbar_init();
    fence_proxy_async_smem();
    if (S > 1) mbar_arrive_expect_tx(recv_bar, (uint32_t)C::RECV_BYTES);
    for (int it = 0; it < pre; ++it) fetch(it, it);
  }
  __syncthreads();
  if (S > 1) cluster_arrive_relaxed();                   // the wait stands before the first access to another CTA
  griddep_launch_dependents();
  griddep_wait();

  // x of this CTA's range: a warp takes 256 of K of a token, four such pieces at a time; a lane has eight elements (16 bytes)
  {
    const int pieces = mt * steps;
    for (int p0 = warp; p0 < pieces; p0 += 4 * (C::WARPS + 1)) {
      uint4 xr[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int p = p0 + i * (C::WARPS + 1), m = p / steps, k = (kt0 + p - m * steps) * C::BK + 8 * lane;
        xr[i] = p < pieces && k < K ? __ldg(reinterpret_cast<const uint4*>(X + (int64_t)(m0 + m) * K + k)) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int p = p0 + i * (C::WARPS + 1), m = p / steps, it = p - m * steps;
        if (p < pieces) {                                // the same for the whole warp
          const uint32_t w[4] = {xr[i].x, xr[i].y, xr[i].z, xr[i].w};
          float v[8];
          float amax = 0.f;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v[2 * e] = __uint_as_float(w[e] << 16);
            v[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
            amax = fmaxf(amax, fmaxf(fabsf(v[2 * e]), fabsf(v[2 * e + 1])));
          }
#pragma unroll
          for (int o = 1; o < 16; o <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, o));
          // 2^14 / 2^floor(log2 amax), at most 2^126: exponent field 127 + 14 - (ef - 127)
          const uint32_t ef = __float_as_uint(amax) >> 23;
          const uint32_t fe = ef > 15u ? 268u - ef : 253u;
          const float f = __uint_as_float(fe << 23);
          uint32_t o4[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float a = FMT == FMT_MXINT4 ? v[e] : v[2 * e], b = FMT == FMT_MXINT4 ? v[e + 4] : v[2 * e + 1];
            const __half2 h = __floats2half2_rn(a * f, b * f);
            o4[e] = *reinterpret_cast<const uint32_t*>(&h);
          }
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(x_base + (uint32_t)(m * x_row + it * (C::BK * 2) + 16 * lane)), "r"(o4[0]),
                       "r"(o4[1]), "r"(o4[2]), "r"(o4[3]) : "memory");
          if ((lane & 15) == 0)
            asm volatile("st.shared.b32 [%0], %1;" ::"r"(sx_base + (uint32_t)((2 * it + (lane >> 4)) * 32 * NT + 4 * m)), "r"((254u - fe) << 23) : "memory");
        }
      }
    }
  }
  __syncthreads();

  if (warp == C::WARPS) {
    // ------------------------------------------------------------------ W
    uint32_t s = 0, phase = 0;
    for (int it = pre; it < steps; ++it) {
      if (!mbar_wait_warp(empty_bar(s), phase, cta_abort, err_word, SITE_PRODUCER_EMPTY)) break;
      if (elect_one()) fetch(it, s);
      __syncwarp();
      if (++s == STAGES) { s = 0; phase ^= 1; }
    }
    if (S > 1) cluster_wait();
  } else {
    // ------------------------------------------------------------------ contraction
    const int g = lane >> 2, t = lane & 3;
    const int t0 = RT * (RT == 2 ? warp & 3 : warp);     // first of this warp's instructions' row groups, 0..7
    const int q0 = RT == 2 ? warp >> 2 : 0;              // and its 128 of K of a stage (RT == 1: both)
    // the row whose address this lane gives ldmatrix (of the first group), and the swizzled address of its first block
    const int lrow = GATED ? 8 * t0 + (lane & 7) + 64 * ((lane >> 3) & 1) : 16 * t0 + (lane & 15);
    const uint32_t w_off = (uint32_t)(lrow * 128 + (((lane >> 4) ^ (lane & 7)) << 4));
    constexpr uint32_t W_GROUP = (GATED ? 8 : 16) * 128;   // from one group to the next
    uint32_t x_addr[NT];                                 // tokens that there are not read another one's: their sums are not stored
#pragma unroll
    for (int j = 0; j < NT; ++j) x_addr[j] = x_base + (uint32_t)(min(8 * j + g, mt - 1) * x_row + 16 * t);
    const uint32_t sel = (uint32_t)((t >> 1) * 0x11);    // NVFP4: words 0, 1 of a 32 are its first block of 16

    // scale bytes of rows g and g + 8; the halves of a gated tile start at row 0 or 64 of a scale tile
    auto sf_cell = [](int r) { return (uint32_t)((r & 31) * 16 + ((r & 127) >> 5) * 4); };
    uint32_t sf0[RT], sf1[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int a = (GATED ? 8 : 16) * (t0 + r) + g;
      sf0[r] = C::W_BYTES + sf_cell((GATED ? (n0 & 64) : 0) + a);
      sf1[r] = GATED ? C::W_BYTES + CH * 512 + sf_cell((row1 & 64) + a) : C::W_BYTES + sf_cell(a + 8);
    }
    float acc[RT][NT][4];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[r][j][e] = 0.f;

    bool ok = true;
    uint32_t s = 0, phase = 0;
    for (int it = 0; it < steps; ++it) {
      if (!__all_sync(0xFFFFFFFFu, mbar_try_wait(full_bar(s), phase)) &&
          !mbar_wait_warp(full_bar(s), phase, cta_abort, err_word, SITE_MMA_FULL)) { ok = false; break; }
      const uint32_t st = base + s * STAGE_BYTES;
#pragma unroll
      for (int qq = 0; qq < 3 - RT; ++qq) {            // 128 of K
        const int q = q0 + qq;
        if (q == 1 && (kt0 + it) * C::BK + 128 >= K) break;
        const uint32_t xk = (uint32_t)(it * (C::BK * 2) + q * 256);
        float part[RT][NT][4];
        uint32_t nv0[RT][2], nv1[RT][2];               // NVFP4: scale words of this 128
        float mx0[RT][4], mx1[RT][4];                  // else: block scales
#pragma unroll
        for (int r = 0; r < RT; ++r) {
          if constexpr (FMT == FMT_NVFP4) {
#pragma unroll
            for (int h = 0; h < 2; ++h) { nv0[r][h] = lds32(st + sf0[r] + (2 * q + h) * 512); nv1[r][h] = lds32(st + sf1[r] + (2 * q + h) * 512); }
          } else {
            e8m0_values(lds32(st + sf0[r] + q * 512), mx0[r]);
            e8m0_values(lds32(st + sf1[r] + q * 512), mx1[r]);
          }
        }
#pragma unroll
        for (int pair = 0; pair < 2; ++pair) {         // two blocks of 32
          const uint32_t wa = (st + w_off) ^ (uint32_t)((2 * q + pair) << 5);
          uint32_t w[RT][4];
#pragma unroll
          for (int r = 0; r < RT; ++r) ldmatrix_x4(wa + r * W_GROUP, w[r]);
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            uint4 x[NT];
#pragma unroll
            for (int j = 0; j < NT; ++j) x[j] = lds128(x_addr[j] + xk + (2 * pair + b) * 64);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
              uint32_t a0[4], a1[4];
              widen8<FMT>(w[r][2 * b], a0);
              widen8<FMT>(w[r][2 * b + 1], a1);
              if constexpr (FMT == FMT_NVFP4) {
                const uint32_t f0 = e4m3_pair(nv0[r][pair], sel + b * 0x22u), f1 = e4m3_pair(nv1[r][pair], sel + b * 0x22u);
#pragma unroll
                for (int e = 0; e < 4; ++e) { a0[e] = hmul2_bits(a0[e], f0); a1[e] = hmul2_bits(a1[e], f1); }
              }
#pragma unroll
              for (int j = 0; j < NT; ++j) {
                if constexpr (FMT == FMT_NVFP4) {
                  if (pair + b == 0) mma_16816_f16_first(part[r][j], a0[0], a1[0], a0[1], a1[1], x[j].x, x[j].y);
                  else mma_16816_f16(part[r][j], a0[0], a1[0], a0[1], a1[1], x[j].x, x[j].y);
                  mma_16816_f16(part[r][j], a0[2], a1[2], a0[3], a1[3], x[j].z, x[j].w);
                } else {
                  float d[4];
                  mma_16816_f16_first(d, a0[0], a1[0], a0[1], a1[1], x[j].x, x[j].y);
                  mma_16816_f16(d, a0[2], a1[2], a0[3], a1[3], x[j].z, x[j].w);
                  const float f0 = mx0[r][2 * pair + b], f1 = mx1[r][2 * pair + b];
                  if (pair + b == 0) {
                    part[r][j][0] = d[0] * f0; part[r][j][1] = d[1] * f0;
                    part[r][j][2] = d[2] * f1; part[r][j][3] = d[3] * f1;
                  } else {
                    part[r][j][0] = fmaf(d[0], f0, part[r][j][0]);
                    part[r][j][1] = fmaf(d[1], f0, part[r][j][1]);
                    part[r][j][2] = fmaf(d[2], f1, part[r][j][2]);
                    part[r][j][3] = fmaf(d[3], f1, part[r][j][3]);
                  }
                }
              }
            }
          }
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {                 // x's power of two: tokens 2 t and 2 t + 1
          uint32_t f0, f1;
          asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(f0), "=r"(f1) : "r"(sx_base + (uint32_t)((2 * it + q) * 32 * NT + 4 * (8 * j + 2 * t))));
#pragma unroll
          for (int r = 0; r < RT; ++r) {
            acc[r][j][0] = fmaf(part[r][j][0], __uint_as_float(f0), acc[r][j][0]);
            acc[r][j][1] = fmaf(part[r][j][1], __uint_as_float(f1), acc[r][j][1]);
            acc[r][j][2] = fmaf(part[r][j][2], __uint_as_float(f0), acc[r][j][2]);
            acc[r][j][3] = fmaf(part[r][j][3], __uint_as_float(f1), acc[r][j][3]);
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty_bar(s));
      if (++s == STAGES) { s = 0; phase ^= 1; }
    }

    // CTA r owns row groups r 8 / S ...: [group of these][source: CTA, warp of the group][eight tokens][lane] 16 bytes
    const int per = C::WARPS / S;
    if (S > 1) cluster_wait();
#pragma unroll
    for (int r = 0; r < RT; ++r) {
      const int owner = (t0 + r) / per, slot = (t0 + r) - owner * per;
      const uint32_t to = recv_base + (uint32_t)(((slot * S + rank) * RT + q0) * NT * 512 + lane * 16);
      if (S > 1) {
        const uint32_t far = map_to_cta(to, (uint32_t)owner), far_bar = map_to_cta(recv_bar, (uint32_t)owner);
#pragma unroll
        for (int j = 0; j < NT; ++j)
          st_async_v4(far + j * 512, __float_as_uint(acc[r][j][0]), __float_as_uint(acc[r][j][1]), __float_as_uint(acc[r][j][2]),
                      __float_as_uint(acc[r][j][3]), far_bar);
      } else {                                           // launched without clusters (st.async then faults): plain stores and a barrier
#pragma unroll
        for (int j = 0; j < NT; ++j)
          asm volatile("st.shared.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to + j * 512), "f"(acc[r][j][0]), "f"(acc[r][j][1]), "f"(acc[r][j][2]),
                       "f"(acc[r][j][3]) : "memory");
      }
    }
    if (S == 1) named_barrier_sync(1, 32 * C::WARPS);
    if (warp < per && ok) {
      if (S > 1) ok = __all_sync(0xFFFFFFFFu, mbar_wait_cluster(recv_bar, 0, cta_abort, err_word, SITE_EPI_ACC_FULL));
      if (ok) {
        const int n = n0 + (rank * per + warp) * (GATED ? 8 : 16) + g;
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          float v[4] = {0.f, 0.f, 0.f, 0.f};
          for (int r = 0; r < RT * S; ++r) {             // the result does not depend on timing
            const uint4 p = lds128(recv_base + (uint32_t)(((warp * S * RT + r) * NT + j) * 512 + lane * 16));
            v[0] += __uint_as_float(p.x); v[1] += __uint_as_float(p.y);
            v[2] += __uint_as_float(p.z); v[3] += __uint_as_float(p.w);
          }
          // lane (g, t) has rows g, g + 8 of tokens 8 j + 2 t, 2 t + 1
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int m = 8 * j + 2 * t + e;
            auto put = [&](int col, float y) {
              if (col < N) {
                const int64_t o = (int64_t)(m0 + m) * N + col;
                if (y_is_bf16) static_cast<__nv_bfloat16*>(Y)[o] = __float2bfloat16_rn(y);
                else static_cast<float*>(Y)[o] = y;
              }
            };
            if (m < mt) {
              if constexpr (GATED) {
                put(n, silu(v[e] * alpha) * (v[2 + e] * alpha));
              } else {
                put(n, v[e] * alpha);
                put(n + 8, v[2 + e] * alpha);
              }
            }
          }
        }
      }
    }
  }
  __syncthreads();
  // After a wait has given up, others may still push to this CTA: stay until they have left or given up as well (the
  // barrier does not count threads that have exited).
  if (S > 1 && *cta_abort) cluster_sync_all();
}

}  // namespace torq
