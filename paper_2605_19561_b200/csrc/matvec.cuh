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
// A CTA has 128 rows of W (gated: 64 of the gate and the 64 of the up projection that belong to them) and a range of K; a
// CLUSTER of S CTAs shares the rows.  Roles: warp 8 fetches W by TMA (256 of K per stage: 128 bytes per row in the
// 128-byte swizzle, and the scales' 512-byte chunks); warps 0..7 have 16 rows each (gated: rows 0..7 of a warp's
// instruction are gates, 8..15 the ups of the same features, so that both sums of a feature meet in one lane).  All eight
// together widen the stage's x for all of them, one stage ahead.  Lane (g, t) = (lane / 4, lane % 4) reads word t of
// a block of rows g and g + 8: eight elements that stay in their order, so that x is read in its own order, 16 bytes per block.
// With S > 1 every warp stores its partial sums straight into the shared memory of the CTA that owns its rows (st.async),
// which adds them in rank order.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <type_traits>
#include "activation.cuh"
#include "sm100_ptx.cuh"

namespace torq {

template <int FMT>
struct MatvecCfg {
  static constexpr int ROWS = 128;
  static constexpr int BK = 256;                       // elements of K per stage (128 bytes per row)
  static constexpr int W_BYTES = ROWS * 128;
  static constexpr int CH = FMT == FMT_NVFP4 ? 4 : 2;  // scale chunks per stage and 128-row tile
  static constexpr int STAGES = 3;
  static constexpr int X_ROW = BK * 2 + 64;            // bytes of a token's float16 row: eight lanes that read 16 bytes of two rows hit all banks
  static constexpr int MAX_CLUSTER = 8;
  static constexpr int WARPS = 8;
  static constexpr int THREADS = 32 * (WARPS + 1);
  static constexpr int BAR_BYTES = 128;
  __host__ __device__ static constexpr int stage_bytes(bool gated) { return W_BYTES + (gated ? 2 : 1) * CH * 512; }
  __host__ __device__ static constexpr int x_bytes(int nt) { return 8 * nt * (X_ROW + 8); }     // values, and two scales per token
  // what arrives at the owner of 8 / S warps' rows: 16 bytes per lane and eight tokens from each of S CTAs
  __host__ __device__ static constexpr int recv_bytes(int nt, int S) { return S > 1 ? WARPS * 512 * nt : 0; }
  __host__ __device__ static constexpr int smem_bytes(int nt, bool gated, int S) {
    return 1024 + STAGES * stage_bytes(gated) + 2 * x_bytes(nt) + recv_bytes(nt, S) + BAR_BYTES;
  }
};

__device__ __forceinline__ void mma_16816_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
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
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      // nibble n of [-8, 8) -> bits of 1024 + (n + 8), minus 1032
      const uint32_t b = ((w >> (4 * i)) & 0x000F000Fu) ^ 0x64086408u;
      const __half2 v = __hsub2(*reinterpret_cast<const __half2*>(&b), __half2half2(__ushort_as_half(0x6408)));
      p[i] = *reinterpret_cast<const uint32_t*>(&v);
    }
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
// Byte j of a word of E8M0 scales as float32 (byte 0 is 2^-127, a subnormal).
template <int J>
__device__ __forceinline__ float e8m0_value(uint32_t word) {
  const uint32_t b = (J == 3 ? word >> 1 : word << (23 - 8 * J)) & 0x7F800000u;
  return __uint_as_float(b < 0x00400000u ? 0x00400000u : b);
}
__device__ __forceinline__ uint32_t hmul2_bits(uint32_t a, uint32_t b) {
  const __half2 v = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&v);
}

// grid = (row tiles * S in clusters of S along x, groups of 8 NT tokens).  tmW: Wq [rows, K / 2 bytes], box [64 x 128 B].
template <int FMT, int NT, bool GATED>
__global__ void __launch_bounds__(MatvecCfg<FMT>::THREADS, NT == 1 ? 3 : 2)
matvec_kernel(const __grid_constant__ CUtensorMap tmW, const __nv_bfloat16* __restrict__ X, const uint8_t* __restrict__ Ws,
              void* __restrict__ Y, int y_is_bf16, int M, int N, int K, int S, float alpha, int* err_word) {
  using C = MatvecCfg<FMT>;
  constexpr int CH = C::CH, STAGES = C::STAGES;
  constexpr int STAGE_BYTES = C::stage_bytes(GATED);
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t x_base = base + STAGES * STAGE_BYTES;
  const uint32_t recv_base = x_base + 2 * C::x_bytes(NT);
  const uint32_t bar_base = recv_base + C::recv_bytes(NT, S);
  auto full_bar = [&](int s) { return bar_base + 8u * s; };
  auto empty_bar = [&](int s) { return bar_base + 8u * (STAGES + s); };
  const uint32_t recv_bar = bar_base + 8u * (2 * STAGES);
  volatile int* cta_abort = reinterpret_cast<volatile int*>(smem_raw + (bar_base + 8u * (2 * STAGES + 1) - smem_u32(smem_raw)));

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x % S, tile = blockIdx.x / S;
  const int m0 = blockIdx.y * 8 * NT;
  const int mt = M - m0 < 8 * NT ? M - m0 : 8 * NT;      // tokens of this CTA
  const int k_tiles = (K + C::BK - 1) / C::BK;           // K % 128 == 0: the last stage may be half
  const int kb4 = K / (CH == 4 ? 64 : 128);              // scale chunks per row tile
  const int kt0 = (int)((long long)k_tiles * rank / S), kt1 = (int)((long long)k_tiles * (rank + 1) / S);
  const int n0 = tile * (GATED ? 64 : 128);
  const int row1 = GATED ? N + n0 : n0 + 64;             // first row of the second half of the tile

  auto fetch = [&](int it) {
    const int s = it % STAGES, kt = kt0 + it;
    const uint32_t st = base + s * STAGE_BYTES;
    const uint32_t sf = 512u * (uint32_t)min(CH, kb4 - CH * kt);
    mbar_arrive_expect_tx(full_bar(s), (uint32_t)C::W_BYTES + (GATED ? 2u : 1u) * sf);
    tma_load_2d(st, &tmW, kt * 128, n0, full_bar(s));
    tma_load_2d(st + C::W_BYTES / 2, &tmW, kt * 128, row1, full_bar(s));
    bulk_load_1d(st + C::W_BYTES, Ws + ((size_t)(n0 >> 7) * kb4 + CH * kt) * 512, sf, full_bar(s));
    if constexpr (GATED) bulk_load_1d(st + C::W_BYTES + CH * 512, Ws + ((size_t)(row1 >> 7) * kb4 + CH * kt) * 512, sf, full_bar(s));
  };
  // The weights are constants of the layer: their first stages are asked for before anything else.
  const int pre = kt1 - kt0 < STAGES ? kt1 - kt0 : STAGES;
  if (threadIdx.x == 32 * C::WARPS) {
    for (int s = 0; s < STAGES; ++s) { mbar_init(full_bar(s), 1); mbar_init(empty_bar(s), C::WARPS); }
    mbar_init(recv_bar, 1);
    *cta_abort = 0;
    fence_mbar_init();
    fence_proxy_async_smem();
    if (S > 1) mbar_arrive_expect_tx(recv_bar, (uint32_t)C::recv_bytes(NT, S));
    for (int it = 0; it < pre; ++it) fetch(it);
  }
  // tokens that there are not: zero, once
  for (int i = threadIdx.x; i < (8 * NT - mt) * ((C::X_ROW + 8) / 4) * 2; i += C::THREADS) {
    constexpr int words = (C::X_ROW + 8) / 4;            // of one token: its values and its two scales
    const int b = i / ((8 * NT - mt) * words), j = i % ((8 * NT - mt) * words), m = mt + j / words, o = j % words;
    const uint32_t xb = x_base + b * C::x_bytes(NT);
    const uint32_t a = o < C::X_ROW / 4 ? xb + m * C::X_ROW + 4 * o : xb + 8 * NT * C::X_ROW + (o - C::X_ROW / 4) * 32 * NT + 4 * m;
    asm volatile("st.shared.b32 [%0], %1;" ::"r"(a), "r"(0) : "memory");
  }
  __syncthreads();
  if (S > 1) cluster_arrive_relaxed();                   // the wait stands before the first access to another CTA
  griddep_launch_dependents();
  griddep_wait();

  if (warp == C::WARPS) {
    for (int it = pre; it < kt1 - kt0; ++it) {
      if (!mbar_wait_warp(empty_bar(it % STAGES), ((it / STAGES) & 1) ^ 1, cta_abort, err_word, SITE_PRODUCER_EMPTY)) break;
      if (elect_one()) fetch(it);
      __syncwarp();
    }
    if (S > 1) cluster_wait();
  } else {
    const int g = lane >> 2, t = lane & 3;
    // x of one stage: a warp has 256 elements of a token, a lane eight (16 bytes)
    uint4 xr[NT];
    auto x_load = [&](int it) {
      const int k = (kt0 + it) * C::BK + 8 * lane;
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int m = 8 * j + warp;
        xr[j] = m < mt && k < K ? __ldg(reinterpret_cast<const uint4*>(X + (int64_t)(m0 + m) * K + k)) : make_uint4(0, 0, 0, 0);
      }
    };
    auto x_store = [&](int it) {
      const uint32_t xb = x_base + (it & 1) * C::x_bytes(NT);
#pragma unroll
      for (int j = 0; j < NT; ++j) {
        const int m = 8 * j + warp;
        if (m < mt) {                                    // the same for the whole warp
          const uint32_t w[4] = {xr[j].x, xr[j].y, xr[j].z, xr[j].w};
          float v[8];
          float amax = 0.f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
            amax = fmaxf(amax, fmaxf(fabsf(v[2 * i]), fabsf(v[2 * i + 1])));
          }
#pragma unroll
          for (int o = 1; o < 16; o <<= 1) amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, o));
          // 2^14 / 2^floor(log2 amax), at most 2^126: exponent field 127 + 14 - (ef - 127)
          const uint32_t ef = __float_as_uint(amax) >> 23;
          const uint32_t fe = ef > 15u ? 268u - ef : 253u;
          const float f = __uint_as_float(fe << 23);
          uint32_t o4[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float a = FMT == FMT_MXINT4 ? v[i] : v[2 * i], b = FMT == FMT_MXINT4 ? v[i + 4] : v[2 * i + 1];
            const __half2 h = __floats2half2_rn(a * f, b * f);
            o4[i] = *reinterpret_cast<const uint32_t*>(&h);
          }
          asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(xb + m * C::X_ROW + 16 * lane), "r"(o4[0]), "r"(o4[1]), "r"(o4[2]),
                       "r"(o4[3]) : "memory");
          if ((lane & 15) == 0)
            asm volatile("st.shared.b32 [%0], %1;" ::"r"(xb + 8 * NT * C::X_ROW + (lane >> 4) * 32 * NT + 4 * m), "r"((254u - fe) << 23) : "memory");
        }
      }
    };
    // this lane's rows g and g + 8 of the warp's instruction, as rows of the stage
    const int r0 = GATED ? 8 * warp + g : 16 * warp + g;
    constexpr int R1 = GATED ? 64 : 8;                   // from the first to the second
    const uint32_t w_off = (uint32_t)(r0 * 128 + (g << 4) + 4 * t);
    // their scale bytes; the halves of a gated tile start at row 0 or 64 of a scale tile
    auto sf_cell = [](int r) { return (uint32_t)((r & 31) * 16 + ((r & 127) >> 5) * 4); };
    const uint32_t sf0 = C::W_BYTES + sf_cell((GATED ? (n0 & 64) : 0) + r0);
    const uint32_t sf1 = GATED ? C::W_BYTES + CH * 512 + sf_cell((row1 & 64) + r0) : C::W_BYTES + sf_cell(r0 + 8);
    const uint32_t sel = (uint32_t)((t >> 1) * 0x11);    // NVFP4: words 0, 1 of a 32 are its first block of 16

    float acc[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[j][i] = 0.f;

    const int steps = kt1 - kt0;
    x_load(0);
    x_store(0);
    bool ok = true;
    for (int it = 0; it < steps; ++it) {
      if (it + 1 < steps) x_load(it + 1);
      named_barrier_sync(1, 32 * C::WARPS);              // x of this stage is there, and that of the stage before has been read
      const int s = it % STAGES;
      ok = ok && mbar_wait_warp(full_bar(s), (it / STAGES) & 1, cta_abort, err_word, SITE_MMA_FULL);
      if (ok) {
        const uint32_t st = base + s * STAGE_BYTES;
        const uint32_t xb = x_base + (it & 1) * C::x_bytes(NT);
        const uint32_t xa = xb + g * C::X_ROW + 16 * t;
#pragma unroll
        for (int q = 0; q < 2; ++q) {                    // 128 of K
          if (q == 1 && (kt0 + it) * C::BK + 128 >= K) break;
          uint32_t sw0[2], sw1[2];
          sw0[0] = lds32(st + sf0 + (CH / 2 * q) * 512);
          sw1[0] = lds32(st + sf1 + (CH / 2 * q) * 512);
          if constexpr (FMT == FMT_NVFP4) {
            sw0[1] = lds32(st + sf0 + (2 * q + 1) * 512);
            sw1[1] = lds32(st + sf1 + (2 * q + 1) * 512);
          }
          float part[NT][4];
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) part[j][i] = 0.f;
          auto block = [&](auto block_of) {
            constexpr int B = decltype(block_of)::value;
            const uint32_t a = (st + w_off) ^ (uint32_t)((4 * q + B) << 4);
            uint32_t a0[4], a1[4];
            widen8<FMT>(lds32(a), a0);
            widen8<FMT>(lds32(a + R1 * 128), a1);
            if constexpr (FMT == FMT_NVFP4) {
              const uint32_t f0 = e4m3_pair(sw0[B >> 1], sel + (B & 1) * 0x22u), f1 = e4m3_pair(sw1[B >> 1], sel + (B & 1) * 0x22u);
#pragma unroll
              for (int i = 0; i < 4; ++i) { a0[i] = hmul2_bits(a0[i], f0); a1[i] = hmul2_bits(a1[i], f1); }
            }
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              const uint4 x = lds128(xa + 8 * j * C::X_ROW + (4 * q + B) * 64);
              if constexpr (FMT == FMT_NVFP4) {
                mma_16816_f16(part[j], a0[0], a1[0], a0[1], a1[1], x.x, x.y);
                mma_16816_f16(part[j], a0[2], a1[2], a0[3], a1[3], x.z, x.w);
              } else {
                float c[4] = {0.f, 0.f, 0.f, 0.f};
                mma_16816_f16(c, a0[0], a1[0], a0[1], a1[1], x.x, x.y);
                mma_16816_f16(c, a0[2], a1[2], a0[3], a1[3], x.z, x.w);
                const float f0 = e8m0_value<B>(sw0[0]), f1 = e8m0_value<B>(sw1[0]);
                part[j][0] = fmaf(c[0], f0, part[j][0]);
                part[j][1] = fmaf(c[1], f0, part[j][1]);
                part[j][2] = fmaf(c[2], f1, part[j][2]);
                part[j][3] = fmaf(c[3], f1, part[j][3]);
              }
            }
          };
          block(std::integral_constant<int, 0>{});
          block(std::integral_constant<int, 1>{});
          block(std::integral_constant<int, 2>{});
          block(std::integral_constant<int, 3>{});
#pragma unroll
          for (int j = 0; j < NT; ++j) {                 // x's power of two: tokens 2 t and 2 t + 1
            uint32_t f0, f1;
            asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(f0), "=r"(f1) : "r"(xb + 8 * NT * C::X_ROW + q * 32 * NT + 4 * (8 * j + 2 * t)));
            acc[j][0] = fmaf(part[j][0], __uint_as_float(f0), acc[j][0]);
            acc[j][1] = fmaf(part[j][1], __uint_as_float(f1), acc[j][1]);
            acc[j][2] = fmaf(part[j][2], __uint_as_float(f0), acc[j][2]);
            acc[j][3] = fmaf(part[j][3], __uint_as_float(f1), acc[j][3]);
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(empty_bar(s));
      if (it + 1 < steps) x_store(it + 1);
    }

    // sums of one warp's 16 rows: lane (g, t) has rows g, g + 8 of tokens 8 j + 2 t, 2 t + 1
    auto finish = [&](int w, const float (&v)[NT][4]) {
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int m = 8 * j + 2 * t + e;
          if (m < mt) {
            auto put = [&](int n, float y) {
              if (n < N) {
                const int64_t o = (int64_t)(m0 + m) * N + n;
                if (y_is_bf16) static_cast<__nv_bfloat16*>(Y)[o] = __float2bfloat16_rn(y);
                else static_cast<float*>(Y)[o] = y;
              }
            };
            if constexpr (GATED) {
              put(n0 + 8 * w + g, silu(v[j][e] * alpha) * (v[j][2 + e] * alpha));
            } else {
              put(n0 + 16 * w + g, v[j][e] * alpha);
              put(n0 + 16 * w + 8 + g, v[j][2 + e] * alpha);
            }
          }
        }
    };
    if (S == 1) {
      if (ok) finish(warp, acc);
    } else {
      // CTA r owns the rows of warps r 8 / S ... : [warp of these][source CTA][eight tokens][lane] 16 bytes
      const int per = C::WARPS / S, owner = warp / per, slot = warp - owner * per;
      const uint32_t dst = map_to_cta(recv_base + (uint32_t)((slot * S + rank) * NT * 512 + lane * 16), (uint32_t)owner);
      const uint32_t dst_bar = map_to_cta(recv_bar, (uint32_t)owner);
      cluster_wait();
#pragma unroll
      for (int j = 0; j < NT; ++j)
        st_async_v4(dst + j * 512, __float_as_uint(acc[j][0]), __float_as_uint(acc[j][1]), __float_as_uint(acc[j][2]), __float_as_uint(acc[j][3]), dst_bar);
      if (warp < per) {
        ok = __all_sync(0xFFFFFFFFu, mbar_wait_cluster(recv_bar, 0, cta_abort, err_word, SITE_EPI_ACC_FULL));
        if (ok) {
          float sum[NT][4];
#pragma unroll
          for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[j][i] = 0.f;
          for (int r = 0; r < S; ++r)                    // rank order: the result does not depend on timing
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              const uint4 p = lds128(recv_base + (uint32_t)(((warp * S + r) * NT + j) * 512 + lane * 16));
              sum[j][0] += __uint_as_float(p.x); sum[j][1] += __uint_as_float(p.y);
              sum[j][2] += __uint_as_float(p.z); sum[j][3] += __uint_as_float(p.w);
            }
          finish(rank * per + warp, sum);
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
