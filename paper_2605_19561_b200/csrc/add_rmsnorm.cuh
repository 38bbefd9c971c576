// Root-mean-square norm with the residual's addition, the step in front of a linear layer:
//   h = x + r                                  float32; stored to the residual stream in r's type
//   y = h / sqrt(mean(h^2) + eps) * w          float32; rounded once to bfloat16, or quantized to MXFP8
// MXFP8: per 32 elements e = clamp(floor(log2 amax) - 8, -127, ...), byte e + 127, code = E4M3(y / 2^e) to nearest even,
// saturating at 448 (the OCP rule with E4M3's largest exponent, 8; amax / 2^e lies in [256, 512)).  The scale bytes go to the
// library's tiled layout: the result is the activation operand of the kind::mxf8f6f4 GEMM.
#pragma once
#include <cuda_bf16.h>
#include "mxint4_quantize.cuh"
#include "quantize.cuh"
#include "sm100_ptx.cuh"

namespace torq {

enum : int { RES_NONE = 0, RES_BF16 = 1, RES_F32 = 2 };

// Eight bfloat16 <-> four pairs of float32.
__device__ __forceinline__ void bf16x8_to_pairs(const uint4& a, uint64_t (&v)[4]) {
  const uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = pair_of(w[i] << 16, w[i] & 0xFFFF0000u);
}
__device__ __forceinline__ uint4 pairs_to_bf16x8(const uint64_t (&v)[4]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = halves(v[i]);
    const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// Eight elements as they lie in memory, bfloat16 or float32.
template <bool F32>
struct Raw8 {
  uint4 v[F32 ? 2 : 1];
  __device__ __forceinline__ void load(const void* p, int64_t i) {
    const char* at = static_cast<const char*>(p) + i * (F32 ? 4 : 2);
    v[0] = load_once(at);
    if constexpr (F32) v[1] = load_once(at + 16);
  }
  __device__ __forceinline__ void zero() {
    v[0] = make_uint4(0, 0, 0, 0);
    if constexpr (F32) v[1] = v[0];
  }
  __device__ __forceinline__ void values(uint64_t (&f)[4]) const {
    if constexpr (F32) {
      f[0] = pair_of(v[0].x, v[0].y); f[1] = pair_of(v[0].z, v[0].w);
      f[2] = pair_of(v[1].x, v[1].y); f[3] = pair_of(v[1].z, v[1].w);
    } else {
      bf16x8_to_pairs(v[0], f);
    }
  }
};

// One row per blockDim.x threads (blockDim.y rows per CTA, more than one only when a row is one warp's), a thread holds VPT
// pieces of eight elements, blockDim.x pieces apart, in registers: one pass over memory.  CTAs walk the rows; the loads of the next
// row go out before the sum of this one is taken, so that they are under way throughout (8192 x 5120, all bfloat16, MXFP8 out: 83 us
// without, 54 with; 295 MB: 5.5 TB/s of the 6.5 that a copy reaches).  What is left: a row's loads are under
// way while another's sum and scales are worked out, 55 % of the DRAM cycles, and scale bytes that go out four at a time, 512 bytes apart
// (1.5 us of the 53).  rows = M, or with scales M rounded up to 128: the rows behind the last one only get their zero scale bytes.
template <int VPT, bool MX, bool XF32, int RES>
__global__ void __launch_bounds__(VPT == 1 ? 1024 : 512)
add_rmsnorm_kernel(const void* X, const void* R, void* R_out, const __nv_bfloat16* __restrict__ weight, float eps, int64_t M, int64_t rows, int d,
                   void* out, uint8_t* __restrict__ scales) {
  __shared__ float part[2][32];
  const int tid = threadIdx.x, nt = blockDim.x, lane = tid & 31;
  const int pieces = d / 8;
  // The products behind it read their weights ahead of their wait, and this may be the only kernel between them and what wrote the weights.
  // (us, blocks of norm, gated pair and product in a graph, released ahead of the wait / behind it: MXFP4, 1 token 1024 -> 2816 8.27 / 8.57, 4096 ->
  // 14336 21.5 / 21.7, 8 tokens 10.6 / 10.45 and 28.5 / 29.2; NVFP4 9.0 / 8.6, 23.5 / 23.5, 11.9 / 11.5 and 32.7 / 32.5; alone the norm is the same.)
  griddep_wait_and_launch();
  Raw8<XF32> x[VPT];
  Raw8<RES == RES_F32> r[VPT];
  auto load = [&](int64_t row) {
    const int64_t base = row * d;
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
      const int p = tid + k * nt;
      if (p < pieces) {
        x[k].load(X, base + 8 * p);
        if constexpr (RES != RES_NONE) r[k].load(R, base + 8 * p);
      } else {
        x[k].zero();
        if constexpr (RES != RES_NONE) r[k].zero();
      }
    }
  };
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  int64_t row = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  if (row < M) load(row);
  uint4 w[VPT];
#pragma unroll
  for (int k = 0; k < VPT; ++k) {
    const int p = tid + k * nt;
    w[k] = p < pieces ? load_once(reinterpret_cast<const uint4*>(weight) + p) : make_uint4(0, 0, 0, 0);
  }
  const int kb4 = (d / 32 + 3) / 4;
  int turn = 0;
  for (; row < rows; row += step) {
    if (MX && row >= M) {                                // all threads of a row agree
      for (int c = tid; c < kb4; c += nt)
        *reinterpret_cast<uint32_t*>(scales + scale_offset(row, 4 * c, kb4)) = 0u;
      continue;
    }
    const int64_t base = row * d;
    uint64_t h[VPT][4], squares = 0;
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
      x[k].values(h[k]);
      if constexpr (RES != RES_NONE) {
        uint64_t a[4];
        r[k].values(a);
#pragma unroll
        for (int i = 0; i < 4; ++i) h[k][i] = add2(h[k][i], a[i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) squares = fma2(h[k][i], h[k][i], squares);
    }
    float sum = halves(squares).x + halves(squares).y;
    if (row + step < M) load(row + step);
    if constexpr (RES != RES_NONE) {
#pragma unroll
      for (int k = 0; k < VPT; ++k) {
        const int p = tid + k * nt;
        if (p < pieces) {
          if constexpr (RES == RES_F32) {
            ulonglong2* o = reinterpret_cast<ulonglong2*>(static_cast<float*>(R_out) + base + 8 * p);
            o[0] = make_ulonglong2(h[k][0], h[k][1]);
            o[1] = make_ulonglong2(h[k][2], h[k][3]);
          } else {
            *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(R_out) + base + 8 * p) = pairs_to_bf16x8(h[k]);
          }
        }
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
    if (nt > 32) {                                       // the two buffers in turn: one barrier per row
      if (lane == 0) part[turn][tid >> 5] = sum;
      __syncthreads();
      sum = lane < (nt >> 5) ? part[turn][lane] : 0.f;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, o);
      turn ^= 1;
    }
    const uint64_t rstd = pair_of(1.0f / sqrtf(sum / (float)d + eps));
#pragma unroll
    for (int k = 0; k < VPT; ++k) {
      const int p = tid + k * nt;
      uint64_t y[4];
      bf16x8_to_pairs(w[k], y);
#pragma unroll
      for (int i = 0; i < 4; ++i) y[i] = mul2(mul2(h[k][i], rstd), y[i]);
      if constexpr (!MX) {
        if (p < pieces) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(out) + base + 8 * p) = pairs_to_bf16x8(y);
      } else {
        // four lanes share a block of 32, sixteen a word of four scale bytes
        float amax = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) amax = fmaxf(amax, fmaxf(fabsf(halves(y[i]).x), fabsf(halves(y[i]).y)));
        amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 1));
        amax = fmaxf(amax, __shfl_xor_sync(0xFFFFFFFFu, amax, 2));
        const uint32_t ef = __float_as_uint(amax) >> 23, sbyte = ef > 8u ? ef - 8u : 0u;
        const uint64_t inv = pair_of((254u - sbyte) << 23, (254u - sbyte) << 23);
        if (p < pieces) {
          float2 q[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) q[i] = halves(mul2(y[i], inv));
          *reinterpret_cast<uint2*>(static_cast<uint8_t*>(out) + base + 8 * p) =
              make_uint2(pack4_e4m3(q[0].x, q[0].y, q[1].x, q[1].y), pack4_e4m3(q[2].x, q[2].y, q[3].x, q[3].y));
        }
        uint32_t word = sbyte << (8 * ((lane >> 2) & 3));
        word |= __shfl_xor_sync(0xFFFFFFFFu, word, 4);
        word |= __shfl_xor_sync(0xFFFFFFFFu, word, 8);
        if ((lane & 15) == 0 && p < 16 * kb4) *reinterpret_cast<uint32_t*>(scales + scale_offset(row, p / 4, kb4)) = word;
      }
    }
  }
}

}  // namespace torq
