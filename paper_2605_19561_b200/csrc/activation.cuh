// The activation of the gated projections, shared by the product of few tokens and the GEMM's epilogue.
#pragma once
#include <cuda_runtime.h>

namespace torq {

// g / (1 + exp(-g)), off by a few units in the last place of float32.  exp(-g) = 2^t with t = -g log2(e) in two parts: the rounded product
// and what the rounding left (an error-free product by fused multiply-add, Dekker 1971), so that far from zero, where t has few
// bits behind the point, nothing is lost; 2^hi and 1 / x are the hardware's approximations (2^-22 and 2^-23).  For g far below zero 2^hi
// is infinite and the quotient -0, its limit.  With expf and a division the GEMM's epilogue took 4.9 us per 256 x 256 tile and was what
// the kernel waited for (8192 x 1024 -> 8192 142 us, the plain GEMM of both projections 72).
__device__ __forceinline__ float silu(float g) {
  constexpr float kLog2e = 1.44269502f, kRest = 1.92596303e-8f, kLn2 = 0.693147181f;   // kLog2e + kRest = log2(e) to 2^-50
  const float hi = -g * kLog2e;
  float lo = fmaf(-g, kRest, fmaf(-g, kLog2e, -hi));
  lo = fmaxf(lo, -1.0f);                                 // g not finite
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(hi));
  e *= fmaf(lo, kLn2, 1.0f);                             // 2^lo for |lo| < 2^-17
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  return g * r;
}

}  // namespace torq
