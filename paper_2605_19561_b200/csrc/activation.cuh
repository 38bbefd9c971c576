// The activation of the gated projections, shared by the product of few tokens and the GEMM's epilogue.
#pragma once
#include <cuda_runtime.h>

namespace torq {

// g / (1 + exp(-g)), off by a few units in the last place of float32 for every finite g from -87.3 on; below, where it lies between -1.1e-36
// and 0, it is -0 (1 + exp(-g) passes 2^126, whose reciprocal the hardware's instruction flushes, and from -88.7 on float32).
// exp(-g) = 2^t with t = -g log2(e) in two parts: the rounded product and what the rounding left (an error-free product by fused multiply-add,
// Dekker 1971), so that far from zero, where t has few bits behind the point, nothing is lost; 2^hi and 1 / x are the hardware's approximations
// (2^-22 and 2^-23).  The rest is held as rest + 1/2 in [0, 1] by the addition's own saturation: it is no more than 2^-17 wherever 2^hi is neither
// 0 nor infinite, and beyond, where hi overflows (|g| > 2.36e38) or g is not finite, it only has to be a number.
// With expf and a division the GEMM's epilogue took 4.9 us per 256 x 256 tile and was what the kernel waited for (8192 x 1024 -> 8192 142 us, the
// plain GEMM of both projections 72).  exp(-|g|) and a choice by sign, which has results down to the smallest number, makes short contractions wait
// for the epilogue (4096 x 256 -> 14336 52 / 65 us, 8192 x 1024 -> 8192 67 / 78); powers of two shifted by 2^24 for the same end cost 2 %.
__device__ __forceinline__ float silu(float g) {
  constexpr float kLog2e = 1.44269502f, kRest = 1.92596303e-8f, kLn2 = 0.693147181f;   // kLog2e + kRest = log2(e) to 2^-50
  const float hi = -g * kLog2e;
  const float lo = __saturatef(fmaf(-g, kLog2e, -hi) + fmaf(-g, kRest, 0.5f));   // what is not a number becomes 0
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(e) : "f"(hi));
  e *= fmaf(lo, kLn2, 1.0f - 0.5f * kLn2);               // 2^(lo - 1/2) for |lo - 1/2| < 2^-17
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.0f + e));
  return g * r;
}

}  // namespace torq
