// The activation of the gated projections, shared by the product of few tokens and the GEMM's epilogue.
#pragma once
#include <cuda_runtime.h>

namespace torq {

// g / (1 + exp(-g)): for g far below zero exp overflows to infinity and the quotient is -0, its limit.
__device__ __forceinline__ float silu(float g) { return g / (1.0f + expf(-g)); }

}  // namespace torq
