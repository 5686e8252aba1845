// The scan's backward kernels, launched from dl_ssm.hip.
#pragma once

#include "dl_ssm.hpp"

namespace dl {

// Tokens of a stretch of the backward pass: the states before its tiles fit LDS.
__host__ __device__ constexpr int ssm_grad_tokens(int states) { return states == 32 ? 64 : states == 16 ? 32 : 16; }

// E, F and the sum of d of every stretch.
hipError_t launch_ssm_ends(int states, bool bf16, const SsmParams& p, hipStream_t s);
// Every gradient, from the states before and the gradients behind every stretch; dA, dskip and dbias
// as partial sums in p.part.
hipError_t launch_ssm_grad(int states, bool bf16, const SsmParams& p, hipStream_t s);

}  // namespace dl
