// The scan's backward kernels, launched from dl_ssm.hip.
#pragma once

#include "dl_ssm.hpp"

namespace dl {

// Tokens whose steps lie in LDS at a time, and whose decays and states a wave holds in registers: 8 with 150
// registers a lane, three waves to a SIMD (16 take 255), or 4 with 110 where a workgroup has 8 or 16 waves.
// A stretch of the backward pass is a whole number of tiles.
__host__ __device__ constexpr int ssm_grad_tile(int states) { return states == 16 ? 8 : 4; }

// E, F and the sum of d of every stretch, and the starts of its tiles.
hipError_t launch_ssm_ends(int states, bool bf16, const SsmParams& p, hipStream_t s);
// Every gradient, from the states before and the gradients behind every stretch; dA, dskip and dbias
// as partial sums in p.part.
hipError_t launch_ssm_grad(int states, bool bf16, const SsmParams& p, hipStream_t s);

}  // namespace dl
