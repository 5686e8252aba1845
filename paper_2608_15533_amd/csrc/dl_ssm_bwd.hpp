// The scan's backward kernels, launched from dl_ssm.hip.
#pragma once

#include "dl_ssm.hpp"

namespace dl {

// Tokens of a stretch of the backward pass.  Longer ones have fewer states to join, shorter ones leave LDS for
// more workgroups on a CU.  4096 tokens, 4096 x 16, 2048 x 32 and 1024 x 64 channels x states, whole step: 16
// states with 64, 40, 32, 24 tokens 618, 623, 549, 571 us (in tiles of 8); 32 states with 64 (in tiles of 8), 24
// (in tiles of 4), 20 600, 553, 563; 64 states with 28, 24, 20, 16 677, 664, 675, 696.
__host__ __device__ constexpr int ssm_grad_tokens(int states) { return states == 16 ? 32 : 24; }

// Workgroups of 256 that sum dB and dC of a stretch.
__host__ __device__ constexpr int ssm_rows_pieces(int states) { return ssm_grad_tokens(states) * 2 * states / 256; }

// E, F and the sum of d of every stretch.
hipError_t launch_ssm_ends(int states, bool bf16, const SsmParams& p, hipStream_t s);
// Every gradient, from the states before and the gradients behind every stretch; dA, dskip and dbias
// as partial sums in p.part.
hipError_t launch_ssm_grad(int states, bool bf16, const SsmParams& p, hipStream_t s);

}  // namespace dl
