// The many-row kernel of dsp_attn_kv4, launched from attn.cu.
#pragma once

#include "attn.cuh"

namespace dsp {

// Bytes of one partial result (a CTA leaves at most two).
size_t attn_block_part_bytes(int D);
// Enqueues the kernel on `grid` CTAs (one per SM) and the join of what they left.
cudaError_t attn_block_launch(const AttnArgs &a, int D, int grid, cudaStream_t st);

}  // namespace dsp
