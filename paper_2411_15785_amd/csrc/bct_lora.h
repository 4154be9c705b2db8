// The host side of the low-rank adapters: argument checks and the launch of their first half.
#ifndef BCT_LORA_H
#define BCT_LORA_H

#include "../../include/bct_model.h"
#include "bct_linear.h"

namespace bct {

// The checks of a call's adapters; segments: outputs (or SwiGLU matrices) with an A of their own.
bct_status check_lora(const bctm_lora* lora, uint32_t rows, uint32_t K, uint32_t N, uint32_t segments, bool swiglu);
// Enqueues t = scale * x A^T into the workspace, as operands of the matrix-core kernel or for the streaming one, and fills in the
// term that the projection's launch takes.
bct_status launch_lora_inputs(const bctm_lora& lora, const void* x, uint32_t rows, uint32_t K, bool x_tiled, uint32_t segments,
                              bool operands, hipStream_t s, LoraTerm* term);

}  // namespace bct

#endif
