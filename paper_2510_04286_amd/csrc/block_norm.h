// Norms on both sides of a block's addition to the residual stream (block_norm.hip): launchers.
#pragma once
#include "common.h"

namespace slicemoe {

int block_norm_backward_blocks(const slicemoe_block_norm_config &c);
hipError_t launch_block_norm(const slicemoe_block_norm_config &c, const void *x, const void *post, const void *gate, const void *residual,
                             const void *pre, void *sum, void *y, uint8_t *mx, int bits, float *stats, hipStream_t s);
hipError_t launch_block_norm_backward(const slicemoe_block_norm_config &c, const void *x, const void *post, const void *gate, const void *sum,
                                      const void *pre, const float *stats, const void *dy, const void *dsum, void *dx, void *dres,
                                      float *dpost, void *dgate, float *dpre, float *part, hipStream_t s);

}  // namespace slicemoe
