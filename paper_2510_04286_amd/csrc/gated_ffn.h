// Gated feed-forward network (gated_ffn.hip): the plan of a call and the launchers.
#pragma once
#include "common.h"

namespace slicemoe {

// What a call lays out in its workspace, in bytes from its start.  Operands that the tiles cannot read as they are (fp32, or rows
// that are not whole 16-byte pieces) get a copy: `terms` arrays of bf16 with padded rows.
struct GatedPlan {
    int terms;                              // bf16 terms of a product's operands: 1 for bf16 storage, 3 for fp32
    size_t x, dy, Wg, Wu, Wd;               // copies (0 bytes apart where none is made)
    bool copy_x, copy_h;                    // rows of d / of H are copied
    int ldd, ldh;                           // elements per row of d / H in the copies and in the hidden arrays
    size_t a, dg, du;                       // [terms][T][ldh]
    size_t part;                            // partial sums of split contractions
    bool few_f32;                           // fp32 rows few enough to multiply as they are: nothing but fp32 hidden rows and part
    size_t total;
};
GatedPlan gated_plan(const slicemoe_gated_config &c, bool backward, bool quantized);
hipError_t launch_gated_ffn(const slicemoe_gated_config &c, const GatedPlan &plan, const void *x, const slicemoe_gated_weights &w,
                            const void *addend, void *y, char *ws, hipStream_t s);
hipError_t launch_gated_ffn_quantized(const slicemoe_gated_config &c, const GatedPlan &plan, const uint8_t *x, const float *x_scale,
                                      const slicemoe_gated_weights_quantized &w, const void *addend, void *y, char *ws, hipStream_t s);
hipError_t launch_gated_ffn_backward(const slicemoe_gated_config &c, const GatedPlan &plan, const void *x, const slicemoe_gated_weights &w,
                                     const void *dy, const void *addend, void *dx, const slicemoe_gated_weight_grads &g, char *ws,
                                     hipStream_t s);
hipError_t launch_gated_quantize_weights(const slicemoe_gated_config &c, const slicemoe_gated_weights &w, uint8_t *Wg, float *Wg_scale,
                                         uint8_t *Wu, float *Wu_scale, hipStream_t s);

}  // namespace slicemoe
