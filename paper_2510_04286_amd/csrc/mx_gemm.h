// Products of microscaled matrices and the gated network on them (mx_gemm.hip), conversions (mx.hip): launchers.
#pragma once
#include "common.h"

namespace slicemoe {

hipError_t launch_mx_quantize(const slicemoe_mx_config &c, const void *x, uint8_t *mx, hipStream_t s);
hipError_t launch_mx_dequantize(const slicemoe_mx_config &c, const uint8_t *mx, void *x, hipStream_t s);

size_t mx_product_workspace(const slicemoe_mx_product_config &c);
hipError_t launch_mx_product(const slicemoe_mx_product_config &c, const uint8_t *x, const uint8_t *w, const void *addend, void *y, char *ws, hipStream_t s);
size_t gated_mx_workspace(const slicemoe_gated_config &c, int bits);
hipError_t launch_gated_mx(const slicemoe_gated_config &c, int bits, const uint8_t *x, const slicemoe_gated_weights_mx &w, const void *addend, void *y,
                           char *ws, hipStream_t s);

}  // namespace slicemoe
