// The operators around the experts as the layer's own calls run them: with the layer's choice of dependent launches and its counter.
#pragma once
#include "../../include/swapmoe.h"

namespace swapmoe {

// swapmoe_rms_norm and swapmoe_adapters_forward; pdl: programmatic dependent launch; *launches grows by the kernels that were launched.
int32_t rms_norm_run(const swapmoe_rms_norm_t* p, void* stream, bool pdl, int64_t* launches);
int32_t adapters_run(swapmoe_adapters_t* b, const void* x, int64_t x_stride, const float* x_scales, const int32_t* ids, const void* y,
                     int64_t y_stride, void* out, int64_t out_stride, int32_t T, void* stream, bool pdl, int64_t* launches);

}  // namespace swapmoe
