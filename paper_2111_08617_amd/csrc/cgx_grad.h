// Launchers of the gradient norm and clipping (cgx_grad.hip); arguments are checked by the caller.
#pragma once

#include <hip/hip_runtime.h>

#include "../../include/cgx.h"

namespace cgx {

constexpr int kNormSlots = 2048;                     // blocks of the norm kernel, each with a partial sum in the workspace

hipError_t launch_grad_norm(const cgx_tensor *tensors, int32_t count, float *norm, double *partial, hipStream_t stream);
hipError_t launch_grad_clip(const cgx_tensor *tensors, int32_t count, const float *norm, float max_norm, void *out, int out_dt,
                            hipStream_t stream);

}  // namespace cgx
