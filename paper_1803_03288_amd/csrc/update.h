// The update of parameters and the norm of their gradients (k10_update.hip): many tensors in one launch, their descriptions among the kernel's arguments.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "tictac.h"

namespace tictac {

hipError_t launch_gradient_norm(int32_t n, const tictac_gradient *g, float scale, float *norm, double *workspace, hipStream_t s);
size_t gradient_norm_workspace(int32_t n);
hipError_t launch_adamw_step(int32_t n, const tictac_adamw_tensor *t, const tictac_adamw_options &o, hipStream_t s);

}  // namespace tictac
