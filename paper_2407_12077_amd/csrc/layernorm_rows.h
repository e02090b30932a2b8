// LayerNorm over whole rows and its gradients (layernorm_rows.hip): what the entry points launch.
#pragma once
#include <hip/hip_runtime.h>

namespace wkv6 {

constexpr int kNormMaxWidth = 16384;

// y = (x - mean) rstd gamma + beta; stats [M][2] (mean, rstd) may be null
hipError_t launch_norm(long long M, int D, const void* x, const float* gamma, const float* beta, float eps, void* y, float* stats, bool x_f32,
                       bool y_f32, hipStream_t stream);

// Rows of partial sums, 2 D floats each, that launch_norm_backward leaves in its workspace; bf16: x and dy both.
int norm_partials(long long M, int D, bool bf16);

// dx, and with dgamma and dbeta (both or neither) their sums over the rows through `partials`
hipError_t launch_norm_backward(long long M, int D, const void* x, const float* stats, const float* gamma, const void* dy, void* dx,
                                float* dgamma, float* dbeta, float* partials, bool x_f32, bool y_f32, hipStream_t stream);

}  // namespace wkv6
