// The short causal convolution (short_conv.hip): what the entry points launch.
#pragma once
#include <hip/hip_runtime.h>

#include "scan_places.h"
#include "wkv6_launch.h"

namespace wkv6 {

constexpr int kConvGroup = 4, kConvStepGroup = 8;    // channels of a thread (prompts and gradients; single tokens)
constexpr int kConvThreads = 256;

struct ConvArgs {
    int B, T, D, W;
    long long rows;
    const void* x;
    long long x_row;                   // bytes from token to token
    const float *w, *bias;             // bias may be null
    bool silu;
    const int* offsets;
    const void* state_in;              // null: zeros
    int segs, seg_len;                 // tokens of a sequence that a workgroup takes
    int lanes;                         // threads side by side over a row's groups: a power of two up to kConvThreads; the others lie over tokens
};

// How a call's tokens and channels are divided; backward: with the sums over tokens.
struct ConvPlan {
    int segs, seg_len, lanes;
    long long workgroups;
};
ConvPlan plan_conv(int B, int T, int D, long long rows, bool backward);

hipError_t launch_conv(const ConvArgs& a, void* out, void* state_out, bool f32, hipStream_t stream);
hipError_t launch_conv_step(const ConvArgs& a, void* out, void* state_out, bool f32, hipStream_t stream);

// dw and dbias (both or neither) through `partials`: segments' sums [place][W + 1][D], of packed sequences by row (whole_places).
inline long long conv_partial_floats(int B, int D, int W, long long rows, const ConvPlan& p, bool packed) {
    return share_places(B, rows, p.segs, p.seg_len, packed) * (W + 1) * D;
}
hipError_t launch_conv_backward(const ConvArgs& a, const void* dout, const void* dstate_out, void* dx, float* dw, float* dbias, void* dstate_in,
                                float* partials, bool f32, hipStream_t stream);

hipError_t launch_conv_fold(const ConvArgs& a, float* dw, float* dbias, const float* partials, hipStream_t stream);

}  // namespace wkv6
