// The selective scan for one token of every sequence: h = exp(dt a) h_in + dt x b,  out = (sum_n c[n] h[n] + skip x) silu(z).
//
// Bound by the states, which are read and written once, past the caches: 1024 x 4096 channels of 16 states 106 us, 5.4 TB/s (a large copy: 5.2).  A lane has
// four states, so a load takes whole lines; what the lanes of a channel have in common each forms for itself.  One sequence: 3 us, a launch.
#include "selective_scan_tiles.h"

namespace wkv6 {
namespace {

using namespace scan;

// N / 4 lanes a channel, four states each.
template <int N, bool kF32, bool kOutF32>
__global__ __launch_bounds__(256) void scan_step_kernel(ScanArgs a, void* out, float* state_out, int across) {
    constexpr int kLanes = N / 4, kItem = kF32 ? 4 : 2;
    const int b = blockIdx.x / across, item = (blockIdx.x - b * across) * 256 + threadIdx.x;
    const int ch = item / kLanes, n0 = item % kLanes * 4;
    if (ch >= a.D) return;                                     // (whole channels: kLanes divides the wave)
    const long long unit = (static_cast<long long>(b) * a.D + ch) * N + n0;
    float4v h = {0.f, 0.f, 0.f, 0.f};
    if (a.state_in) h = __builtin_nontemporal_load(reinterpret_cast<const float4v*>(a.state_in + unit));
    const float4v rate = *reinterpret_cast<const float4v*>(a.a + static_cast<long long>(ch) * N + n0) * kLog2e;
    Raw<kF32, 1> x, delta, z;
    Raw<kF32, 4> bv, cv;
    x.load(static_cast<const char*>(a.x) + b * a.x_row + ch * kItem);
    delta.load(static_cast<const char*>(a.delta) + b * a.delta_row + ch * kItem);
    z.none();
    if (a.z) z.load(static_cast<const char*>(a.z) + b * a.z_row + ch * kItem);
    bv.load(static_cast<const char*>(a.b) + b * a.bc_row + n0 * kItem);
    cv.load(static_cast<const char*>(a.c) + b * a.bc_row + n0 * kItem);
    const float bias = a.bias ? a.bias[ch] : 0.f, skip = a.skip ? a.skip[ch] : 0.f;
    const float dt = step_of(delta[0] + bias, a.softplus), dtx = dt * x[0];
    float y = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        h[i] = __builtin_fmaf(dtx, bv[i], __builtin_amdgcn_exp2f(dt * rate[i]) * h[i]);
        y = __builtin_fmaf(cv[i], h[i], y);
    }
    if (state_out) __builtin_nontemporal_store(h, reinterpret_cast<float4v*>(state_out + unit));
#pragma unroll
    for (int m = 1; m < kLanes; m *= 2) y += __shfl_xor(y, m);
    if (n0 != 0) return;
    y = __builtin_fmaf(skip, x[0], y);
    if (a.z) y *= z[0] * sigmoid_of(z[0]);
    const float v[1] = {y};
    store<kOutF32>(static_cast<char*>(out) + (static_cast<long long>(b) * a.D + ch) * (kOutF32 ? 4 : 2), v);
}

}  // namespace

hipError_t launch_scan_step(const ScanArgs& a, void* out, float* state_out, bool f32_rows, bool f32_out, hipStream_t stream) {
    auto run = [&](auto kernel) {
        const int across = (a.D * (a.N / 4) + 255) / 256;
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(across) * a.B), dim3(256), 0, stream, a, out, state_out, across);
        return hipGetLastError();
    };
    auto go = [&](auto n) {
        constexpr int N = decltype(n)::value;
        if (f32_rows) return run(&scan_step_kernel<N, true, true>);
        return f32_out ? run(&scan_step_kernel<N, false, true>) : run(&scan_step_kernel<N, false, false>);
    };
    switch (a.N) {
        case 8: return go(std::integral_constant<int, 8>());
        case 16: return go(std::integral_constant<int, 16>());
        case 32: return go(std::integral_constant<int, 32>());
        default: return go(std::integral_constant<int, 64>());
    }
}

}  // namespace wkv6
