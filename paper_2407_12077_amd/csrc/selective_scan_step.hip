// The selective scan for one token of every sequence, or a few: h = exp(dt a) h_in + dt x b,  out = (sum_n c[n] h[n] + skip x) silu(z).
//
// Bound by the states, which are read and written once, past the caches: 1024 x 4096 channels of 16 states 106 us, 5.4 TB/s (a large copy: 5.2).  A lane has
// four states, so a load takes whole lines; what the lanes of a channel have in common each forms for itself.  One sequence: 3 us, a launch.
#include "selective_scan_tiles.h"

namespace wkv6 {
namespace {

using namespace scan;

// N / 4 lanes a channel, four states each.  kAtOnce: 1 for one token of every sequence, else tokens whose rows are asked for together.
template <int N, bool kF32, bool kOutF32, int kAtOnce>
__global__ __launch_bounds__(256) void scan_step_kernel(ScanArgs a, void* out, float* state_out, int across) {
    constexpr int kLanes = N / 4, kItem = kF32 ? 4 : 2;
    const int b = blockIdx.x / across, item = (blockIdx.x - b * across) * 256 + threadIdx.x;
    const int ch = item / kLanes, n0 = item % kLanes * 4;
    if (ch >= a.D) return;                                     // (whole channels: kLanes divides the wave)
    const long long unit = (static_cast<long long>(b) * a.D + ch) * N + n0, first = kAtOnce == 1 ? b : first_row_of(a, b);
    const int tokens = kAtOnce == 1 ? 1 : tokens_of(a, b);
    float4v h = {0.f, 0.f, 0.f, 0.f};
    if (a.state_in) h = __builtin_nontemporal_load(reinterpret_cast<const float4v*>(a.state_in + unit));
    const float4v rate = rate_of(a.a + static_cast<long long>(ch) * N + n0);
    const float bias = a.bias ? a.bias[ch] : 0.f, skip = a.skip ? a.skip[ch] : 0.f;
    for (int t = 0; t < tokens; t += kAtOnce) {
        Raw<kF32, 1> x[kAtOnce], delta[kAtOnce], z[kAtOnce];
        Raw<kF32, 4> bv[kAtOnce], cv[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            z[j].none();
            if (t + j >= tokens) continue;
            const long long row = first + t + j;
            x[j].load(static_cast<const char*>(a.x) + row * a.x_row + ch * kItem);
            delta[j].load(static_cast<const char*>(a.delta) + row * a.delta_row + ch * kItem);
            if (a.z) z[j].load(static_cast<const char*>(a.z) + row * a.z_row + ch * kItem);
            bv[j].load(static_cast<const char*>(a.b) + row * a.bc_row + n0 * kItem);
            cv[j].load(static_cast<const char*>(a.c) + row * a.bc_row + n0 * kItem);
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            if (t + j >= tokens) continue;
            const float dt = step_of(delta[j][0] + bias, a.softplus), dtx = dt * x[j][0];
            float y = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                h[i] = __builtin_fmaf(dtx, bv[j][i], __builtin_amdgcn_exp2f(dt * rate[i]) * h[i]);
                y = __builtin_fmaf(cv[j][i], h[i], y);
            }
            // (one token: its state on the way before the lanes' shares meet)
            if (kAtOnce == 1 && state_out) __builtin_nontemporal_store(h, reinterpret_cast<float4v*>(state_out + unit));
#pragma unroll
            for (int m = 1; m < kLanes; m *= 2) y += __shfl_xor(y, m);
            if (n0 == 0) {
                y = __builtin_fmaf(skip, x[j][0], y);
                if (a.z) y *= z[j][0] * sigmoid_of(z[j][0]);
                const float v[1] = {y};
                store<kOutF32>(static_cast<char*>(out) + ((first + t + j) * a.D + ch) * (kOutF32 ? 4 : 2), v);
            }
        }
    }
    if (kAtOnce > 1 && state_out) __builtin_nontemporal_store(h, reinterpret_cast<float4v*>(state_out + unit));
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
        auto some = [&](auto at_once) {
            constexpr int kAtOnce = decltype(at_once)::value;
            if (f32_rows) return run(&scan_step_kernel<N, true, true, kAtOnce>);
            return f32_out ? run(&scan_step_kernel<N, false, true, kAtOnce>) : run(&scan_step_kernel<N, false, false, kAtOnce>);
        };
        return a.T == 1 && !a.offsets ? some(std::integral_constant<int, 1>()) : some(std::integral_constant<int, 4>());
    };
    switch (a.N) {
        case 8: return go(std::integral_constant<int, 8>());
        case 16: return go(std::integral_constant<int, 16>());
        case 32: return go(std::integral_constant<int, 32>());
        default: return go(std::integral_constant<int, 64>());
    }
}

}  // namespace wkv6
