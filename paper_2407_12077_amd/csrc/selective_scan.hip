// The selective scan over whole sequences, for gfx950:
//
//     dt_t = softplus(delta_t + bias)    h_t[n] = exp(dt_t a[n]) h_{t-1}[n] + dt_t b_t[n] x_t    out_t = (sum_n c_t[n] h_t[n] + skip x_t) silu(z_t)
#include "selective_scan_tiles.h"

namespace wkv6 {
namespace {

using namespace scan;

// kStates: the segments' states from nothing, without read-outs.
template <int N, bool kF32, bool kOutF32, bool kStates>
__global__ __launch_bounds__(16 * N) void scan_kernel(ScanArgs a, char* out, float* state_out, int blocks) {
    constexpr int kWaves = N / 4, kC = kScanChunk, kCh = kScanChannels, kItem = kF32 ? 4 : 2, kOutItem = kOutF32 ? 4 : 2;
    constexpr int kPer = kC / kWaves < 8 ? kC / kWaves : 8;    // channels that a thread brings and takes of a token
    constexpr int kAcross = kCh / kPer;
    static_assert(kAcross * kC == 16 * N);
    __shared__ float2v step[2][kC][kCh];                       // dt, dt x
    __shared__ float part[kStates ? 1 : 2][kWaves][kC][kCh];   // shares of the read-outs
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int block = blockIdx.x % blocks, at = blockIdx.x / blocks, b = at % a.B, seg = at / a.B;
    const Span span = span_of(a, b, seg);
    const int D = a.D, c0 = block * kCh, ch = c0 + lane, n0 = 4 * wave;
    const bool mine = ch < D;
    const long long unit = (static_cast<long long>(b) * D + ch) * N + n0, seg_states = static_cast<long long>(a.B) * D * N;
    const long long sums_at = a.segs * seg_states, seg_sums = static_cast<long long>(a.B) * D;
    if (kStates && seg == 0 && mine)
        *reinterpret_cast<float4v*>(a.locals + unit) =
            a.state_in ? *reinterpret_cast<const float4v*>(a.state_in + unit) : float4v{0.f, 0.f, 0.f, 0.f};
    if (kStates ? span.tokens < a.seg_len : span.tokens == 0 && !span.last) return;

    float4v rate = {0.f, 0.f, 0.f, 0.f}, h = {0.f, 0.f, 0.f, 0.f};
    if (mine) {
        rate = *reinterpret_cast<const float4v*>(a.a + static_cast<long long>(ch) * N + n0) * kLog2e;
        if (!kStates && a.segs > 1) {
            h = *reinterpret_cast<const float4v*>(a.locals + unit);
            for (int q = 1; q <= seg; ++q) {
                const float sum = a.locals[sums_at + q * seg_sums + static_cast<long long>(b) * D + ch];
                const float4v local = *reinterpret_cast<const float4v*>(a.locals + q * seg_states + unit);
#pragma unroll
                for (int i = 0; i < 4; ++i) h[i] = __builtin_fmaf(__builtin_amdgcn_exp2f(sum * rate[i]), h[i], local[i]);
            }
        } else if (!kStates && a.state_in) {
            h = *reinterpret_cast<const float4v*>(a.state_in + unit);
        }
    }

    // what this thread brings: channels own .. own + kPer - 1 of token `token` of a chunk
    const int token = threadIdx.x / kAcross, own = c0 + threadIdx.x % kAcross * kPer, in_block = own - c0;
    const bool there = own < D;
    float bias[kPer], skip[kPer], dt_sum = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        bias[i] = there && a.bias ? a.bias[own + i] : 0.f;
        skip[i] = there && a.skip ? a.skip[own + i] : 0.f;
    }
    const char *x = static_cast<const char*>(a.x), *delta = static_cast<const char*>(a.delta), *z = static_cast<const char*>(a.z);
    const char *bp = static_cast<const char*>(a.b) + n0 * kItem, *cp = static_cast<const char*>(a.c) + n0 * kItem;
    struct Chunk {
        Raw<kF32, kPer> x, delta, z;
        StateRow<kF32> b, c;           // of token lane / 4
    };
    auto ask = [&](int first, Chunk& k) {
        k.x.none();
        k.delta.none();
        if (!kStates) k.z.none();
        if (there && first + token < span.tokens) {
            const long long row = span.first_row + first + token;
            k.x.load(x + row * a.x_row + own * kItem);
            k.delta.load(delta + row * a.delta_row + own * kItem);
            if (!kStates && z) k.z.load(z + row * a.z_row + own * kItem);
        }
        k.b.none();
        if (!kStates) k.c.none();
        if (first + lane / 4 < span.tokens) {
            const long long row = span.first_row + first + lane / 4;
            k.b.raw.load(bp + row * a.bc_row);
            if (!kStates) k.c.raw.load(cp + row * a.bc_row);
        }
    };
    auto bring = [&](int first, const Chunk& k, int buffer) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            float dt = step_of(k.delta[i] + bias[i], a.softplus);
            if (first + token >= span.tokens) dt = 0.f;
            step[buffer][token][in_block + i] = float2v{dt, dt * k.x[i]};
        }
    };
    Chunk now, next;
    ask(0, now);
    bring(0, now, 0);
    __syncthreads();
    int buffer = 0;
    for (int first = 0; first < span.tokens; first += kC, buffer ^= 1) {
        ask(first + kC, next);
        const float bv = now.b.plain(lane);
        float cv[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) cv[i] = kStates ? 0.f : now.c.at_token(i, lane);
        float4v y = {0.f, 0.f, 0.f, 0.f};
        each<kC>([&](auto token_of_chunk) {
            constexpr int t = decltype(token_of_chunk)::value;
            const float2v d = step[buffer][t][lane];
            float4v decayed;
#pragma unroll
            for (int i = 0; i < 4; ++i) decayed[i] = __builtin_amdgcn_exp2f(d.x * rate[i]) * h[i];
            h = outer<t>(bv, d.y, decayed);
            if constexpr (kStates) {
                dt_sum += d.x;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) y = outer<t>(cv[i], h[i], y);
                if constexpr (t % 4 == 3) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) part[buffer][wave][t - 3 + i][lane] = y[i];
                    y = float4v{0.f, 0.f, 0.f, 0.f};
                }
            }
        });
        bring(first + kC, next, buffer ^ 1);
        __syncthreads();
        if constexpr (!kStates) {
            if (there && first + token < span.tokens) {
                const long long row = span.first_row + first + token;
                float y[kPer];
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    float v = skip[i] * now.x[i];
#pragma unroll
                    for (int w = 0; w < kWaves; ++w) v += part[buffer][w][token][in_block + i];
                    if (z) v *= now.z[i] * sigmoid_of(now.z[i]);
                    y[i] = v;
                }
                store<kOutF32>(out + (row * D + own) * kOutItem, y);
            }
        }
        now = next;
    }
    if (!mine) return;
    if constexpr (kStates) {
        *reinterpret_cast<float4v*>(a.locals + (seg + 1) * seg_states + unit) = h;
        if (wave == 0) a.locals[sums_at + (seg + 1) * seg_sums + static_cast<long long>(b) * D + ch] = dt_sum;
    } else if (state_out && span.last) {
        *reinterpret_cast<float4v*>(state_out + unit) = h;
    }
}

template <int N, bool kF32>
hipError_t launch_states(const ScanArgs& a, hipStream_t stream) {
    const int blocks = static_cast<int>(scan_blocks(a.D));
    hipLaunchKernelGGL((scan_kernel<N, kF32, true, true>), dim3(static_cast<unsigned>(blocks) * a.B * (a.segs - 1)), dim3(scan_threads(N)), 0, stream, a,
                       nullptr, nullptr, blocks);
    return hipGetLastError();
}
template <int N, bool kF32, bool kOutF32>
hipError_t launch(const ScanArgs& a, void* out, float* state_out, hipStream_t stream) {
    const int blocks = static_cast<int>(scan_blocks(a.D));
    if (a.segs > 1) {
        const hipError_t err = launch_states<N, kF32>(a, stream);
        if (err != hipSuccess) return err;
    }
    hipLaunchKernelGGL((scan_kernel<N, kF32, kOutF32, false>), dim3(static_cast<unsigned>(blocks) * a.B * a.segs), dim3(scan_threads(N)), 0, stream, a,
                       static_cast<char*>(out), state_out, blocks);
    return hipGetLastError();
}

// f(N) with N known to the compiler
template <typename F>
hipError_t by_states(int N, F f) {
    switch (N) {
        case 8: return f(std::integral_constant<int, 8>());
        case 16: return f(std::integral_constant<int, 16>());
        case 32: return f(std::integral_constant<int, 32>());
        default: return f(std::integral_constant<int, 64>());
    }
}

}  // namespace

ScanPlan plan_scan(int B, int T, int D, int N) {
    const long long units = static_cast<long long>(B) * scan_blocks(D) * N / 16;
    long long segs = units > 0 ? 768 / units : 1;
    const long long most = (T + 127) / 128;
    if (segs > most) segs = most;
    if (segs > 64) segs = 64;
    if (segs < 2) return {1, T};
    long long len = (T + segs - 1) / segs;
    len = (len + kScanChunk - 1) / kScanChunk * kScanChunk;
    return {static_cast<int>((T + len - 1) / len), static_cast<int>(len)};
}

hipError_t launch_scan(const ScanArgs& a, void* out, float* state_out, bool f32_rows, bool f32_out, hipStream_t stream) {
    return by_states(a.N, [&](auto n) {
        constexpr int N = decltype(n)::value;
        if (f32_rows) return launch<N, true, true>(a, out, state_out, stream);
        return f32_out ? launch<N, false, true>(a, out, state_out, stream) : launch<N, false, false>(a, out, state_out, stream);
    });
}

hipError_t launch_scan_states(const ScanArgs& a, bool f32_rows, hipStream_t stream) {
    return by_states(a.N, [&](auto n) {
        constexpr int N = decltype(n)::value;
        return f32_rows ? launch_states<N, true>(a, stream) : launch_states<N, false>(a, stream);
    });
}

}  // namespace wkv6
