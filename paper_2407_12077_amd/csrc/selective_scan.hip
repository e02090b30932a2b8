// The selective scan over whole sequences, for gfx950:
//
//     dt_t = softplus(delta_t + bias)    h_t[n] = exp(dt_t a[n]) h_{t-1}[n] + dt_t b_t[n] x_t    out_t = (sum_n c_t[n] h_t[n] + skip x_t) silu(z_t)
//
// Bound by instruction slots: every token, channel and state has an exponential of its own (two slots), a product for its argument, a multiply-add
// into the state and one into the read-out, twenty cycles of a SIMD for a wave; nothing of it is a matrix product, as each decay belongs to one
// (channel, state).  What a token and channel have in common (softplus, gate, types) takes a third more.  8 x 4096 x 4096, N = 16, bf16 with a gate: 453 us, of
// which a vector instruction issues in 90 % (0.994 M of 1.103 M cycles of a SIMD, at 2.43 GHz 409 us; a chunk and wave: some 388 vector instructions, 76 of them double, and 16 matrix ones of
// two slots); its bytes would take 207 at a copy's rate.
//
// A workgroup has 64 channels, a lane each, and a wave four states, so that states stay in registers and neither dt x b nor c h crosses lanes.  Tokens come in
// chunks of 16: their dt and dt x are formed once, by all waves, and lie in LDS as fp32 (two chunks of them); the waves' shares of the read-outs
// meet there too.  b_t[n] is the same for all lanes: a 4 x 4 x 1 matrix instruction forms its products with dt x for a wave's four states at once,
// from a register that holds the chunk's sixteen tokens, in a quarter of the slots (8 cycles for four states; as products and with the multiply-add on the
// vector units, 64).  c_t[n] is taken from other lanes by the multiply-adds themselves: as matrix products of one row each the read-outs took 638 us.
//
// Where there are fewer workgroups than the compute units hold, or one sequence is much longer than the others, the token axis is cut (plan_scan): the
// pieces' states from nothing are formed first (scan_pieces_kernel, three quarters of the walk's time), and a piece adds up those in front of it.
// 1 x 131072 x 2048: 1499 us, of which the pieces' states 674; whole it took 15 ms.
#include "selective_scan_tiles.h"

#include <algorithm>
#include <cmath>

namespace wkv6 {
namespace {

using namespace scan;

// One segment of one sequence, 64 channels.  kStates: its state from nothing, without read-outs.
template <int N, bool kF32, bool kOutF32, bool kStates, bool kGate>
__device__ __forceinline__ void walk(ScanArgs a, char* out, float* state_out, int blocks, int index) {
    constexpr int kWaves = N / 4, kC = kScanChunk, kCh = kScanChannels, kItem = kF32 ? 4 : 2, kOutItem = kOutF32 ? 4 : 2;
    constexpr int kPer = kC / kWaves < 8 ? kC / kWaves : 8;    // channels that a thread brings and takes of a token
    constexpr int kAcross = kCh / kPer;
    static_assert(kAcross * kC == 16 * N);
    __shared__ float2v step[2][kC][kCh];                       // dt, dt x
    __shared__ float part[kStates ? 1 : 2][kWaves][kC][kCh];   // shares of the read-outs
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int block = index % blocks, at = index / blocks, b = at % a.B, seg = at / a.B;
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
        rate = rate_of(a.a + static_cast<long long>(ch) * N + n0);
        if (!kStates && a.segs > 1) {
            h = *reinterpret_cast<const float4v*>(a.locals + unit);
            const float4v third = rate * (1.f / 3);
#pragma unroll 4
            for (int q = 1; q <= seg; ++q)
                pass_on(h, a.locals[sums_at + q * seg_sums + static_cast<long long>(b) * D + ch], third,
                        *reinterpret_cast<const float4v*>(a.locals + q * seg_states + unit));
        } else if (!kStates && a.state_in) {
            h = *reinterpret_cast<const float4v*>(a.state_in + unit);
        }
    }

    // what this thread brings: channels own .. own + kPer - 1 of token `token` of a chunk
    const int token = threadIdx.x / kAcross, own = c0 + threadIdx.x % kAcross * kPer, in_block = own - c0;
    const bool there = own < D;
    const unsigned softplus = softplus_bits(a.softplus);
    float bias[kPer], skip[kPer], dt_sum = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        bias[i] = there && a.bias ? a.bias[own + i] : 0.f;
        skip[i] = there && a.skip ? a.skip[own + i] : 0.f;
    }
    struct Chunk {
        Raw<kF32, kPer> x, delta, z;
        Plain<kF32> b;
        ByRow<kF32, kC / 4> c;
    };
    const int x_at = there ? token * static_cast<int>(a.x_row) + own * kItem : kNowhere;
    const int delta_at = there ? token * static_cast<int>(a.delta_row) + own * kItem : kNowhere;
    const int z_at = there ? token * static_cast<int>(a.z_row) + own * kItem : kNowhere;
    const int out_at = there ? (token * D + own) * kOutItem : kNowhere;
    const int bc_row = static_cast<int>(a.bc_row);
    const long long row0 = span.first_row;
    Rows xs(a.x, row0, a.x_row), deltas(a.delta, row0, a.delta_row), zs(a.z, row0, a.z_row), bs(a.b, row0, a.bc_row), cs(a.c, row0, a.bc_row),
        outs(out, row0 - kC, static_cast<long long>(D) * kOutItem);
    auto ask = [&](int left, Chunk& k) {                       // the next chunk, if `left` tokens are left
        const int count = rows_of<kC>(left);
        k.x.load(xs.first(count), x_at);
        k.delta.load(deltas.first(count), delta_at);
        k.b.load(bs.first(count), lane, bc_row, n0);
        xs.move(kC);
        deltas.move(kC);
        bs.move(kC);
        if constexpr (!kStates) {
            if constexpr (kGate) k.z.load(zs.first(count), z_at);
            k.c.load(cs.first(count), lane, bc_row, n0);
            zs.move(kC);
            cs.move(kC);
        }
    };
    auto bring = [&](int first, const Chunk& k, int buffer) {
        float dts[kPer];
        steps_of(k.delta, bias, softplus, dts);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const float dt = first + token < span.tokens ? dts[i] : 0.f;
            step[buffer][token][in_block + i] = float2v{dt, dt * k.x[i]};
        }
    };
    auto leave = [&](int count, const Chunk& k, int buffer) {
        float y[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            y[i] = skip[i] * k.x[i];
#pragma unroll
            for (int w = 0; w < kWaves; ++w) y[i] += part[buffer][w][token][in_block + i];
            if constexpr (kGate) y[i] *= k.z[i] * sigmoid_of(k.z[i]);
        }
        store<kOutF32>(outs.first(count), out_at, y);
        outs.move(kC);
    };
    Chunk before = {}, now, next;
    ask(span.tokens, now);
    bring(0, now, 0);
    // Between two barriers: a chunk's read-outs, the states of the chunk behind it, and the step sizes of the one behind that; without a branch, so that they
    // hide one another's latencies.
    int buffer = 0, first = 0;
    for (; first < span.tokens; first += kC, buffer ^= 1) {
        __syncthreads();
        // Waves of two workgroups share a SIMD, and the older one would have its way until it is through, and the younger be left alone: whoever is
        // further in its chunk gives way (all alike 530 us, two levels 502, four 457).
        __builtin_amdgcn_s_setprio(3);
        ask(span.tokens - first - kC, next);
        if constexpr (!kStates) leave(first > 0 ? kC : 0, before, buffer ^ 1);     // (nothing in the first turn)
        const float bv = now.b.value();
        float dt_chunk = 0.f;
        each<kC>([&](auto token_of_chunk) {
            constexpr int t = decltype(token_of_chunk)::value;
            const float2v d = step[buffer][t][lane];
            const float4v add = outer<t>(bv, d.y);
            if constexpr (kStates) dt_chunk += d.x;
#pragma unroll
            for (int i = 0; i < 4; ++i) h[i] = __builtin_fmaf(__builtin_amdgcn_exp2f(d.x * rate[i]), h[i], add[i]);
            if constexpr (!kStates) part[buffer][wave][t][lane] = read_out<t % 4>(now.c.value(t / 4), h, h[0]);
            if constexpr (t == 3) __builtin_amdgcn_s_setprio(2);
            if constexpr (t == 7) {
                __builtin_amdgcn_s_setprio(1);
                __builtin_amdgcn_sched_barrier(0);             // (without it the compiler brings too much forward: 558 us)
            }
        });
        __builtin_amdgcn_s_setprio(0);
        if constexpr (kStates) dt_sum += dt_chunk;
        bring(first + kC, next, buffer ^ 1);
        before = now;
        now = next;
    }
    if (!kStates && span.tokens > 0) {
        __syncthreads();
        leave(span.tokens - (first - kC), before, buffer ^ 1);
    }
    if (!mine) return;
    if constexpr (kStates) {
        *reinterpret_cast<float4v*>(a.locals + (seg + 1) * seg_states + unit) = h;
        if (wave == 0) a.locals[sums_at + (seg + 1) * seg_sums + static_cast<long long>(b) * D + ch] = dt_sum;
    } else if (state_out && span.last) {
        *reinterpret_cast<float4v*>(state_out + unit) = h;
    }
}

// What a segment hands to the one in front of it if it gets nothing from behind, and the sum of its step sizes.
template <int N, bool kF32>
__device__ __forceinline__ void walk_behind(const ScanArgs& a, const char* dout, float* behind, int blocks, int index) {
    constexpr int kWaves = N / 4, kC = kScanChunk, kCh = kScanChannels, kItem = kF32 ? 4 : 2;
    constexpr int kPer = kC / kWaves < 8 ? kC / kWaves : 8, kAcross = kCh / kPer;
    __shared__ float2v step[2][kC][kCh];                       // dt, dy
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int block = index % blocks, at = index / blocks, b = at % a.B, seg = 1 + at / a.B;
    const Span span = span_of(a, b, seg);
    if (span.tokens == 0) return;
    const int D = a.D, c0 = block * kCh, ch = c0 + lane, n0 = 4 * wave;
    const bool mine = ch < D;
    float4v rate = {0.f, 0.f, 0.f, 0.f}, g = {0.f, 0.f, 0.f, 0.f};
    if (mine) rate = rate_of(a.a + static_cast<long long>(ch) * N + n0);
    const int token = threadIdx.x / kAcross, own = c0 + threadIdx.x % kAcross * kPer, in_block = own - c0;
    const bool there = own < D;
    const unsigned softplus = softplus_bits(a.softplus);
    float bias[kPer], dt_sum = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) bias[i] = there && a.bias ? a.bias[own + i] : 0.f;
    struct Chunk {
        Raw<kF32, kPer> delta, z, dout;
        Plain<kF32> c;
    };
    const int delta_at = there ? token * static_cast<int>(a.delta_row) + own * kItem : kNowhere;
    const int z_at = there ? token * static_cast<int>(a.z_row) + own * kItem : kNowhere;
    const int out_at = there ? (token * D + own) * kItem : kNowhere;
    int first = (span.tokens - 1) / kC * kC, buffer = 0;
    const long long row0 = span.first_row + first;
    Rows deltas(a.delta, row0, a.delta_row), zs(a.z, row0, a.z_row), douts(dout, row0, static_cast<long long>(D) * kItem), cs(a.c, row0, a.bc_row);
    auto ask = [&](int at, Chunk& k) {                         // chunks in falling order
        const int count = at < 0 ? 0 : rows_of<kC>(span.tokens - at);
        k.delta.load(deltas.first(count), delta_at);
        if (a.z) k.z.load(zs.first(count), z_at);
        k.dout.load(douts.first(count), out_at);
        k.c.load(cs.first(count), lane, static_cast<int>(a.bc_row), n0);
        deltas.move(-kC);
        zs.move(-kC);
        douts.move(-kC);
        cs.move(-kC);
    };
    auto bring = [&](int first, const Chunk& k, int buffer) {
        float dts[kPer], dy[kPer];
        steps_of(k.delta, bias, softplus, dts);
#pragma unroll
        for (int i = 0; i < kPer; ++i) dy[i] = k.dout[i];
        if (a.z) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) dy[i] *= k.z[i] * sigmoid_of(k.z[i]);
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i) step[buffer][token][in_block + i] = float2v{first + token < span.tokens ? dts[i] : 0.f, dy[i]};
    };
    Chunk now, next;
    ask(first, now);
    bring(first, now, 0);
    __syncthreads();
    for (; first >= 0; first -= kC, buffer ^= 1) {
        ask(first - kC, next);
        const float cv = now.c.value();
        float dt_chunk = 0.f;
        each<kC>([&](auto back) {
            constexpr int t = kC - 1 - decltype(back)::value;
            const float2v d = step[buffer][t][lane];
            g = outer<t>(cv, d.y, g);
#pragma unroll
            for (int i = 0; i < 4; ++i) g[i] *= __builtin_amdgcn_exp2f(d.x * rate[i]);
            dt_chunk += d.x;
        });
        dt_sum += dt_chunk;
        bring(first - kC, next, buffer ^ 1);
        __syncthreads();
        now = next;
    }
    if (!mine) return;
    const long long seg_states = static_cast<long long>(a.B) * D * N, unit = (static_cast<long long>(b) * D + ch) * N + n0;
    *reinterpret_cast<float4v*>(behind + seg * seg_states + unit) = g;
    if (wave == 0) behind[a.segs * seg_states + (static_cast<long long>(seg) * a.B + b) * D + ch] = dt_sum;
}

template <int N, bool kF32, bool kOutF32, bool kGate>
__global__ __launch_bounds__(16 * N, N <= 16 ? 3 : 4) void scan_kernel(ScanArgs a, char* out, float* state_out, int blocks) {
    walk<N, kF32, kOutF32, false, kGate>(a, out, state_out, blocks, blockIdx.x);
}

// The pieces' states, by the first `states` workgroups, and what they hand to the pieces in front of them, by the others.
template <int N, bool kF32, bool kBoth>
__global__ __launch_bounds__(16 * N, 4) void scan_pieces_kernel(ScanArgs a, const char* dout, float* behind, int blocks, int states) {
    const int index = blockIdx.x;
    if (!kBoth || index < states) walk<N, kF32, true, true, false>(a, nullptr, nullptr, blocks, index);
    else if constexpr (kBoth) walk_behind<N, kF32>(a, dout, behind, blocks, index - states);
}

template <int N, bool kF32>
hipError_t launch_pieces(const ScanArgs& a, const void* dout, float* behind, hipStream_t stream) {
    const int blocks = static_cast<int>(scan_blocks(a.D));
    const unsigned states = static_cast<unsigned>(blocks) * a.B * (a.segs - 1);
    const auto kernel = behind ? &scan_pieces_kernel<N, kF32, true> : &scan_pieces_kernel<N, kF32, false>;
    hipLaunchKernelGGL(kernel, dim3(behind ? 2 * states : states), dim3(scan_threads(N)), 0, stream, a, static_cast<const char*>(dout), behind, blocks,
                       static_cast<int>(states));
    return hipGetLastError();
}
template <int N, bool kF32, bool kOutF32>
hipError_t launch(const ScanArgs& a, void* out, float* state_out, hipStream_t stream) {
    const int blocks = static_cast<int>(scan_blocks(a.D));
    if (a.segs > 1) {
        const hipError_t err = launch_pieces<N, kF32>(a, nullptr, nullptr, stream);
        if (err != hipSuccess) return err;
    }
    const auto kernel = a.z ? &scan_kernel<N, kF32, kOutF32, true> : &scan_kernel<N, kF32, kOutF32, false>;
    hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks) * a.B * a.segs), dim3(scan_threads(N)), 0, stream, a, static_cast<char*>(out), state_out,
                       blocks);
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

int scan_most_segments(int B, int T, int D, bool packed) {
    long long most = kScanMostSegments, workgroups = B * scan_blocks(D);
    if (packed && workgroups >= compute_units()) {
        most = kScanPackedWorkgroups / workgroups;
        if (most > kScanPackedSegments) most = kScanPackedSegments;
    }
    const long long pairs = (T + kScanChunk - 1) / kScanChunk / 2;
    if (most > pairs) most = pairs;
    return most < 2 ? 1 : static_cast<int>(most);
}

ScanPlan plan_scan(int B, int T, int D, int N, long long packed_rows, bool backward) {
    const double chunks = (T + kScanChunk - 1) / kScanChunk, workgroups = static_cast<double>(B) * scan_blocks(D), units = compute_units();
    if (workgroups < 1 || T < 2) return {1, 1};
    // microseconds of a chunk, and workgroups that a compute unit holds; N = 8, 16, 32, 64
    static constexpr double kAlone[2][4] = {{1.7, 1.46, 1.87, 2.9}, {6.9, 5.5, 7.5, 15.4}}, kShare[2][4] = {{0.85, 0.8, 1.3, 2.3}, {2.8, 3.13, 5.8, 11.8}};
    static constexpr int kHeld[2][4] = {{5, 3, 2, 1}, {4, 2, 1, 1}};
    const int which = N == 8 ? 0 : N == 16 ? 1 : N == 32 ? 2 : 3, held = kHeld[backward][which];
    const double alone = kAlone[backward][which], share = kShare[backward][which], pieces = backward ? 0.4 : 0.74;
    auto together = [&](double count) { return std::max(alone, share * (count + 0.3)); };      // `count` workgroups on a unit, a chunk of each
    // a walk of `count` workgroups over `len` chunks: rounds of as many as there is room for, and a last one
    auto walk = [&](double count, double len) {
        const double rounds = std::floor(count / (units * held)), rest = count - rounds * units * held;
        return rounds * len * together(held) + (rest > 0 ? len * together(std::ceil(rest / units)) : 0);
    };
    // of packed sequences: how many workgroups there are if each takes at most `len` chunks
    auto live = [&](double len) { return (static_cast<double>(packed_rows) / (len * kScanChunk) + 0.5 * B) * scan_blocks(D); };
    double best = packed_rows < 0 ? walk(workgroups, chunks) : std::max(1.13 * chunks * alone, live(1) * together(held) / held / units);
    ScanPlan plan{1, T};
    const int most = scan_most_segments(B, T, D, packed_rows >= 0);
    for (int segs = 2; segs <= most; ++segs) {
        const double len = std::ceil(chunks / segs), one = walk(packed_rows < 0 ? workgroups * std::ceil(chunks / len) : live(len), len);
        const double time = (1 + pieces) * one + (backward ? 8 + segs : 2 + 0.3 * segs);
        if (time >= best) continue;
        best = time;
        plan.seg_len = static_cast<int>(len) * kScanChunk;
        plan.segs = (T - 1) / plan.seg_len + 1;
    }
    return plan;
}

hipError_t launch_scan(const ScanArgs& a, void* out, float* state_out, bool f32_rows, bool f32_out, hipStream_t stream) {
    return by_states(a.N, [&](auto n) {
        constexpr int N = decltype(n)::value;
        if (f32_rows) return launch<N, true, true>(a, out, state_out, stream);
        return f32_out ? launch<N, false, true>(a, out, state_out, stream) : launch<N, false, false>(a, out, state_out, stream);
    });
}

hipError_t launch_scan_pieces(const ScanArgs& a, const ScanGradients& g, bool f32_rows, hipStream_t stream) {
    return by_states(a.N, [&](auto n) {
        constexpr int N = decltype(n)::value;
        return f32_rows ? launch_pieces<N, true>(a, g.dout, g.behind, stream) : launch_pieces<N, false>(a, g.dout, g.behind, stream);
    });
}

}  // namespace wkv6
