// The short causal convolution of every channel over its own tokens, and its gradients, for gfx950:
//
//     p_t = bias + sum_j w[j] x_{t-W+1+j}    out = silu(p)
//     dp_t = dout_t silu'(p_t)    dx_s = sum_j w[j] dp_{s+W-1-j}    dw[j] = sum_t dp_t x_{t-W+1+j}    dbias = sum_t dp_t
//
// Bound by memory.  A thread has four channels (eight of a single token) of a run of 16 tokens (32 of the gradients) and keeps the inputs under its
// taps in registers, so a row is read once, but for the W - 1 rows in front of a run (and behind it, of the gradients), which a neighbour in the same
// workgroup reads too.  8 x 4096 x 4096 bf16, W = 4: 113 us, 4.75 TB/s (a large copy: 5.2); eight channels a thread 118, runs of 8 or 32 tokens 128 and
// 120, addresses by multiplication 118.  Gradients of 8 x 2048 x 4096 101 us, 4.0 TB/s, of which the fold is 5: eight channels a thread 117 (240
// registers), runs of 16 or 64 tokens 127 and 115.  24 x 4096 single tokens 3.7 us: one launch.
#include "short_conv.h"

#include "selective_scan_tiles.h"

#include <algorithm>

namespace wkv6 {
namespace {

using namespace scan;

struct Place {
    long long row0;                    // of the sequence's first token
    int len, first, end;               // tokens of the sequence; this thread's
};
// Tokens first .. end - 1 of sequence b for slice `slice` of segment `seg`.
__device__ __forceinline__ Place place_of(const ConvArgs& a, int b, int seg, int slice, int run) {
    Place p;
    p.row0 = first_row_of(a, b);
    p.len = tokens_of(a, b);
    const long long first = static_cast<long long>(seg) * a.seg_len + slice * run, end = first + run;
    p.first = static_cast<int>(first < p.len ? first : p.len);
    p.end = static_cast<int>(end < p.len ? end : p.len);
    return p;
}

template <bool kF32, int kG>
struct Row {
    Raw<kF32, kG> raw;
    __device__ __forceinline__ void get(float (&v)[kG]) const {
#pragma unroll
        for (int i = 0; i < kG; ++i) v[i] = raw[i];
    }
};

template <int W, int kG>
struct Taps {
    float w[W][kG], bias[kG];
    __device__ __forceinline__ void load(const ConvArgs& a, int ch) {
#pragma unroll
        for (int i = 0; i < kG; ++i) {
#pragma unroll
            for (int j = 0; j < W; ++j) w[j][i] = a.w[static_cast<long long>(ch + i) * W + j];
            bias[i] = a.bias ? a.bias[ch + i] : 0.f;
        }
    }
};

// The threads of a workgroup: `lanes` side by side over groups of channels, 256 / lanes slices of `run` tokens one behind the other.
template <int W, bool kF32, int kG>
__global__ __launch_bounds__(kConvThreads) void conv_kernel(ConvArgs a, char* out, char* state_out, int across, int run) {
    constexpr int kItem = kF32 ? 4 : 2, kBatch = 4;
    const int column = threadIdx.x % a.lanes, slice = threadIdx.x / a.lanes;
    const int block = blockIdx.x % across, at = blockIdx.x / across, b = at % a.B, seg = at / a.B;
    const int ch = (block * a.lanes + column) * kG;
    if (ch >= a.D) return;
    const Place p = place_of(a, b, seg, slice, run);
    const bool head = seg == 0 && slice == 0;
    if (p.first >= p.end && !head) return;
    const char* x = static_cast<const char*>(a.x) + p.row0 * a.x_row + ch * kItem;
    const long long state_row = static_cast<long long>(a.D) * kItem, state_at = static_cast<long long>(b) * (W - 1) * state_row + ch * kItem;
    Taps<W, kG> taps;
    taps.load(a, ch);
    float win[W][kG];                                          // win[W - 1]: the token at hand
    Row<kF32, kG> front[W - 1];
    if (head) {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            front[j].raw.none();
            if (a.state_in) front[j].raw.load(static_cast<const char*>(a.state_in) + state_at + j * state_row);
        }
        if (state_out) {                                       // (no other thread reads these channels' state_in, which may be state_out)
            Row<kF32, kG> last[W - 1];
#pragma unroll
            for (int j = 0; j < W - 1; ++j) {
                const int t = p.len - (W - 1) + j;             // below nought: of the old state
#pragma unroll
                for (int q = 0; q < W - 1; ++q)
                    if (t + W - 1 == q) last[j] = front[q];
                if (t >= 0) last[j].raw.load(x + t * a.x_row);
            }
#pragma unroll
            for (int j = 0; j < W - 1; ++j) last[j].raw.put(state_out + state_at + j * state_row);
        }
    } else {
#pragma unroll
        for (int j = 0; j < W - 1; ++j) front[j].raw.load(x + (p.first - (W - 1) + j) * a.x_row);   // run >= W - 1: rows of the sequence
    }
#pragma unroll
    for (int j = 0; j < W - 1; ++j) front[j].get(win[j + 1]);
    Row<kF32, kG> now[kBatch], next[kBatch];
    const char* from = x + p.first * a.x_row;                  // (addresses by addition: a product costs more than what is done with a row)
    auto ask = [&](int t, Row<kF32, kG>(&r)[kBatch]) {
#pragma unroll
        for (int i = 0; i < kBatch; ++i, from += a.x_row)
            if (t + i < p.end) r[i].raw.load(from);
    };
    char* to = out + (p.row0 + p.first) * state_row + ch * kItem;
    ask(p.first, now);
    for (int t = p.first; t < p.end; t += kBatch) {
        ask(t + kBatch, next);
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            if (t + i >= p.end) break;
            float y[kG];
#pragma unroll
            for (int j = 0; j < W - 1; ++j)
#pragma unroll
                for (int e = 0; e < kG; ++e) win[j][e] = win[j + 1][e];
            now[i].get(win[W - 1]);
#pragma unroll
            for (int e = 0; e < kG; ++e) {
                float v = taps.bias[e];
#pragma unroll
                for (int j = 0; j < W; ++j) v = __builtin_fmaf(taps.w[j][e], win[j][e], v);
                y[e] = a.silu ? v * sigmoid_of(v) : v;
            }
            store<kF32>(to, y);
            to += state_row;
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) now[i] = next[i];
    }
}

template <int W, bool kF32, int kG>
__global__ __launch_bounds__(kConvThreads) void conv_step_kernel(ConvArgs a, char* out, char* state_out, int groups) {
    constexpr int kItem = kF32 ? 4 : 2;
    const long long item = static_cast<long long>(blockIdx.x) * kConvThreads + threadIdx.x;
    if (item >= static_cast<long long>(groups) * a.B) return;
    const int b = static_cast<int>(item / groups), ch = static_cast<int>(item - static_cast<long long>(b) * groups) * kG;
    const long long row = static_cast<long long>(a.D) * kItem, state_at = static_cast<long long>(b) * (W - 1) * row + ch * kItem;
    Taps<W, kG> taps;
    Row<kF32, kG> in[W];
#pragma unroll
    for (int j = 0; j < W - 1; ++j) {
        in[j].raw.none();
        if (a.state_in) in[j].raw.load(static_cast<const char*>(a.state_in) + state_at + j * row);
    }
    in[W - 1].raw.load(static_cast<const char*>(a.x) + b * a.x_row + ch * kItem);
    taps.load(a, ch);
    float y[kG];
#pragma unroll
    for (int e = 0; e < kG; ++e) {
        float v = taps.bias[e];
#pragma unroll
        for (int j = 0; j < W; ++j) v = __builtin_fmaf(taps.w[j][e], in[j].raw[e], v);
        y[e] = a.silu ? v * sigmoid_of(v) : v;
    }
    store<kF32>(out + b * row + ch * kItem, y);
    if (!state_out) return;
#pragma unroll
    for (int j = 0; j < W - 1; ++j) in[j + 1].raw.put(state_out + state_at + j * row);
}

template <int W, bool kF32, int kG>
__global__ __launch_bounds__(kConvThreads) void conv_backward_kernel(ConvArgs a, const char* dout, const char* dstate_out, char* dx, char* dstate_in,
                                                                     float* partials, unsigned whole, int across, int run) {
    constexpr int kItem = kF32 ? 4 : 2;
    __shared__ float meet[kConvThreads / 2][(W + 1) * kG + 1];
    __shared__ int starts[kConvThreads / 64];
    const int column = threadIdx.x % a.lanes, slice = threadIdx.x / a.lanes;
    const int block = blockIdx.x % across, at = blockIdx.x / across, b = at % a.B, seg = at / a.B;
    const int ch = (block * a.lanes + column) * kG;
    const bool there = ch < a.D;
    const Place p = place_of(a, b, seg, slice, run);
    const bool head = seg == 0 && slice == 0;
    if (static_cast<long long>(seg) * a.seg_len >= p.len && seg > 0) return;      // (the whole workgroup)
    // (whether the next sequence starts where this one ends is asked here, with the other offsets, and not at the end: 2000 sequences of up to 40 x 512 66.6 -> 64.4 us)
    const bool by_row = a.offsets && a.segs > 1, followed = by_row && b + 1 < a.B && start_behind(a, b + 1, p.row0 + p.len) == p.row0 + p.len;
    float sums[W + 1][kG];
#pragma unroll
    for (int j = 0; j <= W; ++j)
#pragma unroll
        for (int e = 0; e < kG; ++e) sums[j][e] = 0.f;
    if (there && (p.first < p.end || head)) {
        const long long dense = static_cast<long long>(a.D) * kItem, state_at = static_cast<long long>(b) * (W - 1) * dense + ch * kItem;
        const char* x = static_cast<const char*>(a.x) + p.row0 * a.x_row + ch * kItem;
        const char* dy = dout + p.row0 * dense + ch * kItem;
        char* to = dx + (p.row0 + p.first - (W - 1)) * a.x_row + ch * kItem;     // of the input W - 1 in front of the token at hand
        const char *x_from = x + p.first * a.x_row, *dy_from = dy + p.first * dense;
        Taps<W, kG> taps;
        taps.load(a, ch);
        float win[W][kG], dp[W][kG];                           // dp[W - 1]: of the token at hand
#pragma unroll
        for (int j = 0; j < W; ++j)
#pragma unroll
            for (int e = 0; e < kG; ++e) dp[j][e] = 0.f;
#pragma unroll
        for (int j = 0; j < W - 1; ++j) {
            Row<kF32, kG> r;
            r.raw.none();
            if (!head) r.raw.load(x + (p.first - (W - 1) + j) * a.x_row);
            else if (a.state_in) r.raw.load(static_cast<const char*>(a.state_in) + state_at + j * dense);
            r.get(win[j + 1]);
        }
        // Behind this thread's own tokens W - 1 more, whose dp its last inputs have a share in.
        const int stop = p.end + W - 1;
        constexpr int kBatch = 2;
        Row<kF32, kG> xs[2][kBatch], ds[2][kBatch];
        auto ask = [&](int t, int which) {
#pragma unroll
            for (int i = 0; i < kBatch; ++i, x_from += a.x_row, dy_from += dense) {
                xs[which][i].raw.none();
                ds[which][i].raw.none();
                if (t + i < stop && t + i < p.len) {
                    xs[which][i].raw.load(x_from);
                    ds[which][i].raw.load(dy_from);
                }
            }
        };
        auto one = [&](int t, const Row<kF32, kG>& xr, const Row<kF32, kG>& dr) {
#pragma unroll
            for (int j = 0; j < W - 1; ++j)
#pragma unroll
                for (int e = 0; e < kG; ++e) {
                    win[j][e] = win[j + 1][e];
                    dp[j][e] = dp[j + 1][e];
                }
            xr.get(win[W - 1]);
            dr.get(dp[W - 1]);
            const bool own = t < p.end;
#pragma unroll
            for (int e = 0; e < kG; ++e) {
                if (a.silu && t < p.len) {           // (behind the end dp is nought, whatever is under the taps)
                    float v = taps.bias[e];
#pragma unroll
                    for (int j = 0; j < W; ++j) v = __builtin_fmaf(taps.w[j][e], win[j][e], v);
                    const float q = sigmoid_of(v);
                    dp[W - 1][e] *= q * __builtin_fmaf(v, 1.f - q, 1.f);
                }
                if (own) {
#pragma unroll
                    for (int j = 0; j < W; ++j) sums[j][e] = __builtin_fmaf(dp[W - 1][e], win[j][e], sums[j][e]);
                    sums[W][e] += dp[W - 1][e];
                }
            }
            const int s = t - (W - 1);                         // the input that has all its shares now
            char* place = to;
            to += a.x_row;
            if (s < (head ? -(W - 1) : p.first) || s >= p.end) return;
            if (s < 0) {
                if (!dstate_in) return;
                place = dstate_in + state_at + t * dense;
            }
            float v[kG];
#pragma unroll
            for (int e = 0; e < kG; ++e) {
                v[e] = 0.f;
#pragma unroll
                for (int j = 0; j < W; ++j) v[e] = __builtin_fmaf(taps.w[j][e], dp[W - 1 - j][e], v[e]);
            }
            if (dstate_out && s >= p.len - (W - 1)) {
                Row<kF32, kG> r;
                r.raw.load(dstate_out + state_at + (s - p.len + W - 1) * dense);
#pragma unroll
                for (int e = 0; e < kG; ++e) v[e] += r.raw[e];
            }
            store<kF32>(place, v);
        };
        ask(p.first, 0);
        for (int t = p.first; t < stop; t += 2 * kBatch) {
            ask(t + kBatch, 1);
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (t + i < stop) one(t + i, xs[0][i], ds[0][i]);
            ask(t + 2 * kBatch, 0);
#pragma unroll
            for (int i = 0; i < kBatch; ++i)
                if (t + kBatch + i < stop) one(t + kBatch + i, xs[1][i], ds[1][i]);
        }
    }
    if (!partials) return;
    // the slices' sums meet, half of them at a time
    for (int half = kConvThreads / 2; half >= a.lanes; half /= 2) {
        if (static_cast<int>(threadIdx.x) >= half && static_cast<int>(threadIdx.x) < 2 * half)
#pragma unroll
            for (int j = 0; j <= W; ++j)
#pragma unroll
                for (int e = 0; e < kG; ++e) meet[threadIdx.x - half][j * kG + e] = sums[j][e];
        __syncthreads();
        if (static_cast<int>(threadIdx.x) < half)
#pragma unroll
            for (int j = 0; j <= W; ++j)
#pragma unroll
                for (int e = 0; e < kG; ++e) sums[j][e] += meet[threadIdx.x][j * kG + e];
        __syncthreads();
    }
    // where the sums go, and the places that are nobody's (whole_places)
    const bool last = static_cast<long long>(seg + 1) * a.seg_len >= p.len;
    auto next_start = [&](long long row) {                     // of all sequences
        long long start = a.rows;
        for (int i = threadIdx.x; i < a.B; i += kConvThreads) start = std::min(start, start_behind(a, i, row));
        int first = static_cast<int>(start);
#pragma unroll
        for (int m = 1; m < 64; m *= 2) first = std::min(first, __shfl_xor(first, m));
        if (threadIdx.x % 64 == 0) starts[threadIdx.x / 64] = first;
        __syncthreads();
        first = starts[0];
#pragma unroll
        for (int w = 1; w < kConvThreads / 64; ++w) first = std::min(first, starts[w]);
        __syncthreads();
        return place_of_row(first, a.seg_len);
    };
    long long mine = static_cast<long long>(b) * a.segs + seg, front = 0, behind = 0, next = 0;
    if (by_row) {
        const long long own = place_of_row(p.row0, a.seg_len) + seg;
        mine = last ? static_cast<long long>(whole) + b : own;
        if (b == 0 && seg == 0 && (p.len == 0 || own > 0)) front = next_start(0);
        if (last && p.len > 0) {
            const long long end = p.row0 + p.len;
            behind = own;
            next = place_of_row(end, a.seg_len);
            if (next < whole && !followed) {                   // most often there are some without tokens in between
                int other = b + 2;
                while (other < a.B && other < b + 8 && tokens_of(a, other) == 0) ++other;
                if (other >= a.B || start_behind(a, other, end) != end) next = next_start(end);
            }
        }
    }
    if (slice != 0 || !there) return;
    const long long values = static_cast<long long>(W + 1) * a.D;
    auto leave = [&](long long place, auto v) {
#pragma unroll
        for (int j = 0; j <= W; ++j)
#pragma unroll
            for (int e = 0; e < kG; e += 4)
                *reinterpret_cast<float4v*>(partials + place * values + static_cast<long long>(j) * a.D + ch + e) = float4v{v(j, e), v(j, e + 1), v(j, e + 2), v(j, e + 3)};
    };
    leave(mine, [&](int j, int e) { return sums[j][e]; });
    auto none = [](int, int) { return 0.f; };
    for (long long i = 0; i < front; ++i) leave(i, none);
    for (long long i = behind; i < next; ++i) leave(i, none);
}

// dw [D][W] and dbias [D]: 64 values a workgroup, the places in sixteen turns, in their order.
constexpr int kFoldTurns = 16;
__global__ __launch_bounds__(64 * kFoldTurns) void conv_fold_kernel(int D, int W, long long places, const float* partials, float* dw, float* dbias) {
    __shared__ float meet[kFoldTurns][64];
    const int lane = threadIdx.x & 63, turn = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), values = (W + 1) * D, value = blockIdx.x * 64 + lane;
    float sum = 0.f;
    if (value < values) {
        const float* from = partials + static_cast<long long>(turn) * values + value;
#pragma unroll 8
        for (long long i = turn; i < places; i += kFoldTurns, from += static_cast<long long>(kFoldTurns) * values) sum += *from;
    }
    meet[turn][lane] = sum;
    __syncthreads();
    if (turn != 0 || value >= values) return;
#pragma unroll
    for (int i = 1; i < kFoldTurns; ++i) sum += meet[i][lane];
    const int tap = value / D, ch = value - tap * D;
    if (tap == W) dbias[ch] = sum;
    else dw[static_cast<long long>(ch) * W + tap] = sum;
}

template <typename F>
hipError_t by_taps(int W, bool f32, F f) {
    auto one = [&](auto w) { return f32 ? f(w, std::true_type()) : f(w, std::false_type()); };
    if (W == 2) return one(std::integral_constant<int, 2>());
    if (W == 3) return one(std::integral_constant<int, 3>());
    return one(std::integral_constant<int, 4>());
}

int across_of(const ConvArgs& a) { return (a.D / kConvGroup + a.lanes - 1) / a.lanes; }

}  // namespace

ConvPlan plan_conv(int B, int T, int D, long long rows, bool backward) {
    ConvPlan p;
    const int groups = D / kConvGroup;
    p.lanes = 64;
    while (p.lanes > 1 && p.lanes / 2 >= groups) p.lanes /= 2;
    // Half as many where that leaves fewer without a group; of 256 groups and more few are without one anyway.  With 64 and with 32, microseconds of prompts of 16384 rows x 264, 384, 640,
    // 896: 8.9, 8.8, 10.9, 13.2 and 7.6, 8.2, 10.2, 12.6; x 1056, 2056: 15.3, 39.2 and 16.2, 41.9.  Gradients of 4000 rows 13.4, 13.1, 14.6, 16.6 and 11.3, 11.4, 13.0, 14.7; of
    // 65536 45.0, 45.1, 72.9, 91.1 and 45.0, 47.0, 72.8, 87.2; of 16384, where the runs are short, 19.6, 19.0, 25.4, 27.5 and 20.2, 20.3, 24.4, 30.6.
    if (groups > 32 && groups < 256 && groups % 64 != 0 && groups % 64 <= 32) p.lanes = 32;
    const int slices = kConvThreads / p.lanes, across = (groups + p.lanes - 1) / p.lanes;
    int run = backward ? 32 : 16;
    while (run > 4 && rows * across / (slices * run) < 1024) run /= 2;
    // A launch has places for B sequences of T tokens; where packed ones are mostly shorter, longer runs keep the empty workgroups from taking longer than the
    // others: not more than sixteen for one that has work.
    for (;; run *= 2) {
        p.seg_len = slices * run;
        p.segs = T > 0 ? (T - 1) / p.seg_len + 1 : 1;
        p.workgroups = static_cast<long long>(p.segs) * B * across;
        if (p.segs == 1 || p.workgroups <= 65536 || p.workgroups <= 16 * (rows / p.seg_len + B) * across) break;
    }
    return p;
}

hipError_t launch_conv(const ConvArgs& a, void* out, void* state_out, bool f32, hipStream_t stream) {
    return by_taps(a.W, f32, [&](auto w, auto wide) {
        const int across = across_of(a);
        hipLaunchKernelGGL((conv_kernel<decltype(w)::value, decltype(wide)::value, kConvGroup>), dim3(static_cast<unsigned>(a.segs) * a.B * across), dim3(kConvThreads),
                           0, stream, a, static_cast<char*>(out), static_cast<char*>(state_out), across, a.seg_len / (kConvThreads / a.lanes));
        return hipGetLastError();
    });
}

hipError_t launch_conv_step(const ConvArgs& a, void* out, void* state_out, bool f32, hipStream_t stream) {
    return by_taps(a.W, f32, [&](auto w, auto wide) {
        const int groups = a.D / kConvStepGroup;
        const long long items = static_cast<long long>(groups) * a.B;
        hipLaunchKernelGGL((conv_step_kernel<decltype(w)::value, decltype(wide)::value, kConvStepGroup>), dim3(static_cast<unsigned>((items + kConvThreads - 1) / kConvThreads)),
                           dim3(kConvThreads), 0, stream, a, static_cast<char*>(out), static_cast<char*>(state_out), groups);
        return hipGetLastError();
    });
}

hipError_t launch_conv_backward(const ConvArgs& a, const void* dout, const void* dstate_out, void* dx, float* dw, float* dbias, void* dstate_in,
                                float* partials, bool f32, hipStream_t stream) {
    const int across = across_of(a);
    const hipError_t err = by_taps(a.W, f32, [&](auto w, auto wide) {
        hipLaunchKernelGGL((conv_backward_kernel<decltype(w)::value, decltype(wide)::value, kConvGroup>), dim3(static_cast<unsigned>(a.segs) * a.B * across),
                           dim3(kConvThreads), 0, stream, a, static_cast<const char*>(dout), static_cast<const char*>(dstate_out), static_cast<char*>(dx),
                           static_cast<char*>(dstate_in), dw ? partials : nullptr,
                           static_cast<unsigned>(whole_places(a.rows, a.segs, a.seg_len)), across, a.seg_len / (kConvThreads / a.lanes));
        return hipGetLastError();
    });
    return err != hipSuccess || !dw ? err : launch_conv_fold(a, dw, dbias, partials, stream);
}

hipError_t launch_conv_fold(const ConvArgs& a, float* dw, float* dbias, const float* partials, hipStream_t stream) {
    hipLaunchKernelGGL(conv_fold_kernel, dim3((static_cast<unsigned>(a.D) * (a.W + 1) + 63) / 64), dim3(64 * kFoldTurns), 0, stream, a.D, a.W,
                       share_places(a.B, a.rows, a.segs, a.seg_len, a.offsets != nullptr), partials, dw, dbias);
    return hipGetLastError();
}

}  // namespace wkv6
