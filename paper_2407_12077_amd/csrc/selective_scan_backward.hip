// The gradients of the selective scan, for gfx950.  With dy = dout silu(z) and G_t the gradient of the state behind token t,
//
//     G_t[n] = c_t[n] dy_t + exp(dt_{t+1} a[n]) G_{t+1}[n]        k_t[n] = G_t[n] exp(dt_t a[n]) h_{t-1}[n]        g_t = sum_n G_t[n] b_t[n]
//     dx = g dt + skip dy    ddelta = (g x + sum_n k[n] a[n]) dt'    db[n] = sum_d G[n] dt x    dc[n] = sum_d dy h[n]    da[n] = sum_t k[n] dt
#include "selective_scan_tiles.h"

namespace wkv6 {
namespace {

using namespace scan;

constexpr float kLn2 = 0.6931471805599453f;

// Sums over lanes: two values become one register with half of the lanes' sums each.  halves<32>: lanes below 32 have p's, the others q's.
template <int kBy>
__device__ __forceinline__ float halves(float p, float q, int lane) {
    if constexpr (kBy == 32 || kBy == 16) {
        const auto r = kBy == 32 ? __builtin_amdgcn_permlane32_swap(__float_as_uint(p), __float_as_uint(q), false, false)
                                 : __builtin_amdgcn_permlane16_swap(__float_as_uint(p), __float_as_uint(q), false, false);
        return __uint_as_float(r[0]) + __uint_as_float(r[1]);
    } else {
        // in a row of sixteen lanes: turned by eight; mirrored in eight; pairs, neighbours exchanged
        constexpr int kControl = kBy == 8 ? 0x128 : kBy == 4 ? 0x141 : kBy == 2 ? 0x4e : 0xb1;
        const float keep = lane & kBy ? q : p, give = lane & kBy ? p : q;
        return keep + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(give), kControl, 0xf, 0xf, true));
    }
}

template <int N>
struct Shape {
    static constexpr int kGroups = N == 64 ? 2 : 1;            // of four states a lane
    static constexpr int kStates = 4 * kGroups, kWaves = N / kStates, kThreads = 64 * kWaves;
    static constexpr int kC = scan_back_chunk(N);
    static constexpr int kPer = kC * kScanChannels / kThreads, kAcross = kScanChannels / kPer;
};

// Rows of a chunk that a thread brings: channels own .. own + kPer - 1 of one token.
template <bool kF32, int kPer>
struct Element {
    Raw<kF32, kPer> x, delta, z, dout;
};

// What a segment hands to the one in front of it if it gets nothing from behind, and the sum of its step sizes.
template <int N, bool kF32>
__global__ __launch_bounds__(16 * N) void scan_behind_kernel(ScanArgs a, const char* dout, float* behind, int blocks) {
    constexpr int kWaves = N / 4, kC = kScanChunk, kCh = kScanChannels, kItem = kF32 ? 4 : 2;
    constexpr int kPer = kC / kWaves < 8 ? kC / kWaves : 8, kAcross = kCh / kPer;
    __shared__ float2v step[2][kC][kCh];                       // dt, dy
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int block = blockIdx.x % blocks, at = blockIdx.x / blocks, b = at % a.B, seg = 1 + at / a.B;
    const Span span = span_of(a, b, seg);
    if (span.tokens == 0) return;
    const int D = a.D, c0 = block * kCh, ch = c0 + lane, n0 = 4 * wave;
    const bool mine = ch < D;
    float4v rate = {0.f, 0.f, 0.f, 0.f}, g = {0.f, 0.f, 0.f, 0.f};
    if (mine) rate = *reinterpret_cast<const float4v*>(a.a + static_cast<long long>(ch) * N + n0) * kLog2e;
    const int token = threadIdx.x / kAcross, own = c0 + threadIdx.x % kAcross * kPer, in_block = own - c0;
    const bool there = own < D;
    float bias[kPer], dt_sum = 0.f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) bias[i] = there && a.bias ? a.bias[own + i] : 0.f;
    const char *delta = static_cast<const char*>(a.delta), *z = static_cast<const char*>(a.z), *cp = static_cast<const char*>(a.c) + n0 * kItem;
    struct Chunk {
        Raw<kF32, kPer> delta, z, dout;
        StateRow<kF32> c;
    };
    auto ask = [&](int first, Chunk& k) {
        k.delta.none();
        k.z.none();
        k.dout.none();
        if (there && first >= 0 && first + token < span.tokens) {
            const long long row = span.first_row + first + token;
            k.delta.load(delta + row * a.delta_row + own * kItem);
            if (z) k.z.load(z + row * a.z_row + own * kItem);
            k.dout.load(dout + (row * D + own) * kItem);
        }
        k.c.none();
        if (first >= 0 && first + lane / 4 < span.tokens) k.c.raw.load(cp + (span.first_row + first + lane / 4) * a.bc_row);
    };
    auto bring = [&](int first, const Chunk& k, int buffer) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            float dt = step_of(k.delta[i] + bias[i], a.softplus), dy = k.dout[i];
            if (first + token >= span.tokens) dt = 0.f;
            if (z) dy *= k.z[i] * sigmoid_of(k.z[i]);
            step[buffer][token][in_block + i] = float2v{dt, dy};
        }
    };
    Chunk now, next;
    int first = (span.tokens - 1) / kC * kC, buffer = 0;
    ask(first, now);
    bring(first, now, 0);
    __syncthreads();
    for (; first >= 0; first -= kC, buffer ^= 1) {
        ask(first - kC, next);
        const float cv = now.c.plain(lane);
        each<kC>([&](auto back) {
            constexpr int t = kC - 1 - decltype(back)::value;
            const float2v d = step[buffer][t][lane];
            g = outer<t>(cv, d.y, g);
#pragma unroll
            for (int i = 0; i < 4; ++i) g[i] *= __builtin_amdgcn_exp2f(d.x * rate[i]);
            dt_sum += d.x;
        });
        bring(first - kC, next, buffer ^ 1);
        __syncthreads();
        now = next;
    }
    if (!mine) return;
    const long long seg_states = static_cast<long long>(a.B) * D * N, unit = (static_cast<long long>(b) * D + ch) * N + n0;
    *reinterpret_cast<float4v*>(behind + seg * seg_states + unit) = g;
    if (wave == 0) behind[a.segs * seg_states + (static_cast<long long>(seg) * a.B + b) * D + ch] = dt_sum;
}

template <int N, bool kF32>
__global__ __launch_bounds__(Shape<N>::kThreads) void scan_backward_kernel(ScanArgs a, ScanGradients r, int blocks) {
    using S = Shape<N>;
    constexpr int kG = S::kGroups, kWaves = S::kWaves, kC = S::kC, kCh = kScanChannels, kPer = S::kPer, kItem = kF32 ? 4 : 2;
    __shared__ float4v step[kC][kCh];                          // dt, dt x, dy
    __shared__ float part[3][kWaves][kC][kCh];                 // shares of g, of sum k rate, of the read-outs
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int block = blockIdx.x % blocks, at = blockIdx.x / blocks, b = at % a.B, seg = at / a.B;
    const Span span = span_of(a, b, seg);
    if (span.tokens == 0 && seg > 0) return;
    const int D = a.D, c0 = block * kCh, ch = c0 + lane, n0 = S::kStates * wave;
    const bool mine = ch < D, gate = a.z != nullptr;
    const long long unit = (static_cast<long long>(b) * D + ch) * N + n0, seg_states = static_cast<long long>(a.B) * D * N;
    const long long sums_at = a.segs * seg_states, seg_sums = static_cast<long long>(a.B) * D, channel = static_cast<long long>(b) * D + ch;

    float4v rate[kG], h[kG], grad[kG], da[kG];
#pragma unroll
    for (int q = 0; q < kG; ++q) rate[q] = h[q] = grad[q] = da[q] = float4v{0.f, 0.f, 0.f, 0.f};
    if (mine) {
#pragma unroll
        for (int q = 0; q < kG; ++q) {
            rate[q] = *reinterpret_cast<const float4v*>(a.a + static_cast<long long>(ch) * N + n0 + 4 * q) * kLog2e;
            if (a.segs > 1) h[q] = *reinterpret_cast<const float4v*>(a.locals + unit + 4 * q);
            else if (a.state_in) h[q] = *reinterpret_cast<const float4v*>(a.state_in + unit + 4 * q);
            if (r.dstate_out) grad[q] = *reinterpret_cast<const float4v*>(r.dstate_out + unit + 4 * q);
        }
        for (int s = 1; s <= seg; ++s) {
            const float sum = a.locals[sums_at + s * seg_sums + channel];
#pragma unroll
            for (int q = 0; q < kG; ++q) {
                const float4v local = *reinterpret_cast<const float4v*>(a.locals + s * seg_states + unit + 4 * q);
#pragma unroll
                for (int i = 0; i < 4; ++i) h[q][i] = __builtin_fmaf(__builtin_amdgcn_exp2f(sum * rate[q][i]), h[q][i], local[i]);
            }
        }
        if (a.segs > 1 && !span.last) {
            for (int s = a.segs - 1; s > seg; --s) {
                if (span_of(a, b, s).tokens == 0) continue;
                const float sum = r.behind[sums_at + s * seg_sums + channel];
#pragma unroll
                for (int q = 0; q < kG; ++q) {
                    const float4v local = *reinterpret_cast<const float4v*>(r.behind + s * seg_states + unit + 4 * q);
#pragma unroll
                    for (int i = 0; i < 4; ++i) grad[q][i] = __builtin_fmaf(__builtin_amdgcn_exp2f(sum * rate[q][i]), grad[q][i], local[i]);
                }
            }
        }
    }

    const int token = threadIdx.x / S::kAcross, own = c0 + threadIdx.x % S::kAcross * kPer, in_block = own - c0;
    const bool there = own < D;
    float bias[kPer], skip[kPer], dskip[kPer], dbias[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        bias[i] = there && a.bias ? a.bias[own + i] : 0.f;
        skip[i] = there && a.skip ? a.skip[own + i] : 0.f;
        dskip[i] = dbias[i] = 0.f;
    }
    const char *x = static_cast<const char*>(a.x), *delta = static_cast<const char*>(a.delta), *z = static_cast<const char*>(a.z);
    const char *bp = static_cast<const char*>(a.b) + n0 * kItem, *cp = static_cast<const char*>(a.c) + n0 * kItem, *dout = static_cast<const char*>(r.dout);
    struct Chunk {
        Element<kF32, kPer> e;
        StateRow<kF32> b[kG], c[kG];
    };
    auto ask = [&](int first, Chunk& k, bool back) {
        k.e.x.none();
        k.e.delta.none();
        k.e.z.none();
        k.e.dout.none();
        if (there && first >= 0 && first + token < span.tokens) {
            const long long row = span.first_row + first + token;
            k.e.x.load(x + row * a.x_row + own * kItem);
            k.e.delta.load(delta + row * a.delta_row + own * kItem);
            if (back) {
                if (gate) k.e.z.load(z + row * a.z_row + own * kItem);
                k.e.dout.load(dout + (row * D + own) * kItem);
            }
        }
#pragma unroll
        for (int q = 0; q < kG; ++q) {
            k.b[q].none();
            k.c[q].none();
        }
        if (lane / 4 < kC && first >= 0 && first + lane / 4 < span.tokens) {
            const long long row = span.first_row + first + lane / 4;
#pragma unroll
            for (int q = 0; q < kG; ++q) {
                k.b[q].raw.load(bp + row * a.bc_row + 4 * q * kItem);
                if (back) k.c[q].raw.load(cp + row * a.bc_row + 4 * q * kItem);
            }
        }
    };
    auto bring = [&](int first, const Chunk& k) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            float dt = step_of(k.e.delta[i] + bias[i], a.softplus), dy = k.e.dout[i];
            if (first + token >= span.tokens) dt = 0.f;
            if (gate) dy *= k.e.z[i] * sigmoid_of(k.e.z[i]);
            step[token][in_block + i] = float4v{dt, dt * k.e.x[i], dy, 0.f};
        }
    };

    // the states in front of the chunks
    const int last_first = span.tokens > 0 ? (span.tokens - 1) / kC * kC : 0;
    const long long place0 = (span.first_row - static_cast<long long>(seg) * a.seg_len) / kC + static_cast<long long>(seg) * a.seg_len / kC + b;
    float* const kept = r.states + (place0 * D + ch) * N + n0;
    const long long kept_step = static_cast<long long>(D) * N;
    Chunk now, next;
    ask(0, now, false);
    for (int first = 0; first < last_first; first += kC) {
        bring(first, now);
        __syncthreads();
        ask(first + kC, next, false);
        if (mine) {
#pragma unroll
            for (int q = 0; q < kG; ++q) *reinterpret_cast<float4v*>(kept + first / kC * kept_step + 4 * q) = h[q];
        }
        float bv[kG];
#pragma unroll
        for (int q = 0; q < kG; ++q) bv[q] = now.b[q].plain(lane);
        each<kC>([&](auto token_of_chunk) {
            constexpr int t = decltype(token_of_chunk)::value;
            const float4v d = step[t][lane];
#pragma unroll
            for (int q = 0; q < kG; ++q) {
                float4v decayed;
#pragma unroll
                for (int i = 0; i < 4; ++i) decayed[i] = __builtin_amdgcn_exp2f(d.x * rate[q][i]) * h[q][i];
                h[q] = outer<t>(bv[q], d.y, decayed);
            }
        });
        __syncthreads();
        now = next;
    }

    // and back
    ask(span.tokens > 0 ? last_first : -1, now, true);
    for (int first = last_first; first >= 0 && span.tokens > 0; first -= kC) {
        bring(first, now);
        if (first < last_first && mine) {
#pragma unroll
            for (int q = 0; q < kG; ++q) h[q] = *reinterpret_cast<const float4v*>(kept + first / kC * kept_step + 4 * q);
        }
        __syncthreads();
        ask(first - kC, next, true);
        float4v decay[kC][kG], left[kC][kG];                   // exp(dt a), and that times the state in front
        float bv[kG], cv[kG];
        {
            float ct[kG][4];
#pragma unroll
            for (int q = 0; q < kG; ++q) {
                bv[q] = now.b[q].plain(lane);
                cv[q] = now.c[q].plain(lane);
#pragma unroll
                for (int i = 0; i < 4; ++i) ct[q][i] = now.c[q].at_token(i, lane);
            }
            float4v y = {0.f, 0.f, 0.f, 0.f};
            each<kC>([&](auto token_of_chunk) {
                constexpr int t = decltype(token_of_chunk)::value;
                const float4v d = step[t][lane];
#pragma unroll
                for (int q = 0; q < kG; ++q) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        decay[t][q][i] = __builtin_amdgcn_exp2f(d.x * rate[q][i]);
                        left[t][q][i] = decay[t][q][i] * h[q][i];
                    }
                    h[q] = outer<t>(bv[q], d.y, left[t][q]);
                    if (gate) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) y = outer<t>(ct[q][i], h[q][i], y);
                    }
                }
                if constexpr (t % 4 == 3) {
                    if (gate) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) part[2][wave][t - 3 + i][lane] = y[i];
                        y = float4v{0.f, 0.f, 0.f, 0.f};
                    }
                }
            });
        }
        float bt[kG][4];
#pragma unroll
        for (int q = 0; q < kG; ++q)
#pragma unroll
            for (int i = 0; i < 4; ++i) bt[q][i] = now.b[q].at_token(i, lane);
        float4v into = {0.f, 0.f, 0.f, 0.f}, da_chunk[kG];
        float pairs[kG][2], fours[kG], eights[kG];             // sums over lanes on their way: of one odd token, of two, of four
#pragma unroll
        for (int q = 0; q < kG; ++q) da_chunk[q] = float4v{0.f, 0.f, 0.f, 0.f};
        each<kC>([&](auto back) {
            constexpr int t = kC - 1 - decltype(back)::value;
            const float4v d = step[t][lane];
            float k_rate = 0.f;
#pragma unroll
            for (int q = 0; q < kG; ++q) {
                const float4v state = outer<t>(bv[q], d.y, left[t][q]);
                grad[q] = outer<t>(cv[q], d.z, grad[q]);
                float v[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] = grad[q][i] * d.y;
                    v[4 + i] = state[i] * d.z;
                    const float k = grad[q][i] * left[t][q][i];
                    da_chunk[q][i] = __builtin_fmaf(k, d.x, da_chunk[q][i]);
                    k_rate = __builtin_fmaf(k, rate[q][i], k_rate);
                    into = outer<t>(bt[q][i], grad[q][i], into);
                }
                // lane: value of v by its bits 32, 16, 8, then the token by bits 4, 2, 1
                const float m0 = halves<32>(v[0], v[4], lane), m1 = halves<32>(v[1], v[5], lane), m2 = halves<32>(v[2], v[6], lane),
                            m3 = halves<32>(v[3], v[7], lane);
                const float one = halves<8>(halves<16>(m0, m2, lane), halves<16>(m1, m3, lane), lane);
                if constexpr (t % 2 == 1) {
                    pairs[q][0] = one;
                } else {
                    const float two = halves<4>(one, pairs[q][0], lane);
                    if constexpr (t % 4 == 2) {
                        fours[q] = two;
                    } else {
                        const float four = halves<2>(two, fours[q], lane);
                        if constexpr (t % 8 == 4) {
                            eights[q] = four;
                        } else {
                            const float sum = halves<1>(four, eights[q], lane);
                            const int which = lane >> 5, n = (lane >> 4 & 1) * 2 + (lane >> 3 & 1);
                            const int at_token = first + t + (lane >> 2 & 1) + (lane & 2) + (lane & 1) * 4;
                            if (at_token < span.tokens)
                                r.rows[((span.first_row + at_token) * blocks + block) * (2 * N) + which * N + n0 + 4 * q + n] = sum;
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) grad[q][i] *= decay[t][q][i];
            }
            part[1][wave][t][lane] = k_rate;
            if constexpr (t % 4 == 0) {
#pragma unroll
                for (int i = 0; i < 4; ++i) part[0][wave][t + i][lane] = into[i];
                into = float4v{0.f, 0.f, 0.f, 0.f};
            }
        });
#pragma unroll
        for (int q = 0; q < kG; ++q) da[q] += da_chunk[q];
        __syncthreads();
        if (there && first + token < span.tokens) {
            const long long row = span.first_row + first + token;
            float dx[kPer], dd[kPer], dz[kPer];
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                float g = 0.f, k = 0.f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    g += part[0][w][token][in_block + i];
                    k += part[1][w][token][in_block + i];
                }
                const float4v d = step[token][in_block + i];
                const float xv = now.e.x[i];
                dx[i] = __builtin_fmaf(g, d.x, skip[i] * d.z);
                dd[i] = __builtin_fmaf(g, xv, k * kLn2);
                if (a.softplus) dd[i] *= sigmoid_of(now.e.delta[i] + bias[i]);
                dskip[i] = __builtin_fmaf(d.z, xv, dskip[i]);
                dbias[i] += dd[i];
                if (gate) {
                    float y = skip[i] * xv;
#pragma unroll
                    for (int w = 0; w < kWaves; ++w) y += part[2][w][token][in_block + i];
                    const float zv = now.e.z[i], s = sigmoid_of(zv);
                    dz[i] = now.e.dout[i] * y * (s * __builtin_fmaf(zv, 1.f - s, 1.f));
                }
            }
            store<kF32>(static_cast<char*>(r.dx) + row * a.x_row + own * kItem, dx);
            store<kF32>(static_cast<char*>(r.ddelta) + row * a.delta_row + own * kItem, dd);
            if (gate && r.dz) store<kF32>(static_cast<char*>(r.dz) + row * a.z_row + own * kItem, dz);
        }
        __syncthreads();
        now = next;
    }
    const long long share = static_cast<long long>(seg) * a.B + b;
    if (mine) {
#pragma unroll
        for (int q = 0; q < kG; ++q) {
            if (seg == 0 && r.dstate_in) *reinterpret_cast<float4v*>(r.dstate_in + unit + 4 * q) = grad[q];
            *reinterpret_cast<float4v*>(r.weights + (share * D + ch) * N + n0 + 4 * q) = da[q];
        }
    }
    // the tokens' shares of dskip and dbias meet
    float* const meet = &part[0][0][0][0];                     // [2][kC][kCh]
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        meet[token * kCh + in_block + i] = dskip[i];
        meet[(kC + token) * kCh + in_block + i] = dbias[i];
    }
    __syncthreads();
    if (threadIdx.x < 2 * kCh && c0 + (threadIdx.x & 63) < D) {
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < kC; ++t) sum += meet[((threadIdx.x >> 6) * kC + t) * kCh + lane];
        r.weights[a.segs * seg_states + (share * 2 + (threadIdx.x >> 6)) * D + ch] = sum;
    }
}

// db and dc of a row: the blocks' shares, in their order.
template <bool kF32>
__global__ __launch_bounds__(256) void scan_rows_kernel(ScanArgs a, const float* shares, char* db, char* dc, int blocks, int per) {
    const int N2 = 2 * a.N, value = threadIdx.x % N2;
    const long long row = static_cast<long long>(blockIdx.x) * per + threadIdx.x / N2;
    if (row >= a.rows) return;
    if (a.offsets) {                                           // rows of nobody keep what they hold
        long long lo = 0, hi = a.B;                            // the last sequence that starts at or in front of the row
        while (lo < hi) {
            const long long mid = (lo + hi) / 2;
            if (a.offsets[mid] <= row) lo = mid + 1;
            else hi = mid;
        }
        if (lo == 0) return;
        const long long first = a.offsets[lo - 1] < 0 ? 0 : a.offsets[lo - 1];
        if (row >= a.offsets[lo] || row - first >= a.T) return;
    }
    const float* p = shares + row * blocks * N2 + value;
    float sum = 0.f;
    for (int i = 0; i < blocks; ++i) sum += p[static_cast<long long>(i) * N2];
    const int n = value % a.N;
    const float v[1] = {sum};
    store<kF32>((value < a.N ? db : dc) + row * a.bc_row + n * (kF32 ? 4 : 2), v);
}

// da, dskip, dbias: the segments' shares in the order of sequences and segments.
__global__ __launch_bounds__(256) void scan_weights_kernel(ScanArgs a, const float* shares, float* da, float* dskip, float* dbias) {
    __shared__ float meet[4][64];
    const int lane = threadIdx.x & 63, turn = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long states = static_cast<long long>(a.D) * a.N, value = static_cast<long long>(blockIdx.x) * 64 + lane;
    const bool there = value < states + 2 * a.D;
    const float* from = value < states ? shares + value : shares + a.segs * a.B * states + (value - states);
    const long long stride = value < states ? states : 2 * a.D;
    float sum = 0.f;
    for (int b = turn; b < a.B; b += 4)
        for (int s = 0; s < a.segs; ++s) {
            if (s > 0 && span_of(a, b, s).tokens == 0) break;
            if (there) sum += from[(static_cast<long long>(s) * a.B + b) * stride];
        }
    meet[turn][lane] = sum;
    __syncthreads();
    if (turn != 0 || !there) return;
    sum = (meet[0][lane] + meet[1][lane]) + (meet[2][lane] + meet[3][lane]);
    if (value < states) {
        if (da) da[value] = sum;
    } else if (value < states + a.D) {
        if (dskip) dskip[value - states] = sum;
    } else if (dbias) {
        dbias[value - states - a.D] = sum;
    }
}

template <int N, bool kF32>
hipError_t launch(const ScanArgs& a, const ScanGradients& g, hipStream_t stream) {
    const int blocks = static_cast<int>(scan_blocks(a.D));
    const unsigned units = static_cast<unsigned>(blocks) * a.B;
    hipError_t err = hipSuccess;
    if (a.segs > 1) {
        err = launch_scan_states(a, kF32, stream);
        if (err != hipSuccess) return err;
        hipLaunchKernelGGL((scan_behind_kernel<N, kF32>), dim3(units * (a.segs - 1)), dim3(16 * N), 0, stream, a, static_cast<const char*>(g.dout), g.behind,
                           blocks);
        if ((err = hipGetLastError()) != hipSuccess) return err;
    }
    hipLaunchKernelGGL((scan_backward_kernel<N, kF32>), dim3(units * a.segs), dim3(Shape<N>::kThreads), 0, stream, a, g, blocks);
    if ((err = hipGetLastError()) != hipSuccess) return err;
    if (a.rows > 0 && a.T > 0) {
        const int per = 256 / (2 * N);
        hipLaunchKernelGGL((scan_rows_kernel<kF32>), dim3(static_cast<unsigned>((a.rows + per - 1) / per)), dim3(256), 0, stream, a, g.rows,
                           static_cast<char*>(g.db), static_cast<char*>(g.dc), blocks, per);
        if ((err = hipGetLastError()) != hipSuccess) return err;
    }
    return launch_scan_weights(a, g, stream);
}

}  // namespace

hipError_t launch_scan_weights(const ScanArgs& a, const ScanGradients& g, hipStream_t stream) {
    if (!g.da && !g.dskip && !g.dbias) return hipSuccess;
    const long long values = static_cast<long long>(a.D) * (a.N + 2);
    hipLaunchKernelGGL(scan_weights_kernel, dim3(static_cast<unsigned>((values + 63) / 64)), dim3(256), 0, stream, a, g.weights, g.da, g.dskip, g.dbias);
    return hipGetLastError();
}

hipError_t launch_scan_backward(const ScanArgs& a, const ScanGradients& g, bool f32, hipStream_t stream) {
    auto go = [&](auto n) {
        constexpr int N = decltype(n)::value;
        return f32 ? launch<N, true>(a, g, stream) : launch<N, false>(a, g, stream);
    };
    switch (a.N) {
        case 8: return go(std::integral_constant<int, 8>());
        case 16: return go(std::integral_constant<int, 16>());
        case 32: return go(std::integral_constant<int, 32>());
        default: return go(std::integral_constant<int, 64>());
    }
}

}  // namespace wkv6
