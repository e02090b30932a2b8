// The gradients of the selective scan, for gfx950.  With dy = dout silu(z) and G_t the gradient of the state behind token t,
//
//     G_t[n] = c_t[n] dy_t + exp(dt_{t+1} a[n]) G_{t+1}[n]        k_t[n] = G_t[n] exp(dt_t a[n]) h_{t-1}[n]        g_t = sum_n G_t[n] b_t[n]
//     dx = g dt + skip dy    ddelta = (g x + sum_n k[n] a[n]) dt'    db[n] = sum_d G[n] dt x    dc[n] = sum_d dy h[n]    da[n] = sum_t k[n] dt
//
// Divided as the forward walk (selective_scan.hip) and bound by instruction slots like it: 8 x 2048 x 4096, N = 16, bf16 with a gate: 893 us, of which the folds are 23;
// a vector instruction issues in 93 % of the walk's cycles (1.952 M of 2.090 M of a SIMD, at 2.40 GHz 813 us); its bytes would take 180.  A workgroup walks its segment forwards once, leaving the
// state in front of every chunk in the workspace (a quarter of the work), and back: a chunk's decays and states are formed again and stay in
// registers, 16 tokens of both (8 of many states), for the way from its last token to its first.  k needs no product of its own, as G exp(dt a) is what
// the token in front takes over.  db and dc are sums over channels, that is over lanes: products are added in pairs, each pair in one register with half
// of the lanes' sums, so that eight tokens' sixty-four values end as one register, after 141 instructions (a quarter of the way back).  Letting
// lanes exchange factors in front of the products saved instructions on paper and cost copies: 976 us.  da is summed by chunks,
// dskip and dbias by every sixteenth (or eighth) token of a segment, and the workgroups' sums are folded in a fixed order.
#include "selective_scan_tiles.h"

namespace wkv6 {
namespace {

using namespace scan;

constexpr float kLn2 = 0.6931471805599453f;

// Sums over lanes: two values become one register with half of the lanes' sums each.  halves<32>: lanes below 32 have p's, the others q's; and so
// on inside the halves.
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

struct BackwardArgs {
    ScanArgs a;
    ScanGradients r;
    int blocks;
};

// A kernel's only argument once more, as it lies in memory: what is needed at the end only would else stay in scalar registers, of which there are
// too few: 94 were spilled, now 3 to 15 (gradients of 8 x 2048 x 4096 914 -> 895 us, 1 x 512 x 2048 39.9 -> 37.2).
template <typename Args>
__device__ __forceinline__ const Args& argument_again() {
    auto at = __builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(at));
    return *(const Args*)at;
}

template <int N, bool kF32, bool kGate>
__global__ __launch_bounds__(Shape<N>::kThreads, 2) void scan_backward_kernel(BackwardArgs args) {
    using S = Shape<N>;
    const ScanArgs& a = args.a;
    const ScanGradients& r = args.r;
    const int blocks = args.blocks;
    constexpr int kG = S::kGroups, kWaves = S::kWaves, kC = S::kC, kCh = kScanChannels, kPer = S::kPer, kItem = kF32 ? 4 : 2;
    __shared__ float2v step[2][kC][kCh];                       // dt, dt x
    __shared__ float grad_out[2][kC][kCh];                     // dy
    __shared__ float part[kGate ? 3 : 2][kWaves][kC][kCh];     // shares of g, of sum k rate, of the read-outs
    __shared__ int in_front[kWaves];                           // segments of other sequences
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int block = blockIdx.x % blocks, at = blockIdx.x / blocks, b = at % a.B, seg = at / a.B;
    const Span span = span_of(a, b, seg);
    if (span.tokens == 0 && seg > 0) return;
    const int D = a.D, c0 = block * kCh, ch = c0 + lane, n0 = S::kStates * wave;
    const bool mine = ch < D;
    const long long unit = (static_cast<long long>(b) * D + ch) * N + n0, seg_states = static_cast<long long>(a.B) * D * N;
    const long long sums_at = a.segs * seg_states, seg_sums = static_cast<long long>(a.B) * D, channel = static_cast<long long>(b) * D + ch;

    float4v rate[kG], h[kG], grad[kG], da[kG];
#pragma unroll
    for (int q = 0; q < kG; ++q) rate[q] = h[q] = grad[q] = da[q] = float4v{0.f, 0.f, 0.f, 0.f};
    if (mine) {
        float4v third[kG];
#pragma unroll
        for (int q = 0; q < kG; ++q) {
            rate[q] = rate_of(a.a + static_cast<long long>(ch) * N + n0 + 4 * q);
            third[q] = rate[q] * (1.f / 3);
            if (a.segs > 1) h[q] = *reinterpret_cast<const float4v*>(a.locals + unit + 4 * q);
            else if (a.state_in) h[q] = *reinterpret_cast<const float4v*>(a.state_in + unit + 4 * q);
            if (r.dstate_out) grad[q] = *reinterpret_cast<const float4v*>(r.dstate_out + unit + 4 * q);
        }
#pragma unroll 4
        for (int s = 1; s <= seg; ++s) {
            const float sum = a.locals[sums_at + s * seg_sums + channel];
#pragma unroll
            for (int q = 0; q < kG; ++q) pass_on(h[q], sum, third[q], *reinterpret_cast<const float4v*>(a.locals + s * seg_states + unit + 4 * q));
        }
        if (!span.last) {
#pragma unroll 4
            for (int s = (tokens_of(a, b) - 1) / a.seg_len; s > seg; --s) {
                const float sum = r.behind[sums_at + s * seg_sums + channel];
#pragma unroll
                for (int q = 0; q < kG; ++q) pass_on(grad[q], sum, third[q], *reinterpret_cast<const float4v*>(r.behind + s * seg_states + unit + 4 * q));
            }
        }
    }

    const int token = threadIdx.x / S::kAcross, own = c0 + threadIdx.x % S::kAcross * kPer, in_block = own - c0;
    const bool there = own < D;
    const unsigned softplus = softplus_bits(a.softplus);
    float bias[kPer], skip[kPer], dskip[kPer], dbias[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        bias[i] = there && a.bias ? a.bias[own + i] : 0.f;
        skip[i] = there && a.skip ? a.skip[own + i] : 0.f;
        dskip[i] = dbias[i] = 0.f;
    }
    struct Chunk {
        Raw<kF32, kPer> x, delta, z, dout;
        float dt[kPer], dy[kPer];
        Plain<kF32> b[kG], c[kG];
        ByRow<kF32, kC / 4> bt[kG], ct[kG];
        float4v h[kG];
    };
    const int bc_row = static_cast<int>(a.bc_row);
    const int x_at = there ? token * static_cast<int>(a.x_row) + own * kItem : kNowhere;
    const int delta_at = there ? token * static_cast<int>(a.delta_row) + own * kItem : kNowhere;
    const int z_at = there ? token * static_cast<int>(a.z_row) + own * kItem : kNowhere;
    const int out_at = there ? (token * D + own) * kItem : kNowhere;
    const int kept_at = mine ? (ch * N + n0) * 4 : kNowhere;
    const long long row0 = span.first_row, out_row = static_cast<long long>(D) * kItem;
    Rows xs(a.x, row0, a.x_row), deltas(a.delta, row0, a.delta_row), bs(a.b, row0, a.bc_row), kept(r.states, chunk_place(row0, kC), static_cast<long long>(D) * N * 4);
    auto bring = [&](int first, Chunk& k, int buffer, auto on_the_way_back) {
        steps_of(k.delta, bias, softplus, k.dt);
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            k.dt[i] = first + token < span.tokens ? k.dt[i] : 0.f;
            step[buffer][token][in_block + i] = float2v{k.dt[i], k.dt[i] * k.x[i]};
            if constexpr (decltype(on_the_way_back)::value) {
                k.dy[i] = k.dout[i];
                if constexpr (kGate) k.dy[i] *= k.z[i] * sigmoid_of(k.z[i]);
                grad_out[buffer][token][in_block + i] = k.dy[i];
            }
        }
    };
    constexpr std::true_type kBackward{};
    constexpr std::false_type kForward{};

    // the states in front of the chunks
    const int last_first = span.tokens > 0 ? (span.tokens - 1) / kC * kC : -kC;
    Chunk now, next;
    int buffer = 0;
    {
        auto ask = [&](int left, Chunk& k) {
            const int count = rows_of<kC>(left);
            k.x.load(xs.first(count), x_at);
            k.delta.load(deltas.first(count), delta_at);
#pragma unroll
            for (int q = 0; q < kG; ++q) k.b[q].load(bs.first(count), lane, bc_row, n0 + 4 * q);
            xs.move(kC);
            deltas.move(kC);
            bs.move(kC);
        };
        ask(span.tokens, now);
        bring(0, now, 0, kForward);
        for (int first = 0; first < last_first; first += kC, buffer ^= 1) {
            __syncthreads();
            __builtin_amdgcn_s_setprio(3);
            ask(span.tokens - first - kC, next);
#pragma unroll
            for (int q = 0; q < kG; ++q) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uint4v, h[q]), kept.first(1), kept_at + 16 * q, 0, 0);
            kept.move(1);
            each<kC>([&](auto token_of_chunk) {
                constexpr int t = decltype(token_of_chunk)::value;
                const float2v d = step[buffer][t][lane];
#pragma unroll
                for (int q = 0; q < kG; ++q) {
                    const float4v add = outer<t>(now.b[q].value(), d.y);
#pragma unroll
                    for (int i = 0; i < 4; ++i) h[q][i] = __builtin_fmaf(__builtin_amdgcn_exp2f(d.x * rate[q][i]), h[q][i], add[i]);
                }
                if constexpr (t == 3) __builtin_amdgcn_s_setprio(2);
                if constexpr (t == 7) __builtin_amdgcn_s_setprio(1);
            });
            __builtin_amdgcn_s_setprio(0);
            bring(first + kC, next, buffer ^ 1, kForward);
            now = next;
        }
        __syncthreads();
    }

    // and back
    xs = Rows(a.x, row0 + last_first, a.x_row);
    deltas = Rows(a.delta, row0 + last_first, a.delta_row);
    bs = Rows(a.b, row0 + last_first, a.bc_row);
    Rows zs(a.z, row0 + last_first, a.z_row), douts(r.dout, row0 + last_first, out_row), cs(a.c, row0 + last_first, a.bc_row);
    Rows dxs(r.dx, row0 + last_first, a.x_row), ddeltas(r.ddelta, row0 + last_first, a.delta_row), dzs(r.dz, row0 + last_first, a.z_row);
    Rows shares(r.rows, row0 + last_first, static_cast<long long>(blocks) * 2 * N * 4);
    const int share_token = (lane >> 2 & 1) + (lane & 2) + (lane & 1) * 4;
    const int share_at = share_token * shares.row + (block * 2 * N + (lane >> 5) * N + n0 + (lane >> 4 & 1) * 2 + (lane >> 3 & 1)) * 4;
    auto ask = [&](int at, Chunk& k) {                         // chunks in falling order
        const int count = at < 0 ? 0 : rows_of<kC>(span.tokens - at);
        k.x.load(xs.first(count), x_at);
        k.delta.load(deltas.first(count), delta_at);
        if constexpr (kGate) k.z.load(zs.first(count), z_at);
        k.dout.load(douts.first(count), out_at);
        kept.move(-1);
        const __amdgpu_buffer_rsrc_t b_rows = bs.first(count), c_rows = cs.first(count), states = kept.first(at < 0 ? 0 : 1);
#pragma unroll
        for (int q = 0; q < kG; ++q) {
            k.b[q].load(b_rows, lane, bc_row, n0 + 4 * q);
            k.c[q].load(c_rows, lane, bc_row, n0 + 4 * q);
            k.bt[q].load(b_rows, lane, bc_row, n0 + 4 * q);
            if constexpr (kGate) k.ct[q].load(c_rows, lane, bc_row, n0 + 4 * q);
            k.h[q] = __builtin_bit_cast(float4v, __builtin_amdgcn_raw_buffer_load_b128(states, kept_at + 16 * q, 0, 0));
        }
        xs.move(-kC);
        deltas.move(-kC);
        zs.move(-kC);
        douts.move(-kC);
        bs.move(-kC);
        cs.move(-kC);
    };
    kept.move(1);
    ask(last_first, now);                                      // (its states are in registers: what is read there is not used)
#pragma unroll
    for (int q = 0; q < kG; ++q) now.h[q] = h[q];
    buffer = 0;
    bring(last_first, now, 0, kBackward);
    for (int first = last_first; first >= 0; first -= kC, buffer ^= 1) {
        __syncthreads();
        __builtin_amdgcn_s_setprio(3);
        ask(first - kC, next);
        float4v decay[kC][kG], state[kC + 1][kG];              // exp(dt a), and the states: state[t] in front of token t
#pragma unroll
        for (int q = 0; q < kG; ++q) state[0][q] = now.h[q];
        each<kC>([&](auto token_of_chunk) {
            constexpr int t = decltype(token_of_chunk)::value;
            const float2v d = step[buffer][t][lane];
            float y = 0.f;
#pragma unroll
            for (int q = 0; q < kG; ++q) {
                const float4v add = outer<t>(now.b[q].value(), d.y);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    decay[t][q][i] = __builtin_amdgcn_exp2f(d.x * rate[q][i]);
                    state[t + 1][q][i] = __builtin_fmaf(decay[t][q][i], state[t][q][i], add[i]);
                }
                if constexpr (kGate) {
                    const float share = read_out<t % 4>(now.ct[q].value(t / 4), state[t + 1][q], state[t + 1][q][0]);
                    y = q == 0 ? share : y + share;
                }
            }
            if constexpr (kGate) part[2][wave][t][lane] = y;
        });
        __builtin_amdgcn_s_setprio(2);
        const int count = rows_of<kC>(span.tokens - first);
        float4v da_chunk[kG];
        float pairs[kG], fours[kG], eights[kG];                // sums over lanes on their way: of one odd token, of two, of four
#pragma unroll
        for (int q = 0; q < kG; ++q) da_chunk[q] = float4v{0.f, 0.f, 0.f, 0.f};
        each<kC>([&](auto back) {
            constexpr int t = kC - 1 - decltype(back)::value;
            const float2v d = step[buffer][t][lane];
            const float dy = grad_out[buffer][t][lane];
            float k_rate = 0.f, into = 0.f;
#pragma unroll
            for (int q = 0; q < kG; ++q) {
                grad[q] = outer<t>(now.c[q].value(), dy, grad[q]);
                float v[8];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    v[i] = grad[q][i] * d.y;
                    v[4 + i] = state[t + 1][q][i] * dy;
                }
                const float share = read_out<t % 4>(now.bt[q].value(t / 4), grad[q], v[0]);
                into = q == 0 ? share : into + share;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    grad[q][i] *= decay[t][q][i];
                    const float k = grad[q][i] * state[t][q][i];
                    da_chunk[q][i] = __builtin_fmaf(k, d.x, da_chunk[q][i]);
                    k_rate = __builtin_fmaf(k, rate[q][i], k_rate);
                }
                // lane: value of v by its bits 32, 16, 8, then the token by bits 4, 2, 1
                const float m0 = halves<32>(v[0], v[4], lane), m1 = halves<32>(v[1], v[5], lane), m2 = halves<32>(v[2], v[6], lane),
                            m3 = halves<32>(v[3], v[7], lane);
                const float one = halves<8>(halves<16>(m0, m2, lane), halves<16>(m1, m3, lane), lane);
                if constexpr (t % 2 == 1) {
                    pairs[q] = one;
                } else {
                    const float two = halves<4>(one, pairs[q], lane);
                    if constexpr (t % 4 == 2) {
                        fours[q] = two;
                    } else {
                        const float four = halves<2>(two, fours[q], lane);
                        if constexpr (t % 8 == 4) {
                            eights[q] = four;
                        } else {
                            const float sum = halves<1>(four, eights[q], lane);
                            __builtin_amdgcn_raw_buffer_store_b32(__float_as_uint(sum), shares.first(count), share_at + t * shares.row + 16 * q, 0, 0);
                        }
                    }
                }
            }
            part[0][wave][t][lane] = into;
            part[1][wave][t][lane] = k_rate;
            if constexpr (t % 4 == 0) {                        // (else the compiler keeps the k of all tokens for the end)
#pragma unroll
                for (int q = 0; q < kG; ++q)
#pragma unroll
                    for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(da_chunk[q][i]));
            }
            if constexpr (t == kC / 2) __builtin_amdgcn_s_setprio(1);
        });
        shares.move(-kC);
#pragma unroll
        for (int q = 0; q < kG; ++q) da[q] += da_chunk[q];
        bring(first - kC, next, buffer ^ 1, kBackward);
        __syncthreads();
        __builtin_amdgcn_s_setprio(3);
        {
            float dx[kPer], dd[kPer], dz[kPer];
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                float g = 0.f, k = 0.f;
#pragma unroll
                for (int w = 0; w < kWaves; ++w) {
                    g += part[0][w][token][in_block + i];
                    k += part[1][w][token][in_block + i];
                }
                const float xv = now.x[i];
                dx[i] = __builtin_fmaf(g, now.dt[i], skip[i] * now.dy[i]);
                dd[i] = __builtin_fmaf(g, xv, k * kLn2);
                const float slope = sigmoid_of(now.delta[i] + bias[i]);
                dd[i] *= chosen(softplus, slope, 1.f);
                dskip[i] = __builtin_fmaf(now.dy[i], xv, dskip[i]);
                dbias[i] += first + token < span.tokens ? dd[i] : 0.f;       // (behind the end k is not nought)
                if constexpr (kGate) {
                    float y = skip[i] * xv;
#pragma unroll
                    for (int w = 0; w < kWaves; ++w) y += part[2][w][token][in_block + i];
                    const float zv = now.z[i], s = sigmoid_of(zv);
                    dz[i] = now.dout[i] * y * (s * __builtin_fmaf(zv, 1.f - s, 1.f));
                }
            }
            store<kF32>(dxs.first(count), x_at, dx);
            store<kF32>(ddeltas.first(count), delta_at, dd);
            if (kGate && r.dz) store<kF32>(dzs.first(count), z_at, dz);
            dxs.move(-kC);
            ddeltas.move(-kC);
            dzs.move(-kC);
        }
        now = next;
    }
    __builtin_amdgcn_s_setprio(0);
    const BackwardArgs& end = argument_again<BackwardArgs>();
    const ScanArgs& call = end.a;
    const ScanGradients& to = end.r;
    const bool counts = counts_segments(call);
    const int others = counts ? segments_in_front<S::kThreads>(call, b) : 0;
    __syncthreads();
    // the tokens' shares of dskip and dbias meet
    float* const meet = &part[0][0][0][0];                     // [2][kC][kCh]
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        meet[token * kCh + in_block + i] = dskip[i];
        meet[(kC + token) * kCh + in_block + i] = dbias[i];
    }
    if (lane == 0) in_front[wave] = others;
    __syncthreads();
    if (call.offsets && block == 0) {
        const Span rows = span_of(call, b, seg);
        for (int t = threadIdx.x; t < rows.tokens; t += S::kThreads) to.owners[rows.first_row + t] = b;
    }
    if (!mine) return;
    if (seg == 0 && to.dstate_in) {
#pragma unroll
        for (int q = 0; q < kG; ++q) *reinterpret_cast<float4v*>(to.dstate_in + unit + 4 * q) = grad[q];
    }
    long long share = static_cast<long long>(b) * call.segs + seg;
    if (counts) {
        share = seg;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) share += in_front[w];
        if (b == call.B - 1 && seg == 0 && block == 0 && threadIdx.x == 0) *to.used = share + segments_of(tokens_of(call, b), call.seg_len);
    }
    if (share >= to.places) return;                            // (sequences that overlap)
#pragma unroll
    for (int q = 0; q < kG; ++q) *reinterpret_cast<float4v*>(to.weights + (share * D + ch) * N + n0 + 4 * q) = da[q];
    if (threadIdx.x < 2 * kCh) {
        float sum = 0.f;
#pragma unroll
        for (int t = 0; t < kC; ++t) sum += meet[((threadIdx.x >> 6) * kC + t) * kCh + lane];
        to.weights[to.places * D * N + (2 * share + (threadIdx.x >> 6)) * D + ch] = sum;
    }
}

// db and dc of a row: a wave adds the blocks' shares, lanes four values of a block each, as many blocks at once as it has lanes for.
template <int N, bool kF32>
__device__ __forceinline__ void fold_row(const ScanArgs& a, const ScanGradients& r, int blocks, long long row) {
    constexpr int kAcross = 2 * N / 4, kAtOnce = 64 / kAcross;
    const int lane = threadIdx.x & 63;
    if (row >= a.rows) return;
    const int owner = a.offsets ? r.owners[row] : 0;
    const float* const shares = r.rows;
    const float4v* p = reinterpret_cast<const float4v*>(shares + row * blocks * (2 * N)) + lane;
    float4v sum = {0.f, 0.f, 0.f, 0.f};
    const int mine = lane / kAcross;
#pragma unroll 8
    for (int i = mine; i < blocks; i += kAtOnce, p += 64) sum += __builtin_nontemporal_load(p);
#pragma unroll
    for (int m = kAcross; m < 64; m *= 2)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += __shfl_xor(sum[i], m);
    if (mine != 0 || (a.offsets && !owns(a, owner, row))) return;      // (rows of nobody keep what they hold)
    const int value = 4 * (lane % kAcross);
    const float v[4] = {sum[0], sum[1], sum[2], sum[3]};
    store<kF32>(static_cast<char*>(value < N ? r.db : r.dc) + row * a.bc_row + value % N * (kF32 ? 4 : 2), v);
}

// da, dskip, dbias: 64 values a workgroup, the places in sixteen turns, in their order.
constexpr int kTurns = kScanFoldRows;
__device__ __forceinline__ void fold_weights(const ScanArgs& a, const ScanGradients& r, unsigned group) {
    __shared__ float meet[kTurns][64];
    const int D = a.D, N = a.N, lane = threadIdx.x & 63, turn = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long places = r.places, counted = counts_segments(a) ? *r.used : places, used = counted < places ? counted : places;
    const long long states = static_cast<long long>(D) * N, value = static_cast<long long>(group) * 64 + lane;
    const bool there = value < states + 2 * D;
    const long long stride = value < states ? states : 2 * D;
    const float* from = (value < states ? r.weights + value : r.weights + places * states + (value - states)) + turn * stride;
    float sum = 0.f;
    if (there) {
#pragma unroll 8
        for (long long i = turn; i < used; i += kTurns, from += kTurns * stride) sum += *from;
    }
    meet[turn][lane] = sum;
    __syncthreads();
    if (turn != 0 || !there) return;
#pragma unroll
    for (int i = 1; i < kTurns; ++i) sum += meet[i][lane];
    if (value < states) {
        if (r.da) r.da[value] = sum;
    } else if (value < states + D) {
        if (r.dskip) r.dskip[value - states] = sum;
    } else if (r.dbias) {
        r.dbias[value - states - D] = sum;
    }
}

__global__ __launch_bounds__(64 * kTurns) void scan_weights_kernel(ScanArgs a, ScanGradients r) {
    fold_weights(a, r, blockIdx.x);
}
// Both folds in one launch, as each alone leaves most of the card idle: `rows` workgroups of the one, a row a wave, and the others behind them (in two launches 1 x 512 x 2048
// took 42 us for 39.5, 16 x 64 x 768 33 for 30.8; the others in front 0.8 % more for 2 x 2048 x 4096 with 64 states).
template <int N, bool kF32>
__global__ __launch_bounds__(64 * kTurns) void scan_folds_kernel(ScanArgs a, ScanGradients r, int blocks, unsigned rows) {
    if (blockIdx.x < rows) {
        fold_row<N, kF32>(a, r, blocks, static_cast<long long>(blockIdx.x) * kTurns + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
    } else {
        fold_weights(a, r, blockIdx.x - rows);
    }
}
unsigned weight_groups(const ScanArgs& a, const ScanGradients& g) {
    return g.da || g.dskip || g.dbias ? static_cast<unsigned>((static_cast<long long>(a.D) * (a.N + 2) + 63) / 64) : 0;
}

template <int N, bool kF32>
hipError_t launch(const ScanArgs& a, const ScanGradients& g, hipStream_t stream) {
    const int blocks = static_cast<int>(scan_blocks(a.D));
    const unsigned units = static_cast<unsigned>(blocks) * a.B;
    hipError_t err = hipSuccess;
    if (a.segs > 1) {
        err = launch_scan_pieces(a, g, kF32, stream);
        if (err != hipSuccess) return err;
    }
    const auto kernel = a.z ? &scan_backward_kernel<N, kF32, true> : &scan_backward_kernel<N, kF32, false>;
    hipLaunchKernelGGL(kernel, dim3(units * a.segs), dim3(Shape<N>::kThreads), 0, stream, BackwardArgs{a, g, blocks});
    if ((err = hipGetLastError()) != hipSuccess) return err;
    if (a.rows == 0 || a.T == 0) return launch_scan_weights(a, g, stream);
    const unsigned rows = static_cast<unsigned>((a.rows + kScanFoldRows - 1) / kScanFoldRows);
    const bool together = fits_a_launch(static_cast<long long>(rows) + weight_groups(a, g), 64 * kTurns);
    hipLaunchKernelGGL((scan_folds_kernel<N, kF32>), dim3(rows + (together ? weight_groups(a, g) : 0)), dim3(64 * kTurns), 0, stream, a, g, blocks, rows);
    if ((err = hipGetLastError()) != hipSuccess || together) return err;
    return launch_scan_weights(a, g, stream);
}

}  // namespace

hipError_t launch_scan_weights(const ScanArgs& a, const ScanGradients& g, hipStream_t stream) {
    const unsigned weights = weight_groups(a, g);
    if (weights == 0) return hipSuccess;
    hipLaunchKernelGGL(scan_weights_kernel, dim3(weights), dim3(64 * kTurns), 0, stream, a, g);
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
