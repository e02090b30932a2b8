// C ABI of the head-decay time mix and of the LayerNorm with its gradients: argument validation and dispatch only.
#include "../../include/wkv6_head_decay.h"
#include "../../include/wkv6_layernorm.h"
#include "head_decay.h"
#include "layernorm_rows.h"

#include <cstdint>

namespace {

using wkv6::kHeadSize;

bool misaligned(const void* p) { return (reinterpret_cast<std::uintptr_t>(p) & 15u) != 0; }
bool misaligned4(const void* p) { return (reinterpret_cast<std::uintptr_t>(p) & 3u) != 0; }
template <typename... P>
bool any_null(const P*... p) { return ((p == nullptr) || ...); }
template <typename... P>
bool any_misaligned(const P*... p) { return (misaligned(p) || ...); }

bool known(int dtype) { return dtype == WKV6_DTYPE_BF16 || dtype == WKV6_DTYPE_F32; }
int status_of(hipError_t err) { return err == hipSuccess ? WKV6_OK : WKV6_ERR_LAUNCH; }

// 32-bit offsets inside a chunk of 64 tokens
constexpr long long kMaxStride = 1ll << 22;
constexpr int kMaxHeads = 65536;
constexpr int kMaxTokens = 1 << 30;
constexpr long long kStateFloats = kHeadSize * kHeadSize;

// Sizes and types that every call of the mix has; the strides are looked at where there are rows.
int check_mix(int B, int T, int H, int N, long long rows, bool packed, int dtype, int out_dtype) {
    if (N != kHeadSize || !known(dtype) || !known(out_dtype)) return WKV6_ERR_UNSUPPORTED;
    if (dtype == WKV6_DTYPE_F32 && out_dtype != WKV6_DTYPE_F32) return WKV6_ERR_UNSUPPORTED;
    if (B < 0 || T < 0 || T > kMaxTokens || H < 1 || H > kMaxHeads || rows < 0 || rows > 0x7fffffffLL) return WKV6_ERR_SHAPE;
    if (!packed && rows != static_cast<long long>(B) * T) return WKV6_ERR_SHAPE;
    return WKV6_OK;
}
int check_strides(int H, long long token_stride, long long g_stride, int dtype) {
    if (token_stride < static_cast<long long>(H) * kHeadSize || token_stride > kMaxStride) return WKV6_ERR_SHAPE;
    if (g_stride != 0 && (g_stride < H || g_stride > kMaxStride)) return WKV6_ERR_SHAPE;
    return token_stride % (dtype == WKV6_DTYPE_F32 ? 4 : 8) != 0 ? WKV6_ERR_ALIGN : WKV6_OK;
}

// Workspace in floats, every part a multiple of four; false where the launches would not fit.
struct Space {
    wkv6::MixPlan plan;
    long long locals = 0, sums = 0, anchors = 0, head_sums = 0, floats = 0;
};
long long four(long long n) { return (n + 3) / 4 * 4; }
bool space_of(int B, int T, int H, long long rows, bool packed, bool backward, bool f32_rows, Space* s) {
    s->plan = wkv6::plan_mix(B, T, H, packed ? rows : -1, backward, f32_rows);
    const long long units = static_cast<long long>(B) * H;
    if (!wkv6::fits_a_launch(units, wkv6::kMixThreads) || !wkv6::fits_a_launch(units * s->plan.segs * (backward ? 3 : 1), wkv6::kMixThreads) ||
        (backward && !wkv6::fits_a_launch(units * s->plan.blocks, wkv6::kDecayGradientThreads)))
        return false;
    if (s->plan.segs > 1) s->locals = s->plan.segs * units * (kStateFloats + 4);
    s->floats = s->locals;
    if (backward) {
        s->sums = four(H * rows);
        s->anchors = s->plan.places * H * kStateFloats;
        s->head_sums = four(units * s->plan.blocks);
        s->floats = 2 * s->locals + 2 * s->sums + 2 * s->anchors + s->head_sums;
    }
    return true;
}
// for rows of either type, packed or, if there are B T, not.  rows < 0: not known, for packed sequences of as many as may be
long long workspace_bytes_of(int B, int T, int H, long long rows, bool backward) {
    long long most = 0;
    for (int i = 0; i < 4; ++i) {
        const bool packed = i & 1 && rows >= 0;
        if (!packed && rows >= 0 && rows != static_cast<long long>(B) * T) continue;
        Space s;
        if (!space_of(B, T, H, rows < 0 ? 0 : rows, packed, backward, i & 2, &s)) return -1;
        if (s.floats > most) most = s.floats;
    }
    const long long units = static_cast<long long>(B) * H, pieces = T > 0 ? (T - 1) / wkv6::kMixBlock + 1 : 1;
    if (rows < 0 && units < wkv6::kMixFewUnits && pieces > 1) {
        const long long cut = (pieces < wkv6::kMixPackedSegments ? pieces : wkv6::kMixPackedSegments) * units * (kStateFloats + 4);
        if (cut > most) most = cut;
    }
    return 4 * most;
}

wkv6::MixArgs mix_args(int B, int T, int H, long long rows, const float* g, long long g_stride, const int* offsets, const wkv6::MixPlan& p) {
    wkv6::MixArgs a;
    a.B = B; a.T = T; a.H = H; a.rows = rows;
    a.g = g; a.g_row = g_stride; a.offsets = offsets;
    a.segs = p.segs; a.seg_len = p.seg_len; a.anchor_len = p.anchor_len; a.blocks = p.blocks; a.whole_places = p.whole_places;
    a.sweeps = 1;
    return a;
}

}  // namespace

extern "C" {

long long wkv6_head_decay_workspace_bytes(int B, int T, int H, int N) {
    if (N != kHeadSize || B < 0 || T < 0 || T > kMaxTokens || H < 1 || H > kMaxHeads) return -1;
    return B == 0 ? 0 : workspace_bytes_of(B, T, H, -1, false);
}

long long wkv6_head_decay_backward_workspace_bytes(int B, int T, int H, int N, long long rows) {
    if (N != kHeadSize || B < 0 || T < 0 || T > kMaxTokens || H < 1 || H > kMaxHeads || rows < 0 || rows > 0x7fffffffLL) return -1;
    return B == 0 ? 0 : workspace_bytes_of(B, T, H, rows, true);
}

int wkv6_head_decay_prefill(int B, int T, int H, int N, long long rows, const void* r, const void* k, const void* v,
                            long long token_stride, const float* g, long long g_stride, const int* offsets, const float* state_in,
                            void* out, float* state_out, int dtype, int out_dtype, void* workspace, long long workspace_bytes,
                            void* stream) {
    int status = check_mix(B, T, H, N, rows, offsets != nullptr, dtype, out_dtype);
    if (status != WKV6_OK) return status;
    if (B == 0) return WKV6_OK;
    if (rows > 0 && T > 0) {
        if (any_null(r, k, v, g, out)) return WKV6_ERR_NULL;
        status = check_strides(H, token_stride, g_stride, dtype);
        if (status != WKV6_OK) return status;
    }
    if (any_misaligned(r, k, v, out, state_in, state_out) || misaligned4(g) || misaligned4(offsets)) return WKV6_ERR_ALIGN;
    Space s;
    if (!space_of(B, T, H, rows, offsets != nullptr, false, dtype == WKV6_DTYPE_F32, &s)) return WKV6_ERR_SHAPE;
    if (s.floats > 0) {
        if (!workspace) return WKV6_ERR_NULL;
        if (misaligned(workspace)) return WKV6_ERR_ALIGN;
        if (workspace_bytes < 4 * s.floats) return WKV6_ERR_WORKSPACE;
    }
    const bool f32 = dtype == WKV6_DTYPE_F32, f32_out = out_dtype == WKV6_DTYPE_F32;
    const int item = f32 ? 4 : 2;
    wkv6::MixArgs a = mix_args(B, T, H, rows, g, g_stride, offsets, s.plan);
    wkv6::Sweep& w = a.sweep[0];
    w.q = static_cast<const char*>(r);
    w.k = static_cast<const char*>(k);
    w.v = static_cast<const char*>(v);
    w.q_row = w.k_row = w.v_row = token_stride * item;
    w.out = static_cast<char*>(out);
    w.out_row = static_cast<long long>(H) * kHeadSize * (f32_out ? 4 : 2);
    w.state_in = state_in;
    w.state_out = state_out;
    w.locals = static_cast<float*>(workspace);
    hipStream_t st = static_cast<hipStream_t>(stream);
    hipError_t err = wkv6::raise_mix_limits();
    if (err == hipSuccess && a.segs > 1) err = wkv6::launch_mix_locals(a, 1, f32, st);
    if (err == hipSuccess) err = wkv6::launch_mix(a, f32, f32_out, st);
    return status_of(err);
}

int wkv6_head_decay_decode(int B, int H, int N, const void* r, const void* k, const void* v, long long token_stride, const float* g,
                           long long g_stride, const float* state_in, void* out, float* state_out, int dtype, int out_dtype,
                           void* stream) {
    int status = check_mix(B, 1, H, N, B, false, dtype, out_dtype);
    if (status != WKV6_OK) return status;
    if (B == 0) return WKV6_OK;
    if (any_null(r, k, v, g, out)) return WKV6_ERR_NULL;
    status = check_strides(H, token_stride, g_stride, dtype);
    if (status != WKV6_OK) return status;
    if (any_misaligned(r, k, v, out, state_in, state_out) || misaligned4(g)) return WKV6_ERR_ALIGN;
    if (static_cast<long long>(B) * H >= 1ll << 24) return WKV6_ERR_SHAPE;
    return status_of(wkv6::launch_mix_step(B, H, r, k, v, token_stride, g, g_stride, state_in, out, state_out, dtype == WKV6_DTYPE_F32,
                                           out_dtype == WKV6_DTYPE_F32, static_cast<hipStream_t>(stream)));
}

int wkv6_head_decay_backward(int B, int T, int H, int N, long long rows, const void* r, const void* k, const void* v,
                             long long token_stride, const float* g, long long g_stride, const int* offsets, const float* state_in,
                             const void* dout, const float* dstate_out, void* dr, void* dk, void* dv, float* dg, float* dstate_in,
                             int dtype, void* workspace, long long workspace_bytes, void* stream) {
    int status = check_mix(B, T, H, N, rows, offsets != nullptr, dtype, dtype);
    if (status != WKV6_OK) return status;
    if (B == 0) {                                              // no sequence: but the sum over no tokens is nought
        if (!dg || g_stride != 0) return WKV6_OK;
        return misaligned4(dg) ? WKV6_ERR_ALIGN : status_of(wkv6::launch_head_sums(0, H, nullptr, dg, static_cast<hipStream_t>(stream)));
    }
    if (rows > 0 && T > 0) {
        if (any_null(r, k, v, g, dout, dr, dk, dv, dg)) return WKV6_ERR_NULL;
        status = check_strides(H, token_stride, g_stride, dtype);
        if (status != WKV6_OK) return status;
    }
    if (any_misaligned(r, k, v, dout, dr, dk, dv) || any_misaligned(state_in, dstate_out, dstate_in) || misaligned4(g) ||
        misaligned4(dg) || misaligned4(offsets))
        return WKV6_ERR_ALIGN;
    Space s;
    if (!space_of(B, T, H, rows, offsets != nullptr, true, dtype == WKV6_DTYPE_F32, &s)) return WKV6_ERR_SHAPE;
    if (s.floats > 0) {
        if (!workspace) return WKV6_ERR_NULL;
        if (misaligned(workspace)) return WKV6_ERR_ALIGN;
        if (workspace_bytes < 4 * s.floats) return WKV6_ERR_WORKSPACE;
    }
    const bool f32 = dtype == WKV6_DTYPE_F32;
    const int item = f32 ? 4 : 2;
    const long long row = token_stride * item, dense = static_cast<long long>(H) * kHeadSize * item;
    float* at = static_cast<float*>(workspace);
    auto take = [&](long long floats) {
        float* p = at;
        at += floats;
        return p;
    };
    float *states = take(s.locals), *gradients = take(s.locals), *r_sums = take(s.sums), *k_sums = take(s.sums), *behind = take(s.anchors),
          *front = take(s.anchors), *head_sums = take(s.head_sums);
    const char *rp = static_cast<const char*>(r), *kp = static_cast<const char*>(k), *vp = static_cast<const char*>(v),
               *op = static_cast<const char*>(dout);
    wkv6::MixArgs a = mix_args(B, T, H, rows, g, g_stride, offsets, s.plan);
    a.sweeps = 3;
    wkv6::Sweep &wr = a.sweep[0], &wv = a.sweep[1], &wk = a.sweep[2];
    // dr: the transposed states from the first token on
    wr.q = op; wr.q_row = dense;
    wr.k = vp; wr.k_row = row;
    wr.v = kp; wr.v_row = row;
    wr.out = static_cast<char*>(dr); wr.out_row = row;
    wr.with = rp; wr.with_row = row; wr.sums = r_sums;
    wr.state_in = state_in; wr.turned = true;
    wr.locals = states; wr.anchors = behind;
    // dv: the states' gradients from the last token on
    wv.q = kp; wv.q_row = row;
    wv.k = rp; wv.k_row = row;
    wv.v = op; wv.v_row = dense;
    wv.out = static_cast<char*>(dv); wv.out_row = row;
    wv.state_in = dstate_out; wv.state_out = dstate_in;
    wv.locals = gradients; wv.reverse = true;
    // dk: the same, transposed
    wk.q = vp; wk.q_row = row;
    wk.k = op; wk.k_row = dense;
    wk.v = rp; wk.v_row = row;
    wk.out = static_cast<char*>(dk); wk.out_row = row;
    wk.with = kp; wk.with_row = row; wk.sums = k_sums;
    wk.state_in = dstate_out; wk.turned = true;
    wk.locals = gradients; wk.locals_turned = true; wk.reverse = true;
    wk.anchors = front;
    hipStream_t st = static_cast<hipStream_t>(stream);
    hipError_t err = wkv6::raise_mix_limits();
    if (err == hipSuccess && a.segs > 1) err = wkv6::launch_mix_locals(a, 2, f32, st);
    if (err == hipSuccess) err = wkv6::launch_mix(a, f32, f32, st);
    if (err == hipSuccess && dg) err = wkv6::launch_decay_gradient(a, r_sums, k_sums, behind, front, head_sums, dg, st);
    return status_of(err);
}

int wkv6_layernorm_forward(long long M, int D, const void* x, const float* gamma, const float* beta, float eps, void* y, float* mean_rstd,
                           int dtype, int out_dtype, void* stream) {
    if (!known(dtype) || !known(out_dtype) || D < 8 || D % 8 != 0 || D > wkv6::kNormMaxWidth) return WKV6_ERR_UNSUPPORTED;
    if (M < 0 || M >= 1ll << 24 || !(eps >= 0.f)) return WKV6_ERR_SHAPE;
    if (M == 0) return WKV6_OK;
    if (any_null(x, y) || any_null(gamma, beta)) return WKV6_ERR_NULL;
    if (any_misaligned(x, y) || any_misaligned(gamma, beta, mean_rstd)) return WKV6_ERR_ALIGN;
    return status_of(wkv6::launch_norm(M, D, x, gamma, beta, eps, y, mean_rstd, dtype == WKV6_DTYPE_F32, out_dtype == WKV6_DTYPE_F32,
                                       static_cast<hipStream_t>(stream)));
}

long long wkv6_layernorm_backward_workspace_bytes(long long M, int D) {
    if (D < 8 || D % 8 != 0 || D > wkv6::kNormMaxWidth || M < 0 || M >= 1ll << 24) return -1;
    const int bf16 = wkv6::norm_partials(M, D, true), other = wkv6::norm_partials(M, D, false);
    return 8ll * D * (bf16 > other ? bf16 : other);
}

int wkv6_layernorm_backward(long long M, int D, const void* x, const float* mean_rstd, const float* gamma, const void* dy, void* dx,
                            float* dgamma, float* dbeta, int dtype, int out_dtype, void* workspace, long long workspace_bytes, void* stream) {
    if (!known(dtype) || !known(out_dtype) || D < 8 || D % 8 != 0 || D > wkv6::kNormMaxWidth) return WKV6_ERR_UNSUPPORTED;
    if (M < 0 || M >= 1ll << 24) return WKV6_ERR_SHAPE;
    if ((dgamma == nullptr) != (dbeta == nullptr)) return WKV6_ERR_NULL;
    if (M > 0 && (any_null(x, dy, dx) || any_null(mean_rstd, gamma))) return WKV6_ERR_NULL;
    if (any_misaligned(x, dy, dx, workspace) || any_misaligned(mean_rstd, gamma, dgamma, dbeta)) return WKV6_ERR_ALIGN;
    if (M == 0 && !dgamma) return WKV6_OK;
    if (dgamma && M > 0) {
        if (!workspace) return WKV6_ERR_NULL;
        if (workspace_bytes < wkv6_layernorm_backward_workspace_bytes(M, D)) return WKV6_ERR_WORKSPACE;
    }
    return status_of(wkv6::launch_norm_backward(M, D, x, mean_rstd, gamma, dy, dx, dgamma, dbeta, static_cast<float*>(workspace),
                                                dtype == WKV6_DTYPE_F32, out_dtype == WKV6_DTYPE_F32, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
