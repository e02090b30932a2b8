// C ABI of the selective scan and of the short convolution in front of it: argument validation and dispatch only.
#include "../../include/wkv6_selective_scan.h"
#include "../../include/wkv6_short_conv.h"
#include "selective_scan.h"
#include "short_conv.h"

#include <cstdint>

namespace {

bool misaligned(const void* p) { return (reinterpret_cast<std::uintptr_t>(p) & 15u) != 0; }
bool misaligned4(const void* p) { return (reinterpret_cast<std::uintptr_t>(p) & 3u) != 0; }
template <typename... P>
bool any_null(const P*... p) { return ((p == nullptr) || ...); }
template <typename... P>
bool any_misaligned(const P*... p) { return (misaligned(p) || ...); }

bool known(int dtype) { return dtype == WKV6_DTYPE_BF16 || dtype == WKV6_DTYPE_F32; }
int status_of(hipError_t err) { return err == hipSuccess ? WKV6_OK : WKV6_ERR_LAUNCH; }
int item_of(int dtype) { return dtype == WKV6_DTYPE_F32 ? 4 : 2; }

constexpr long long kMaxStride = 1ll << 22;
constexpr int kMaxChannels = 65536, kMaxTokens = 1 << 30;
constexpr long long kMaxRows = 0x7fffffffLL;

bool channels_fit(int D) { return D % 8 == 0; }
bool states_fit(int N) { return N == 8 || N == 16 || N == 32 || N == 64; }
bool sizes_fit(int B, int T, int D, long long rows) {
    return B >= 0 && T >= 0 && T <= kMaxTokens && D >= 8 && D <= kMaxChannels && rows >= 0 && rows <= kMaxRows;
}
bool rows_fit(int B, int T, long long rows, bool packed) { return packed || rows == static_cast<long long>(B) * T; }
// rows of `width` values that lie `stride` apart
int check_stride(long long stride, int width, int dtype) {
    if (stride < width || stride > kMaxStride) return WKV6_ERR_SHAPE;
    return stride * item_of(dtype) % 16 != 0 ? WKV6_ERR_ALIGN : WKV6_OK;
}
int check_workspace(const void* workspace, long long bytes, long long needed) {
    if (needed == 0) return WKV6_OK;
    if (!workspace) return WKV6_ERR_NULL;
    if (misaligned(workspace)) return WKV6_ERR_ALIGN;
    return bytes < needed ? WKV6_ERR_WORKSPACE : WKV6_OK;
}

// ---------------------------------------------------------------------------------------------- scan
// What every call of the scan has; strides and row pointers are looked at where there are rows.
struct ScanCall {
    int B, T, D, N;
    long long rows;
    const void* x;
    long long x_stride;
    const void* delta;
    long long delta_stride;
    const float* bias;
    int softplus;
    const float* a;
    const void *b, *c;
    long long bc_stride;
    const float* skip;
    const void* z;
    long long z_stride;
    const int* offsets;
    const float* state_in;
    int dtype, out_dtype;

    int check_sizes() const {
        if (!states_fit(N) || !known(dtype) || !known(out_dtype) || !channels_fit(D)) return WKV6_ERR_UNSUPPORTED;
        if (dtype == WKV6_DTYPE_F32 && out_dtype != WKV6_DTYPE_F32) return WKV6_ERR_UNSUPPORTED;
        return sizes_fit(B, T, D, rows) && rows_fit(B, T, rows, offsets != nullptr) ? WKV6_OK : WKV6_ERR_SHAPE;
    }
    bool any_rows() const { return rows > 0 && T > 0; }
    int check_inputs() const {
        if (!a) return WKV6_ERR_NULL;
        if (any_rows()) {
            if (any_null(x, delta, b, c)) return WKV6_ERR_NULL;
            for (const int status : {check_stride(x_stride, D, dtype), check_stride(delta_stride, D, dtype), check_stride(bc_stride, N, dtype),
                                     z ? check_stride(z_stride, D, dtype) : static_cast<int>(WKV6_OK)})
                if (status != WKV6_OK) return status;
        }
        return any_misaligned(x, delta, b, c, z) || any_misaligned(bias, a, skip, state_in) || misaligned4(offsets) ? WKV6_ERR_ALIGN : WKV6_OK;
    }
    wkv6::ScanArgs args(const wkv6::ScanPlan& p) const {
        wkv6::ScanArgs s;
        const int item = item_of(dtype);
        s.B = B; s.T = T; s.D = D; s.N = N; s.rows = rows;
        s.x = x; s.delta = delta; s.z = z; s.b = b; s.c = c;
        s.x_row = x_stride * item; s.delta_row = delta_stride * item; s.z_row = z_stride * item; s.bc_row = bc_stride * item;
        s.a = a; s.bias = bias; s.skip = skip; s.softplus = softplus != 0;
        s.offsets = offsets; s.state_in = state_in;
        s.segs = p.segs; s.seg_len = p.seg_len;
        s.locals = nullptr;
        return s;
    }
};

bool step_fits(int B, int D, int N) {
    return wkv6::fits_a_launch(static_cast<long long>(B) * ((static_cast<long long>(D) * (N / 4) + 255) / 256), 256);
}

long long four(long long n) { return (n + 3) / 4 * 4; }

// Workspaces in floats, every part a multiple of four; false where a launch would not fit.
struct ScanSpace {
    wkv6::ScanPlan plan;
    long long locals = 0, states = 0, rows = 0, owners = 0, places = 0, weights = 0, used = 0, floats = 0;
};
bool space_of(const wkv6::ScanPlan& plan, int B, int D, int N, long long rows, bool packed, bool backward, ScanSpace* s) {
    s->plan = plan;
    const long long blocks = wkv6::scan_blocks(D);
    if (!wkv6::fits_a_launch((backward && plan.segs > 1 ? 2 : 1) * B * blocks * plan.segs, wkv6::scan_threads(N))) return false;
    s->locals = four(wkv6::scan_local_floats(plan, B, D, N));
    s->floats = s->locals;
    if (backward) {
        if (!wkv6::fits_a_launch((rows + wkv6::kScanFoldRows - 1) / wkv6::kScanFoldRows, 64 * wkv6::kScanFoldRows)) return false;
        s->states = wkv6::chunk_places(rows, wkv6::scan_back_chunk(N)) * D * N;
        s->rows = rows * blocks * 2 * N;
        s->owners = packed ? four(rows) : 0;
        s->places = wkv6::share_places(B, rows, plan.segs, plan.seg_len, packed);
        s->weights = s->places * D * (N + 2);
        s->used = packed && plan.segs > 1 ? 4 : 0;
        s->floats = 2 * s->locals + s->states + s->rows + s->owners + s->weights + s->used;
    }
    return true;
}
bool scan_space(int B, int T, int D, int N, long long rows, bool packed, bool backward, ScanSpace* s) {
    return space_of(wkv6::plan_scan(B, T, D, N, packed ? rows : -1, backward), B, D, N, rows, packed, backward, s);
}
constexpr int kAnyLength = 1;
// For calls with offsets or, if there are B T rows, without.  A prefill's rows are not known: for any that fit.
long long scan_bytes(int B, int T, int D, int N, long long rows, bool backward) {
    ScanSpace s;
    long long most = 0;
    if (!backward || rows == static_cast<long long>(B) * T) {
        if (!scan_space(B, T, D, N, rows, false, backward, &s)) return -1;
        most = s.floats;
    }
    if (backward) {
        if (!scan_space(B, T, D, N, rows, true, true, &s)) return -1;
    } else {
        const int segs = wkv6::scan_most_segments(B, T, D, true);
        if (!space_of({segs, kAnyLength}, B, D, N, 0, true, false, &s)) return -1;
    }
    return 4 * (s.floats > most ? s.floats : most);
}

// ---------------------------------------------------------------------------------------------- convolution
struct ConvCall {
    int B, T, D, W;
    long long rows;
    const void* x;
    long long x_stride;
    const float *w, *bias;
    int silu;
    const int* offsets;
    const void* state_in;
    int dtype;

    int check_sizes() const {
        if (W < 2 || W > 4 || !known(dtype) || !channels_fit(D)) return WKV6_ERR_UNSUPPORTED;
        return sizes_fit(B, T, D, rows) && rows_fit(B, T, rows, offsets != nullptr) ? WKV6_OK : WKV6_ERR_SHAPE;
    }
    bool any_rows() const { return rows > 0 && T > 0; }
    int check_inputs() const {
        if (!w) return WKV6_ERR_NULL;
        if (any_rows()) {
            if (!x) return WKV6_ERR_NULL;
            const int status = check_stride(x_stride, D, dtype);
            if (status != WKV6_OK) return status;
        }
        return any_misaligned(x, state_in) || any_misaligned(w, bias) || misaligned4(offsets) ? WKV6_ERR_ALIGN : WKV6_OK;
    }
    wkv6::ConvArgs args(const wkv6::ConvPlan& p) const {
        wkv6::ConvArgs s;
        s.B = B; s.T = T; s.D = D; s.W = W; s.rows = rows;
        s.x = x; s.x_row = x_stride * item_of(dtype);
        s.w = w; s.bias = bias; s.silu = silu != 0;
        s.offsets = offsets; s.state_in = state_in;
        s.segs = p.segs; s.seg_len = p.seg_len; s.lanes = p.lanes;
        return s;
    }
};

}  // namespace

extern "C" {

long long wkv6_selective_scan_workspace_bytes(int B, int T, int D, int N) {
    if (!states_fit(N) || !channels_fit(D) || !sizes_fit(B, T, D, 0)) return -1;
    return B == 0 ? 0 : scan_bytes(B, T, D, N, 0, false);
}

long long wkv6_selective_scan_backward_workspace_bytes(int B, int T, int D, int N, long long rows) {
    if (!states_fit(N) || !channels_fit(D) || !sizes_fit(B, T, D, rows)) return -1;
    return B == 0 ? 0 : scan_bytes(B, T, D, N, rows, true);
}

int wkv6_selective_scan_prefill(int B, int T, int D, int N, long long rows, const void* x, long long x_stride, const void* delta,
                                long long delta_stride, const float* delta_bias, int softplus, const float* a, const void* b, const void* c,
                                long long bc_stride, const float* skip, const void* z, long long z_stride, const int* offsets,
                                const float* state_in, void* out, float* state_out, int dtype, int out_dtype, void* workspace,
                                long long workspace_bytes, void* stream) {
    const ScanCall call{B, T, D, N, rows, x, x_stride, delta, delta_stride, delta_bias, softplus, a, b, c, bc_stride, skip, z, z_stride, offsets,
                        state_in, dtype, out_dtype};
    int status = call.check_sizes();
    if (status != WKV6_OK || B == 0) return status;
    if ((status = call.check_inputs()) != WKV6_OK) return status;
    if (call.any_rows() && !out) return WKV6_ERR_NULL;
    if (any_misaligned(out) || any_misaligned(state_out)) return WKV6_ERR_ALIGN;
    ScanSpace s;
    if (!scan_space(B, T, D, N, rows, offsets != nullptr, false, &s)) return WKV6_ERR_SHAPE;
    if ((status = check_workspace(workspace, workspace_bytes, 4 * s.floats)) != WKV6_OK) return status;
    wkv6::ScanArgs args = call.args(s.plan);
    args.locals = static_cast<float*>(workspace);
    if (T > 0 && T <= wkv6::kScanFewTokens && step_fits(B, D, N))
        return status_of(wkv6::launch_scan_step(args, out, state_out, dtype == WKV6_DTYPE_F32, out_dtype == WKV6_DTYPE_F32, static_cast<hipStream_t>(stream)));
    return status_of(wkv6::launch_scan(args, out, state_out, dtype == WKV6_DTYPE_F32, out_dtype == WKV6_DTYPE_F32, static_cast<hipStream_t>(stream)));
}

int wkv6_selective_scan_decode(int B, int D, int N, const void* x, long long x_stride, const void* delta, long long delta_stride,
                               const float* delta_bias, int softplus, const float* a, const void* b, const void* c, long long bc_stride,
                               const float* skip, const void* z, long long z_stride, const float* state_in, void* out, float* state_out, int dtype,
                               int out_dtype, void* stream) {
    const ScanCall call{B, 1, D, N, B, x, x_stride, delta, delta_stride, delta_bias, softplus, a, b, c, bc_stride, skip, z, z_stride, nullptr,
                        state_in, dtype, out_dtype};
    int status = call.check_sizes();
    if (status != WKV6_OK || B == 0) return status;
    if ((status = call.check_inputs()) != WKV6_OK) return status;
    if (!out) return WKV6_ERR_NULL;
    if (any_misaligned(out) || any_misaligned(state_out)) return WKV6_ERR_ALIGN;
    if (!step_fits(B, D, N)) return WKV6_ERR_SHAPE;
    return status_of(wkv6::launch_scan_step(call.args({1, 1}), out, state_out, dtype == WKV6_DTYPE_F32, out_dtype == WKV6_DTYPE_F32,
                                            static_cast<hipStream_t>(stream)));
}

int wkv6_selective_scan_backward(int B, int T, int D, int N, long long rows, const void* x, long long x_stride, const void* delta,
                                 long long delta_stride, const float* delta_bias, int softplus, const float* a, const void* b, const void* c,
                                 long long bc_stride, const float* skip, const void* z, long long z_stride, const int* offsets,
                                 const float* state_in, const void* dout, const float* dstate_out, void* dx, void* ddelta, void* db, void* dc,
                                 void* dz, float* da, float* dskip, float* ddelta_bias, float* dstate_in, int dtype, void* workspace,
                                 long long workspace_bytes, void* stream) {
    const ScanCall call{B, T, D, N, rows, x, x_stride, delta, delta_stride, delta_bias, softplus, a, b, c, bc_stride, skip, z, z_stride, offsets,
                        state_in, dtype, dtype};
    int status = call.check_sizes();
    if (status != WKV6_OK) return status;
    if (any_misaligned(da, dskip, ddelta_bias)) return WKV6_ERR_ALIGN;
    hipStream_t st = static_cast<hipStream_t>(stream);
    wkv6::ScanGradients g = {};
    g.da = da; g.dskip = dskip; g.dbias = ddelta_bias;
    if (B == 0) return status_of(wkv6::launch_scan_weights(call.args({1, 1}), g, st));      // no sequence: but sums over no tokens are nought
    if ((status = call.check_inputs()) != WKV6_OK) return status;
    if (call.any_rows() && any_null(dout, static_cast<const void*>(dx), static_cast<const void*>(ddelta), static_cast<const void*>(db), static_cast<const void*>(dc)))
        return WKV6_ERR_NULL;
    if (any_misaligned(dout, static_cast<const void*>(dx), static_cast<const void*>(ddelta), static_cast<const void*>(db), static_cast<const void*>(dc),
                       static_cast<const void*>(dz)) || any_misaligned(dstate_out, static_cast<const float*>(dstate_in)))
        return WKV6_ERR_ALIGN;
    ScanSpace s;
    if (!scan_space(B, T, D, N, rows, offsets != nullptr, true, &s)) return WKV6_ERR_SHAPE;
    if ((status = check_workspace(workspace, workspace_bytes, 4 * s.floats)) != WKV6_OK) return status;
    wkv6::ScanArgs args = call.args(s.plan);
    float* at = static_cast<float*>(workspace);
    auto take = [&](long long floats) {
        float* p = at;
        at += floats;
        return p;
    };
    args.locals = take(s.locals);
    g.behind = take(s.locals);
    g.states = take(s.states);
    g.rows = take(s.rows);
    g.owners = reinterpret_cast<int*>(take(s.owners));
    g.weights = take(s.weights);
    g.places = s.places;
    g.used = reinterpret_cast<long long*>(take(s.used));
    g.dout = dout; g.dstate_out = dstate_out;
    g.dx = dx; g.ddelta = ddelta; g.db = db; g.dc = dc; g.dz = dz; g.dstate_in = dstate_in;
    return status_of(wkv6::launch_scan_backward(args, g, dtype == WKV6_DTYPE_F32, st));
}

long long wkv6_short_conv_backward_workspace_bytes(int B, int T, int D, int W, long long rows) {
    if (W < 2 || W > 4 || !channels_fit(D) || !sizes_fit(B, T, D, rows)) return -1;
    const wkv6::ConvPlan p = wkv6::plan_conv(B, T, D, rows, true);
    return wkv6::fits_a_launch(p.workgroups, wkv6::kConvThreads) ? 4 * wkv6::conv_partial_floats(B, D, W, rows, p, true) : -1;     // (without offsets fewer)
}

int wkv6_short_conv_prefill(int B, int T, int D, int W, long long rows, const void* x, long long x_stride, const float* w, const float* bias,
                            int silu, const int* offsets, const void* state_in, void* out, void* state_out, int dtype, void* stream) {
    const ConvCall call{B, T, D, W, rows, x, x_stride, w, bias, silu, offsets, state_in, dtype};
    int status = call.check_sizes();
    if (status != WKV6_OK || B == 0) return status;
    if ((status = call.check_inputs()) != WKV6_OK) return status;
    if (call.any_rows() && !out) return WKV6_ERR_NULL;
    if (any_misaligned(out, state_out)) return WKV6_ERR_ALIGN;
    const wkv6::ConvPlan p = wkv6::plan_conv(B, T, D, rows, false);
    if (!wkv6::fits_a_launch(p.workgroups, wkv6::kConvThreads)) return WKV6_ERR_SHAPE;
    return status_of(wkv6::launch_conv(call.args(p), out, state_out, dtype == WKV6_DTYPE_F32, static_cast<hipStream_t>(stream)));
}

int wkv6_short_conv_decode(int B, int D, int W, const void* x, long long x_stride, const float* w, const float* bias, int silu,
                           const void* state_in, void* out, void* state_out, int dtype, void* stream) {
    const ConvCall call{B, 1, D, W, B, x, x_stride, w, bias, silu, nullptr, state_in, dtype};
    int status = call.check_sizes();
    if (status != WKV6_OK || B == 0) return status;
    if ((status = call.check_inputs()) != WKV6_OK) return status;
    if (!out) return WKV6_ERR_NULL;
    if (any_misaligned(out, state_out)) return WKV6_ERR_ALIGN;
    if (!wkv6::fits_a_launch(static_cast<long long>(B) * (D / wkv6::kConvStepGroup) + wkv6::kConvThreads, 1)) return WKV6_ERR_SHAPE;
    return status_of(wkv6::launch_conv_step(call.args({1, 1, 1, 1}), out, state_out, dtype == WKV6_DTYPE_F32, static_cast<hipStream_t>(stream)));
}

int wkv6_short_conv_backward(int B, int T, int D, int W, long long rows, const void* x, long long x_stride, const float* w, const float* bias,
                             int silu, const int* offsets, const void* state_in, const void* dout, const void* dstate_out, void* dx, float* dw,
                             float* dbias, void* dstate_in, int dtype, void* workspace, long long workspace_bytes, void* stream) {
    const ConvCall call{B, T, D, W, rows, x, x_stride, w, bias, silu, offsets, state_in, dtype};
    int status = call.check_sizes();
    if (status != WKV6_OK) return status;
    if ((dw == nullptr) != (dbias == nullptr)) return WKV6_ERR_NULL;
    if (any_misaligned(dw, dbias)) return WKV6_ERR_ALIGN;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const wkv6::ConvPlan p = wkv6::plan_conv(B, T, D, rows, true);
    if (B == 0) return dw ? status_of(wkv6::launch_conv_fold(call.args(p), dw, dbias, nullptr, st)) : WKV6_OK;   // sums over no tokens are nought
    if ((status = call.check_inputs()) != WKV6_OK) return status;
    if (call.any_rows() && any_null(dout, dx)) return WKV6_ERR_NULL;
    if (any_misaligned(dout, dstate_out) || any_misaligned(dx, dstate_in)) return WKV6_ERR_ALIGN;
    if (!wkv6::fits_a_launch(p.workgroups, wkv6::kConvThreads)) return WKV6_ERR_SHAPE;
    if (dw && (status = check_workspace(workspace, workspace_bytes, 4 * wkv6::conv_partial_floats(B, D, W, rows, p, offsets != nullptr))) != WKV6_OK)
        return status;
    return status_of(wkv6::launch_conv_backward(call.args(p), dout, dstate_out, dx, dw, dbias, dstate_in, static_cast<float*>(workspace),
                                                dtype == WKV6_DTYPE_F32, st));
}

}  // extern "C"
