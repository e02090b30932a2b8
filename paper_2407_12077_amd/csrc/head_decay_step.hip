// The head-decay time mix for one token of every sequence: S = exp(g) S_in + k^T v, o = r S.
//
// Bound by the states, which are read and written once: 1024 x 32 heads 168.7 us, 6.4 TB/s.  A workgroup of four waves a unit; a lane holds four
// columns of four key rows, so that a load takes whole lines, r and k of a lane's rows are consecutive, and all of its state is on its way at
// once.  (A wave a unit, sixteen rows a lane: 187 us, and from 512 units on slower at every number: 16 x 32 5.5 against 4.7.)  The states go past
// the caches: with stores that stay in them 183 us.
#include "head_decay.h"
#include "wkv6_math.h"

namespace wkv6 {
namespace {

typedef float float4v __attribute__((ext_vector_type(4)));
typedef unsigned uint2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

template <bool kF32>
__device__ __forceinline__ float4v four(const char* p) {
    if constexpr (kF32) {
        return *reinterpret_cast<const float4v*>(p);
    } else {
        const uint2v u = *reinterpret_cast<const uint2v*>(p);
        return float4v{bf16_lo(u.x), bf16_hi(u.x), bf16_lo(u.y), bf16_hi(u.y)};
    }
}

template <bool kF32, bool kOutF32>
__global__ __launch_bounds__(256) void mix_step_kernel(int H, const char* r, const char* k, const char* v, long long row_bytes,
                                                       const float* g, long long g_row, const float* state_in, void* out, float* state_out) {
    constexpr int kSize = kF32 ? 4 : 2, kRows = 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), unit = blockIdx.x;
    const int b = unit / H, h = unit - b * H;
    const int j = 4 * (lane & 15), c0 = 16 * (lane >> 4) + 4 * wave;
    const long long state = static_cast<long long>(unit) * (kHeadSize * kHeadSize) + c0 * kHeadSize + j;
    float4v s[kRows];
    if (state_in) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) s[i] = __builtin_nontemporal_load(reinterpret_cast<const float4v*>(state_in + state + i * kHeadSize));
    } else {
#pragma unroll
        for (int i = 0; i < kRows; ++i) s[i] = float4v{0.f, 0.f, 0.f, 0.f};
    }
    const long long row = b * row_bytes + h * (kHeadSize * kSize);
    const float4v vj = four<kF32>(v + row + j * kSize);
    const float4v rc = four<kF32>(r + row + c0 * kSize), kc = four<kF32>(k + row + c0 * kSize);
    const float decay = expf(g[b * g_row + h]);
    float4v o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        s[i] = s[i] * decay + vj * kc[i];
        o += s[i] * rc[i];
        if (state_out) __builtin_nontemporal_store(s[i], reinterpret_cast<float4v*>(state_out + state + i * kHeadSize));
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        o[e] += __shfl_xor(o[e], 16);
        o[e] += __shfl_xor(o[e], 32);
    }
    __shared__ float4v part[4][16];
    if (lane < 16) part[wave][lane] = o;
    __syncthreads();
    if (wave > 0) return;
    o = (part[0][lane & 15] + part[1][lane & 15]) + (part[2][lane & 15] + part[3][lane & 15]);
    if (lane < 16) {
        const long long to = static_cast<long long>(unit) * kHeadSize + j;
        if constexpr (kOutF32) *reinterpret_cast<float4v*>(static_cast<float*>(out) + to) = o;
        else *reinterpret_cast<uint2v*>(static_cast<char*>(out) + 2 * to) = __builtin_bit_cast(uint2v, __builtin_convertvector(o, bf16x4));
    }
}

}  // namespace

hipError_t launch_mix_step(int B, int H, const void* r, const void* k, const void* v, long long row_stride, const float* g,
                           long long g_row, const float* state_in, void* out, float* state_out, bool f32_rows, bool f32_out,
                           hipStream_t stream) {
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(B * H)), dim3(256), 0, stream, H, static_cast<const char*>(r),
                           static_cast<const char*>(k), static_cast<const char*>(v), row_stride * (f32_rows ? 4 : 2), g, g_row, state_in, out,
                           state_out);
        return hipGetLastError();
    };
    if (f32_rows) return go(&mix_step_kernel<true, true>);
    return f32_out ? go(&mix_step_kernel<false, true>) : go(&mix_step_kernel<false, false>);
}

}  // namespace wkv6
