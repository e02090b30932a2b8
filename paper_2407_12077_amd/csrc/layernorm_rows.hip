// LayerNorm over rows of D values, and its gradients, for gfx950:
//
//     u = (x - mean) rstd        y = u gamma + beta
//     dx = rstd (a - mean(a) - u mean(a u)),  a = gamma dy        dgamma = sum over rows of dy u        dbeta = sum over rows of dy
//
// Both are bound by memory: a row is read once, stays in registers between its sums and its results, and every value leaves once.  A
// row's values lie eight to a lane over one wave (64 lanes, sums without LDS) or over a workgroup of four.
//
// The sums over the rows: a workgroup takes every gridDim.x-th group of rows and a lane always the same columns, so its shares
// of dgamma and dbeta stay in registers to the end; the waves' meet in LDS, the workgroups' in a second kernel that adds them in a
// fixed order.  fp32 throughout; the variance is that of the deviations from the mean.
#include "layernorm_rows.h"

#include "wkv6_launch.h"
#include "wkv6_math.h"

#include <type_traits>

namespace wkv6 {
namespace {

typedef float float4v __attribute__((ext_vector_type(4)));
typedef unsigned uint4v __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float float8v __attribute__((ext_vector_type(8)));

// eight values of a row
template <bool kF32>
__device__ __forceinline__ float8v load8(const void* p, long long item) {
    if constexpr (kF32) {
        const float4v* f = static_cast<const float4v*>(p) + 2 * item;
        const float4v a = __builtin_nontemporal_load(f), b = __builtin_nontemporal_load(f + 1);
        return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
    } else {
        const uint4v u = __builtin_nontemporal_load(static_cast<const uint4v*>(p) + item);
        return float8v{bf16_lo(u.x), bf16_hi(u.x), bf16_lo(u.y), bf16_hi(u.y), bf16_lo(u.z), bf16_hi(u.z), bf16_lo(u.w), bf16_hi(u.w)};
    }
}
template <bool kF32>
__device__ __forceinline__ void store8(void* p, long long item, float8v v) {
    if constexpr (kF32) {
        float4v* f = static_cast<float4v*>(p) + 2 * item;
        __builtin_nontemporal_store(__builtin_shufflevector(v, v, 0, 1, 2, 3), f);
        __builtin_nontemporal_store(__builtin_shufflevector(v, v, 4, 5, 6, 7), f + 1);
    } else {
        __builtin_nontemporal_store(__builtin_bit_cast(uint4v, __builtin_convertvector(v, bf16x8)), static_cast<uint4v*>(p) + item);
    }
}
__device__ __forceinline__ float8v param8(const float* p, int item) {
    const float4v* f = reinterpret_cast<const float4v*>(p) + 2 * item;
    return __builtin_shufflevector(f[0], f[1], 0, 1, 2, 3, 4, 5, 6, 7);
}
__device__ __forceinline__ float sum8(float8v v) { return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7])); }

template <int kBy>
__device__ __forceinline__ float rotated(float v) {        // within a row of sixteen lanes
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x120 + kBy, 0xf, 0xf, false));
}
// sum over a wave, in every lane
__device__ __forceinline__ float wave_sum(float v) {
    v += rotated<8>(v);
    v += rotated<4>(v);
    v += rotated<2>(v);
    v += rotated<1>(v);
    auto q = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(q[0]) + __uint_as_float(q[1]);
    q = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(q[0]) + __uint_as_float(q[1]);
}
// sums over a row's lanes; `place` is used by no other sum until the workgroup has met again
template <int kLanes, int kCount>
__device__ __forceinline__ void row_sums(float (&v)[kCount], float (*place)[kCount]) {
#pragma unroll
    for (int i = 0; i < kCount; ++i) v[i] = wave_sum(v[i]);
    if constexpr (kLanes == 256) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < kCount; ++i) place[threadIdx.x >> 6][i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kCount; ++i) v[i] = (place[0][i] + place[1][i]) + (place[2][i] + place[3][i]);
    }
}

template <bool kXF32, bool kYF32, int kLanes, int kItems>
__global__ __launch_bounds__(256) void norm_kernel(long long M, int items, const void* x, const float* gamma, const float* beta, float eps,
                                                   void* y, float2* stats) {
    __shared__ float place[2][4][1];
    const int at = threadIdx.x % kLanes;
    const long long row = static_cast<long long>(blockIdx.x) * (256 / kLanes) + threadIdx.x / kLanes;
    if (row >= M) return;                                      // whole waves, and with 256 lanes no workgroup
    const long long first = row * items;
    float8v v[kItems];
    float sum[1] = {0.f};
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int item = at + i * kLanes;
        v[i] = item < items ? load8<kXF32>(x, first + item) : float8v{};
        sum[0] += sum8(v[i]);
    }
    row_sums<kLanes>(sum, place[0]);
    const float width = 1.f / static_cast<float>(8 * items);
    const float mean = sum[0] * width;
    float dev[1] = {0.f};
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        v[i] -= mean;
        if (at + i * kLanes < items) dev[0] += sum8(v[i] * v[i]);
    }
    row_sums<kLanes>(dev, place[1]);
    const float rstd = 1.f / sqrtf(dev[0] * width + eps);
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int item = at + i * kLanes;
        if (item < items) store8<kYF32>(y, first + item, v[i] * rstd * param8(gamma, item) + param8(beta, item));
    }
    if (stats && at == 0) stats[row] = make_float2(mean, rstd);
}

template <bool kXF32, bool kYF32, int kLanes, int kItems>
__global__ __launch_bounds__(256) void norm_backward_kernel(long long M, int items, const void* x, const float2* stats, const float* gamma,
                                                            const void* dy, void* dx, float* partials) {
    constexpr int kRows = 256 / kLanes;                        // of a workgroup at a time
    __shared__ float place[2][4][2];
    __shared__ float8v meet[kRows > 1 ? 2 * 64 : 1];
    const int at = threadIdx.x % kLanes;
    float8v gm[kItems], dg[kItems], db[kItems];
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        const int item = at + i * kLanes;
        gm[i] = item < items ? param8(gamma, item) : float8v{};
        dg[i] = db[i] = float8v{};
    }
    const float width = 1.f / static_cast<float>(8 * items);
    int turn = 0;
    for (long long row = static_cast<long long>(blockIdx.x) * kRows + threadIdx.x / kLanes; row < M;
         row += static_cast<long long>(gridDim.x) * kRows, turn ^= 1) {
        const long long first = row * items;
        const float2 ms = stats[row];
        float8v u[kItems], a[kItems];
        float sums[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int item = at + i * kLanes;
            const bool there = item < items;
            u[i] = there ? (load8<kXF32>(x, first + item) - ms.x) * ms.y : float8v{};
            a[i] = there ? load8<kYF32>(dy, first + item) : float8v{};
            db[i] += a[i];
            dg[i] += a[i] * u[i];
            a[i] *= gm[i];
            sums[0] += sum8(a[i]);
            sums[1] += sum8(a[i] * u[i]);
        }
        row_sums<kLanes>(sums, place[turn]);
        const float m0 = sums[0] * width, m1 = sums[1] * width;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const int item = at + i * kLanes;
            if (item < items) store8<kXF32>(dx, first + item, (a[i] - m0 - u[i] * m1) * ms.y);
        }
    }
    if (!partials) return;
    float* mine = partials + static_cast<long long>(blockIdx.x) * 16 * items;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
        if constexpr (kRows > 1) {                             // the other waves' shares of these columns, in their order
            for (int wave = 1; wave < kRows; ++wave) {
                __syncthreads();
                if (static_cast<int>(threadIdx.x >> 6) == wave) {
                    meet[at] = dg[i];
                    meet[64 + at] = db[i];
                }
                __syncthreads();
                if (threadIdx.x < 64) {
                    dg[i] += meet[at];
                    db[i] += meet[64 + at];
                }
            }
        }
        const int item = at + i * kLanes;
        if (threadIdx.x < kLanes && item < items) {
            store8<true>(mine, item, dg[i]);
            store8<true>(mine, items + item, db[i]);
        }
    }
}

// 64 columns a workgroup; a thread adds every sixteenth row of four of them
__global__ __launch_bounds__(256) void norm_fold_kernel(int rows, int D, const float4v* partials, float4v* dgamma, float4v* dbeta) {
    __shared__ float4v part[16][16];
    const int lane = threadIdx.x & 15, group = threadIdx.x >> 4;
    const int column = blockIdx.x * 16 + lane, columns = D / 2;          // fours of dgamma, then of dbeta
    float4v sum = {0.f, 0.f, 0.f, 0.f};
    if (column < columns)
        for (int r = group; r < rows; r += 16) sum += partials[static_cast<long long>(r) * columns + column];
    part[group][lane] = sum;
    __syncthreads();
    if (group > 0 || column >= columns) return;
#pragma unroll
    for (int i = 1; i < 16; ++i) sum += part[i][lane];
    if (column < D / 4) dgamma[column] = sum;
    else dbeta[column - D / 4] = sum;
}

// Lanes of a row: one wave, or four where a wave would hold too much or would leave most of the card idle.
bool wide_rows(long long M, int D, int most) { return D > most || (D >= 1024 && M <= 1024); }
constexpr int kNormWave = 4096, kBackwardWave = 2048;          // widest rows of one wave

// f(lanes, items of a lane) with the least that hold a row of up to kMost items a wave, or any in a workgroup
template <int kMost, typename F>
hipError_t with_width(bool wide, int items, F f) {
    const int n = (items + (wide ? 255 : 63)) / (wide ? 256 : 64);
    auto pick = [&](auto lanes) {
        constexpr int kLanes = decltype(lanes)::value;
        if (n <= 1) return f(lanes, std::integral_constant<int, 1>{});
        if (n <= 2) return f(lanes, std::integral_constant<int, 2>{});
        if constexpr (kLanes == 256 || kMost > 4)
            if (n > 4) return f(lanes, std::integral_constant<int, 8>{});
        return f(lanes, std::integral_constant<int, 4>{});
    };
    return wide ? pick(std::integral_constant<int, 256>{}) : pick(std::integral_constant<int, 64>{});
}
// f(type of x, type of y)
template <typename F>
hipError_t with_types(bool x_f32, bool y_f32, F f) {
    if (x_f32) return y_f32 ? f(std::true_type{}, std::true_type{}) : f(std::true_type{}, std::false_type{});
    return y_f32 ? f(std::false_type{}, std::true_type{}) : f(std::false_type{}, std::false_type{});
}

}  // namespace

hipError_t launch_norm(long long M, int D, const void* x, const float* gamma, const float* beta, float eps, void* y, float* stats, bool x_f32,
                       bool y_f32, hipStream_t stream) {
    const bool wide = wide_rows(M, D, kNormWave);
    const unsigned grid = static_cast<unsigned>(wide ? M : (M + 3) / 4);
    return with_types(x_f32, y_f32, [&](auto xf, auto yf) {
        return with_width<kNormWave / 512>(wide, D / 8, [&](auto lanes, auto count) {
            hipLaunchKernelGGL(HIP_KERNEL_NAME(norm_kernel<decltype(xf)::value, decltype(yf)::value, decltype(lanes)::value, decltype(count)::value>),
                               dim3(grid), dim3(256), 0, stream, M, D / 8, x, gamma, beta, eps, y, reinterpret_cast<float2*>(stats));
            return hipGetLastError();
        });
    });
}

int norm_partials(long long M, int D) {
    const int rows = wide_rows(M, D, kBackwardWave) ? 1 : 4;
    const long long most = (M + rows - 1) / rows;
    return static_cast<int>(most < 512 ? most : 512);
}

hipError_t launch_norm_backward(long long M, int D, const void* x, const float* stats, const float* gamma, const void* dy, void* dx,
                                float* dgamma, float* dbeta, float* partials, bool x_f32, bool y_f32, hipStream_t stream) {
    const bool wide = wide_rows(M, D, kBackwardWave);
    const int grid = norm_partials(M, D);
    if (grid > 0) {
        const hipError_t err = with_types(x_f32, y_f32, [&](auto xf, auto yf) {
            return with_width<kBackwardWave / 512>(wide, D / 8, [&](auto lanes, auto count) {
                hipLaunchKernelGGL(HIP_KERNEL_NAME(norm_backward_kernel<decltype(xf)::value, decltype(yf)::value, decltype(lanes)::value, decltype(count)::value>),
                                   dim3(grid), dim3(256), 0, stream, M, D / 8, x, reinterpret_cast<const float2*>(stats), gamma, dy, dx,
                                   dgamma ? partials : nullptr);
                return hipGetLastError();
            });
        });
        if (err != hipSuccess) return err;
    }
    if (dgamma)
        hipLaunchKernelGGL(norm_fold_kernel, dim3(static_cast<unsigned>((D / 2 + 15) / 16)), dim3(256), 0, stream, grid, D,
                           reinterpret_cast<const float4v*>(partials), reinterpret_cast<float4v*>(dgamma), reinterpret_cast<float4v*>(dbeta));
    return hipGetLastError();
}

}  // namespace wkv6
