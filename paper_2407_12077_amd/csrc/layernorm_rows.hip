// LayerNorm over rows of D values, and its gradients, for gfx950:
//
//     u = (x - mean) rstd        y = u gamma + beta
//     dx = rstd (a - mean(a) - u mean(a u)),  a = gamma dy        dgamma = sum over rows of dy u        dbeta = sum over rows of dy
//
// Both are bound by memory: a row is read once, stays in registers between its sums and its results, and every value leaves once, past
// the caches.  32768 x 2048 bf16 rows: forward 53 us, 5.1 TB/s, a large copy's rate; gradients 74.5 us, 5.4 TB/s, of which the fold is 4.5.
// Few rows wait on their latency: 24 x 4096 4.0 us, gradients of 1531 x 768 10.3 (6 and 4 in two launches).
// A row's values lie eight to a lane over one wave (64 lanes, sums without LDS) or over a workgroup of four, or of eight.
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

// eight values of a row, as they lie in memory
template <bool kF32>
struct Raw8 {
    std::conditional_t<kF32, float8v, uint4v> bits;
    __device__ __forceinline__ void load(const void* p, long long item) {
        if constexpr (kF32) {
            const float4v* f = static_cast<const float4v*>(p) + 2 * item;
            const float4v a = __builtin_nontemporal_load(f), b = __builtin_nontemporal_load(f + 1);
            bits = __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        } else {
            bits = __builtin_nontemporal_load(static_cast<const uint4v*>(p) + item);
        }
    }
    __device__ __forceinline__ float8v values() const {
        if constexpr (kF32) return bits;
        else return float8v{bf16_lo(bits.x), bf16_hi(bits.x), bf16_lo(bits.y), bf16_hi(bits.y), bf16_lo(bits.z), bf16_hi(bits.z), bf16_lo(bits.w), bf16_hi(bits.w)};
    }
};
template <bool kF32>
__device__ __forceinline__ float8v load8(const void* p, long long item) {
    Raw8<kF32> r;
    r.load(p, item);
    return r.values();
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
    if constexpr (kLanes > 64) {
        if ((threadIdx.x & 63) == 0)
#pragma unroll
            for (int i = 0; i < kCount; ++i) place[threadIdx.x >> 6][i] = v[i];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kCount; ++i) {
            v[i] = 0.f;
#pragma unroll
            for (int w = 0; w < kLanes / 64; w += 4) v[i] += (place[w][i] + place[w + 1][i]) + (place[w + 2][i] + place[w + 3][i]);
        }
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
__global__ __launch_bounds__(kLanes < 256 ? 256 : kLanes) void norm_backward_kernel(long long M, int items, const void* x, const float2* stats, const float* gamma,
                                                            const void* dy, void* dx, float* partials) {
    constexpr int kRows = kLanes < 256 ? 256 / kLanes : 1;     // of a workgroup at a time
    __shared__ float place[2][kLanes < 256 ? 4 : kLanes / 64][2];
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
    // the next row of this lane's is on its way while one is worked on
    Raw8<kXF32> x_raw[kItems] = {};
    Raw8<kYF32> y_raw[kItems] = {};
    float2 ms_next = make_float2(0.f, 0.f);
    auto ask = [&](long long row) {
        ms_next = stats[row];
#pragma unroll
        for (int i = 0; i < kItems; ++i)
            if (at + i * kLanes < items) {
                x_raw[i].load(x, row * items + at + i * kLanes);
                y_raw[i].load(dy, row * items + at + i * kLanes);
            }
    };
    const long long step = static_cast<long long>(gridDim.x) * kRows;
    long long row = static_cast<long long>(blockIdx.x) * kRows + threadIdx.x / kLanes;
    // (the widest fp32 rows leave no registers for it: 4096 x 16384 262 us with, 212 without; bf16 109 and 117)
    constexpr bool kNext = kLanes < 512 || !kXF32 || !kYF32;
    if (kNext && row < M) ask(row);
    for (int turn = 0; row < M; row += step, turn ^= 1) {
        if (!kNext) ask(row);
        const long long first = row * items;
        const float2 ms = ms_next;
        float8v u[kItems], a[kItems];
        float sums[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            u[i] = (x_raw[i].values() - ms.x) * ms.y;
            a[i] = y_raw[i].values();                          // (nought where there is nothing)
        }
        if (kNext && row + step < M) ask(row + step);
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
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

// Sixteen columns a workgroup: a thread adds every 64th row of four of them, eight asked for at a time.  (64 columns a workgroup and one row
// at a time: 13 to 15 us, most of it waiting, where this takes 4.)
__global__ __launch_bounds__(256) void norm_fold_kernel(int rows, int D, const float4v* partials, float4v* dgamma, float4v* dbeta) {
    __shared__ float4v part[64][4];
    const int lane = threadIdx.x & 3, group = threadIdx.x >> 2;
    const int column = blockIdx.x * 4 + lane, columns = D / 2;           // fours of dgamma, then of dbeta (D / 2 is a multiple of four)
    float4v sum = {0.f, 0.f, 0.f, 0.f};
    for (int r0 = group; r0 < rows; r0 += 512) {
        float4v v[8];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = r0 + 64 * i < rows ? partials[static_cast<long long>(r0 + 64 * i) * columns + column] : float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += v[i];
    }
    part[group][lane] = sum;
    __syncthreads();
    for (int half = 32; half > 0; half /= 2) {
        if (group < half) part[group][lane] += part[group + half][lane];
        __syncthreads();
    }
    if (group > 0) return;
    if (column < D / 4) dgamma[column] = part[0][lane];
    else dbeta[column - D / 4] = part[0][lane];
}

// Lanes of a row: a wave, which needs no LDS and no barrier, up to 1024 columns; four waves where one would hold too much, or would be too few to
// keep memory busy.  Measured, a wave against four, us:
//                      bf16 x 1024   x 2048       fp32 x 1024    x 2048       gradients, bf16 x 1024   x 2048      fp32 x 1024   x 2048
//     1500 rows         4.4   4.6     5.8  4.5     4.5   4.5      7.7   6.0    9.7  10.4                12.9  12.2   11.8  11.8    20.3  15.7
//     4096 rows         4.8   6.3     7.9  9.1     8.1   9.1     16.3  16.0   12.8  14.6                18.0  18.3   17.9  18.7    33.0  27.6
//     32768 rows       25.6  35.4    53.0 55.2    58.4  58.3    122.8 109.5   40.6  60.2                74.5  78.6   84.2  95.5   161.1 161.2
// (one type of either: as fp32.)  4096 columns, 32768 rows: bf16 119.5 against 110.6.
int norm_lanes(long long M, int D, bool bf16) { return D > 2048 || (D > 1024 && (!bf16 || M < 4096)) ? 256 : 64; }
// The gradients keep a row, the next one, gamma and two sums for every column, which four waves with eight items a lane barely hold: eight waves beyond
// 8192 columns.  Eight against four at 4096 x 10240: bf16 71 and 89 us, fp32 134 and 164 (fp32 rows with bf16 dy 136 and 127); at 4096 x 8192
// 60 and 54, 107 and 96.
int norm_backward_lanes(long long M, int D, bool bf16) { return D > 8192 ? 512 : norm_lanes(M, D, bf16); }

// f(lanes, items of a lane), items of eight columns: the least of 1, 2, 4 and, in the forward pass, 8 that hold a row
template <bool kForward, typename F>
hipError_t with_items(int lanes, int items, F f) {
    constexpr std::integral_constant<int, 64> wave;
    constexpr std::integral_constant<int, 256> four;
    constexpr std::integral_constant<int, 1> one;
    constexpr std::integral_constant<int, 2> two;
    constexpr std::integral_constant<int, 4> most;
    const int n = (items + lanes - 1) / lanes;
    if (lanes == 64) return n <= 1 ? f(wave, one) : n <= 2 ? f(wave, two) : f(wave, most);
    if constexpr (!kForward)
        if (lanes == 512) return f(std::integral_constant<int, 512>{}, most);
    if constexpr (kForward)
        if (n > 4) return f(four, std::integral_constant<int, 8>{});
    return n <= 1 ? f(four, one) : n <= 2 ? f(four, two) : f(four, most);
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
    const int row_lanes = norm_lanes(M, D, !x_f32 && !y_f32);
    const unsigned grid = static_cast<unsigned>(row_lanes == 256 ? M : (M + 3) / 4);
    return with_types(x_f32, y_f32, [&](auto xf, auto yf) {
        return with_items<true>(row_lanes, D / 8, [&](auto lanes, auto count) {
            hipLaunchKernelGGL(HIP_KERNEL_NAME(norm_kernel<decltype(xf)::value, decltype(yf)::value, decltype(lanes)::value, decltype(count)::value>),
                               dim3(grid), dim3(256), 0, stream, M, D / 8, x, gamma, beta, eps, y, reinterpret_cast<float2*>(stats));
            return hipGetLastError();
        });
    });
}

int norm_partials(long long M, int D, bool bf16) {
    const int rows = norm_backward_lanes(M, D, bf16) == 64 ? 4 : 1;
    const long long most = (M + rows - 1) / rows;
    return static_cast<int>(most < 512 ? most : 512);
}

hipError_t launch_norm_backward(long long M, int D, const void* x, const float* stats, const float* gamma, const void* dy, void* dx,
                                float* dgamma, float* dbeta, float* partials, bool x_f32, bool y_f32, hipStream_t stream) {
    const bool bf16 = !x_f32 && !y_f32;
    const int row_lanes = norm_backward_lanes(M, D, bf16);
    const int grid = norm_partials(M, D, bf16);
    if (grid > 0) {
        const hipError_t err = with_types(x_f32, y_f32, [&](auto xf, auto yf) {
            return with_items<false>(row_lanes, D / 8, [&](auto lanes, auto count) {
                hipLaunchKernelGGL(HIP_KERNEL_NAME(norm_backward_kernel<decltype(xf)::value, decltype(yf)::value, decltype(lanes)::value, decltype(count)::value>),
                                   dim3(grid), dim3(row_lanes < 256 ? 256 : row_lanes), 0, stream, M, D / 8, x, reinterpret_cast<const float2*>(stats), gamma, dy, dx,
                                   dgamma ? partials : nullptr);
                return hipGetLastError();
            });
        });
        if (err != hipSuccess) return err;
    }
    if (dgamma)
        hipLaunchKernelGGL(norm_fold_kernel, dim3(static_cast<unsigned>(D / 8)), dim3(256), 0, stream, grid, D,
                           reinterpret_cast<const float4v*>(partials), reinterpret_cast<float4v*>(dgamma), reinterpret_cast<float4v*>(dbeta));
    return hipGetLastError();
}

}  // namespace wkv6
