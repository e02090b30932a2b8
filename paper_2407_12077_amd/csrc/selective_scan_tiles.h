// What the kernels of the selective scan share: rows as they lie in memory, step sizes, gates, the rows of a workgroup.
#pragma once
#include "selective_scan.h"
#include "wkv6_math.h"

#include <type_traits>
#include <utility>

namespace wkv6 {
namespace scan {

typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef unsigned uint2v __attribute__((ext_vector_type(2)));
typedef unsigned uint4v __attribute__((ext_vector_type(4)));

__device__ __forceinline__ unsigned bf16_of(float v) { return __builtin_bit_cast(unsigned short, static_cast<__bf16>(v)); }
__device__ __forceinline__ unsigned bf16_pair(float a, float b) { return bf16_of(a) | bf16_of(b) << 16; }

// kCount consecutive values of a row, as they lie in memory; none: zeros.
template <bool kF32, int kCount>
struct Raw {
    static constexpr int kWords = kF32 ? kCount : (kCount + 1) / 2;
    unsigned word[kWords];
    __device__ __forceinline__ void none() {
#pragma unroll
        for (int i = 0; i < kWords; ++i) word[i] = 0;
    }
    __device__ __forceinline__ void load(const char* p) {
        if constexpr (!kF32 && kCount == 1) {
            word[0] = *reinterpret_cast<const unsigned short*>(p);
        } else if constexpr (kWords == 1) {
            word[0] = *reinterpret_cast<const unsigned*>(p);
        } else if constexpr (kWords == 2) {
            const uint2v v = *reinterpret_cast<const uint2v*>(p);
            word[0] = v.x;
            word[1] = v.y;
        } else {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                const uint4v v = *reinterpret_cast<const uint4v*>(p + 4 * i);
                word[i] = v.x;
                word[i + 1] = v.y;
                word[i + 2] = v.z;
                word[i + 3] = v.w;
            }
        }
    }
    __device__ __forceinline__ float operator[](int i) const {
        if constexpr (kF32) return __uint_as_float(word[i]);
        else return i & 1 ? bf16_hi(word[i / 2]) : bf16_lo(word[i / 2]);
    }
};
template <bool kF32, int kCount>
__device__ __forceinline__ void store(char* p, const float (&v)[kCount]) {
    if constexpr (kF32) {
        if constexpr (kCount == 1) {
            *reinterpret_cast<float*>(p) = v[0];
        } else if constexpr (kCount == 2) {
            *reinterpret_cast<float2v*>(p) = float2v{v[0], v[1]};
        } else {
#pragma unroll
            for (int i = 0; i < kCount; i += 4) *reinterpret_cast<float4v*>(p + 4 * i) = float4v{v[i], v[i + 1], v[i + 2], v[i + 3]};
        }
    } else {
        if constexpr (kCount == 1) *reinterpret_cast<unsigned short*>(p) = static_cast<unsigned short>(bf16_of(v[0]));
        else if constexpr (kCount == 2) *reinterpret_cast<unsigned*>(p) = bf16_pair(v[0], v[1]);
        else if constexpr (kCount == 4) *reinterpret_cast<uint2v*>(p) = uint2v{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3])};
        else *reinterpret_cast<uint4v*>(p) = uint4v{bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
    }
}

// log(1 + exp(v)) = max(v, 0) + log(1 + e), e = exp(-|v|).  1 + e is rounded, and what it lost is added to its logarithm: (e - ((1 + e) - 1)) is exact,
// and as a share of 1 + e it is below 2^-24, so that leaving out the division by 1 + e costs less than a rounding.  The hardware's logarithm is
// good to two roundings of its own value, near one too.
__device__ __forceinline__ float softplus_of(float v) {
    const float e = __builtin_amdgcn_exp2f(-fabsf(v) * kLog2e), u = 1.f + e;
    return fmaxf(v, 0.f) + __builtin_fmaf(__builtin_amdgcn_logf(u), 0.6931471805599453f, e - (u - 1.f));
}
__device__ __forceinline__ float sigmoid_of(float v) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-v * kLog2e)); }
__device__ __forceinline__ float step_of(float v, bool softplus) { return softplus ? softplus_of(v) : v; }

// A workgroup's rows: tokens of sequence b from the segment's first on; first_row is that token's row.
struct Span {
    long long first_row;
    int tokens;                        // of this segment, 0: none
    bool last;                         // the sequence ends in it (or has no tokens, and this is the first segment)
};
__device__ __forceinline__ Span span_of(const ScanArgs& a, int b, int seg) {
    long long lo = static_cast<long long>(b) * a.T, len = a.T;
    if (a.offsets) {
        long long f = a.offsets[b], e = a.offsets[b + 1];
        f = f < 0 ? 0 : f > a.rows ? a.rows : f;
        e = e < 0 ? 0 : e > a.rows ? a.rows : e;
        len = e - f;
        len = len < 0 ? 0 : len > a.T ? a.T : len;
        lo = f;
    }
    const long long from = static_cast<long long>(seg) * a.seg_len, left = len - from;
    Span s;
    s.first_row = lo + from;
    s.tokens = static_cast<int>(left < 0 ? 0 : left > a.seg_len ? a.seg_len : left);
    s.last = left <= a.seg_len && (left > 0 || seg == 0);
    return s;
}

// f(0), f(1), .. f(kCount - 1), their numbers known to the compiler
template <typename F, int... kI>
__device__ __forceinline__ void each_of(F f, std::integer_sequence<int, kI...>) {
    (f(std::integral_constant<int, kI>()), ...);
}
template <int kCount, typename F>
__device__ __forceinline__ void each(F f) {
    each_of(f, std::make_integer_sequence<int, kCount>());
}

// b or c of a chunk, as operands of outer products (4 x 4 x 1 matrix instructions of sixteen blocks, of whose first operand one block is
// taken for all): a block of four lanes belongs to a token.  plain: its four states.  at_token(n): state n in the lane that has the token's
// number modulo four, nothing in the others, so that the product lands in that row of the result and four tokens share one.
template <bool kF32>
struct StateRow {
    Raw<kF32, 4> raw;
    __device__ __forceinline__ void none() { raw.none(); }
    __device__ __forceinline__ float plain(int lane) const {
        const float low = lane & 1 ? raw[1] : raw[0], high = lane & 1 ? raw[3] : raw[2];
        return lane & 2 ? high : low;
    }
    __device__ __forceinline__ float at_token(int n, int lane) const { return (lane & 3) == (lane >> 2 & 3) ? raw[n] : 0.f; }
};

// c + (rows of one block of a) x b: c[i] += a(lane 4 kBlock + i) b
template <int kBlock>
__device__ __forceinline__ float4v outer(float a, float b, float4v c) {
    return __builtin_amdgcn_mfma_f32_4x4x1f32(a, b, c, 4, kBlock, 0);
}

}  // namespace scan
}  // namespace wkv6
