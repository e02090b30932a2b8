// What the kernels of the selective scan and of the short convolution share: rows as they lie in memory, step sizes, gates, the rows of a workgroup,
// and the matrix cores' outer products with read-outs beside them.
#pragma once
#include "selective_scan.h"
#include "wkv6_math.h"

#include <type_traits>
#include <utility>

namespace wkv6 {
namespace scan {

typedef float float4v __attribute__((ext_vector_type(4)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef unsigned uint2v __attribute__((ext_vector_type(2)));
typedef unsigned uint4v __attribute__((ext_vector_type(4)));

__device__ __forceinline__ unsigned bf16_of(float v) { return __builtin_bit_cast(unsigned short, static_cast<__bf16>(v)); }
__device__ __forceinline__ unsigned bf16_pair(float a, float b) {
    return __builtin_bit_cast(unsigned, __builtin_convertvector((float2v{a, b}), bf16x2));     // (one instruction)
}

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
    // back, as it is
    __device__ __forceinline__ void put(char* p) const {
        static_assert(kWords == 2 || kWords % 4 == 0);
        if constexpr (kWords == 2) *reinterpret_cast<uint2v*>(p) = uint2v{word[0], word[1]};
#pragma unroll
        for (int i = 0; i + 4 <= kWords; i += 4) *reinterpret_cast<uint4v*>(p + 4 * i) = uint4v{word[i], word[i + 1], word[i + 2], word[i + 3]};
    }
    // from a buffer; what lies behind its end is zeros
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t from, int at) {
        if constexpr (!kF32 && kCount == 1) {
            word[0] = __builtin_amdgcn_raw_buffer_load_b16(from, at, 0, 0);
        } else if constexpr (kWords == 1) {
            word[0] = __builtin_amdgcn_raw_buffer_load_b32(from, at, 0, 0);
        } else if constexpr (kWords == 2) {
            const auto v = __builtin_bit_cast(uint2v, __builtin_amdgcn_raw_buffer_load_b64(from, at, 0, 0));
            word[0] = v.x;
            word[1] = v.y;
        } else {
#pragma unroll
            for (int i = 0; i < kWords; i += 4) {
                const auto v = __builtin_bit_cast(uint4v, __builtin_amdgcn_raw_buffer_load_b128(from, at + 4 * i, 0, 0));
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
// the words of kCount values of either type
template <bool kF32, int kCount>
__device__ __forceinline__ void words_of(const float (&v)[kCount], unsigned (&word)[Raw<kF32, kCount>::kWords]) {
#pragma unroll
    for (int i = 0; i < Raw<kF32, kCount>::kWords; ++i) {
        if constexpr (kF32) word[i] = __float_as_uint(v[i]);
        else if constexpr (kCount == 1) word[i] = bf16_of(v[i]);
        else word[i] = bf16_pair(v[2 * i], v[2 * i + 1]);
    }
}
// into a buffer; nothing behind its end
template <bool kF32, int kCount>
__device__ __forceinline__ void store(__amdgpu_buffer_rsrc_t to, int at, const float (&v)[kCount]) {
    constexpr int kWords = Raw<kF32, kCount>::kWords;
    unsigned word[kWords];
    words_of<kF32>(v, word);
    if constexpr (!kF32 && kCount == 1) {
        __builtin_amdgcn_raw_buffer_store_b16(static_cast<unsigned short>(word[0]), to, at, 0, 0);
    } else if constexpr (kWords == 1) {
        __builtin_amdgcn_raw_buffer_store_b32(word[0], to, at, 0, 0);
    } else if constexpr (kWords == 2) {
        __builtin_amdgcn_raw_buffer_store_b64(uint2v{word[0], word[1]}, to, at, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < kWords; i += 4) __builtin_amdgcn_raw_buffer_store_b128(uint4v{word[i], word[i + 1], word[i + 2], word[i + 3]}, to, at + 4 * i, 0, 0);
    }
}
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
// (1 / (1 + inf) is nought, so that values far below nought need no care)
__device__ __forceinline__ float sigmoid_of(float v) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-v * kLog2e)); }
// a log2(e) of four states, no infinity: a step size of nought (behind a sequence's end too) leaves a state as it is, however large a.  By comparisons, as
// minima, maxima and medians take the other operand for a NaN, and a weight that is none has to show.
__device__ __forceinline__ float4v rate_of(const float* a) {
    float4v rate = *reinterpret_cast<const float4v*>(a) * kLog2e;
#pragma unroll
    for (int i = 0; i < 4; ++i) rate[i] = rate[i] < -__FLT_MAX__ ? -__FLT_MAX__ : rate[i] > __FLT_MAX__ ? __FLT_MAX__ : rate[i];
    return rate;
}
// Over a piece: state <- exp2(sum rate) state + local, with what the piece leaves of nothing.  Where states grow the factor may pass what fp32 holds though the product does not
// (nought stays nought), so it comes in three equal parts, none above 2^127: 2^-149, the smallest state, times 2^381 is none any more.  `third`: of the rates.
// (Two ways, and the question which, cost the gradients of 1 x 512 x 2048 1 us of 39.)
__device__ __forceinline__ void pass_on(float4v& state, float sum, float4v third, float4v local) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float part = __builtin_amdgcn_exp2f(fminf(sum * third[i], 127.f));       // (of a NaN local is one too)
        state[i] = __builtin_fmaf(part, part * (part * state[i]), local[i]);
    }
}
__device__ __forceinline__ float step_of(float v, bool softplus) { return softplus ? softplus_of(v) : v; }

// All bits for softplus, none without; the compiler is not to know which, or it makes a branch of it and two blocks of what surrounds that.
__device__ __forceinline__ unsigned softplus_bits(bool softplus) {
    unsigned bits = softplus ? ~0u : 0u;
    asm("" : "+s"(bits));
    return bits;
}
__device__ __forceinline__ float chosen(unsigned bits, float yes, float no) {
    const unsigned y = __float_as_uint(yes), n = __float_as_uint(no);
    return __uint_as_float(((y ^ n) & bits) ^ n);              // (one instruction)
}
template <bool kF32, int kCount>
__device__ __forceinline__ void steps_of(const Raw<kF32, kCount>& delta, const float (&bias)[kCount], unsigned softplus, float (&dt)[kCount]) {
#pragma unroll
    for (int i = 0; i < kCount; ++i) {
        const float v = delta[i] + bias[i];
        dt[i] = chosen(softplus, softplus_of(v), v);
    }
}

// Segments of the sequences in front of b (share_places), counted by a workgroup's threads: what this wave has counted, in all its lanes.
template <int kThreads, typename Args>
__device__ __forceinline__ int segments_in_front(const Args& a, int b) {
    int n = 0;
    for (int i = threadIdx.x; i < b; i += kThreads) n += segments_of(tokens_of(a, i), a.seg_len);
#pragma unroll
    for (int m = 1; m < 64; m *= 2) n += __shfl_xor(n, m);
    return n;
}
template <typename Args>
__device__ __forceinline__ bool counts_segments(const Args& a) { return a.offsets && a.segs > 1; }

// A workgroup's rows: those of a segment of sequence b.
struct Span {
    long long first_row;
    int tokens;                        // of this segment, 0: none
    bool last;                         // the sequence ends in it (or has no tokens, and this is the first segment)
};
__device__ __forceinline__ Span span_of(const ScanArgs& a, int b, int seg) {
    const long long from = static_cast<long long>(seg) * a.seg_len, left = tokens_of(a, b) - from;
    Span s;
    s.first_row = first_row_of(a, b) + from;
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

// Rows of a tensor, a chunk at a time: what lies behind `count` rows is not read, and stores there are dropped.  All of it is the same in a wave, so
// addresses cost no vector instruction, and few scalar ones.
struct Rows {
    char* at;                          // the chunk's first row
    int row;                           // bytes
    __device__ __forceinline__ Rows(const void* base, long long first, long long row_bytes)
        : at(static_cast<char*>(const_cast<void*>(base)) + first * row_bytes), row(static_cast<int>(row_bytes)) {}
    __device__ __forceinline__ void move(int rows) { at += static_cast<long long>(rows) * row; }
    __device__ __forceinline__ __amdgpu_buffer_rsrc_t first(int count) const { return __builtin_amdgcn_make_buffer_rsrc(at, 0, count * row, 0x00020000); }
};
// how many of a chunk's rows there are if `left` are left
template <int kC>
__device__ __forceinline__ int rows_of(int left) {
    return left < 0 ? 0 : left > kC ? kC : left;
}
constexpr int kNowhere = 0x7fffff00;   // an offset behind the end of any such rows

// c[0] h[0] + c[1] h[1] + c[2] h[2] + c[3] h[3] where c's values lie in lanes 4 kFirst .. 4 kFirst + 3 of every row of sixteen lanes: operands that
// come from another lane cost nothing, but the compiler makes moves of them in front of a multiply-add.  It does not know what is in here, so it
// keeps no distance to it: a register that a vector instruction has written may be read from other lanes two states later (the s_nop, here and
// not where the compiler could move it), and one that a matrix instruction has written only after more.  h has to come from vector
// instructions, or `after` from one that has read it, for which the compiler has waited.
template <int kFirst>
__device__ __forceinline__ float read_out(float c, float4v h, float after) {
    float y;
    asm("s_nop 1\n\t"
        "v_mul_f32_dpp %0, %1, %2 row_newbcast:%c7 row_mask:0xf bank_mask:0xf\n\t"
        "v_fmac_f32_dpp %0, %1, %3 row_newbcast:%c8 row_mask:0xf bank_mask:0xf\n\t"
        "v_fmac_f32_dpp %0, %1, %4 row_newbcast:%c9 row_mask:0xf bank_mask:0xf\n\t"
        "v_fmac_f32_dpp %0, %1, %5 row_newbcast:%c10 row_mask:0xf bank_mask:0xf"
        : "=&v"(y)
        : "v"(c), "v"(h[0]), "v"(h[1]), "v"(h[2]), "v"(h[3]), "v"(after), "n"(4 * kFirst), "n"(4 * kFirst + 1), "n"(4 * kFirst + 2), "n"(4 * kFirst + 3));
    return y;
}

// c[i] + a(lane 4 kBlock + i) b for i < 4, of every lane's b and c: a 4 x 4 x 1 matrix instruction of sixteen blocks of four lanes, of whose first
// operand one block is taken for all.
template <int kBlock>
__device__ __forceinline__ float4v outer(float a, float b, float4v c = float4v{0.f, 0.f, 0.f, 0.f}) {
    return __builtin_amdgcn_mfma_f32_4x4x1f32(a, b, c, 4, kBlock, 0);
}

// A chunk's b or c for one wave's four states: in the order of outer(), and of read_out() by groups of four tokens.  Tokens behind `left`: zeros.
template <bool kF32>
struct Plain {
    Raw<kF32, 1> raw;                  // state lane % 4 of token lane / 4
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rows, int lane, int row_bytes, int n0) {
        raw.load(rows, lane / 4 * row_bytes + (n0 + lane % 4) * (kF32 ? 4 : 2));
    }
    __device__ __forceinline__ float value() const { return raw[0]; }
};
template <bool kF32, int kGroups>
struct ByRow {
    Raw<kF32, 1> raw[kGroups];         // [g]: state lane % 4 of token 4 g + lane / 4 % 4
    __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t rows, int lane, int row_bytes, int n0) {
#pragma unroll
        for (int g = 0; g < kGroups; ++g) raw[g].load(rows, (4 * g + lane / 4 % 4) * row_bytes + (n0 + lane % 4) * (kF32 ? 4 : 2));
    }
    __device__ __forceinline__ float value(int g) const { return raw[g][0]; }
};

}  // namespace scan
}  // namespace wkv6
