// The head-decay time mix over whole sequences (one decay w_t = exp(g_t) per head and token) and its gradients for gfx950:
//
//     S_t = w_t S_{t-1} + k_t^T v_t        o_t = q_t S_t
//
// in chunks of kC tokens.  With A_t the decays from the chunk's first token to t and S_0 the state in front of the chunk
//
//     o_t = A_t q_t S_0 + sum_{i <= t} P_ti v_i        P_ti = (q_t . k_i) exp(g_{i+1} + .. + g_t)
//     S   = A_last S_0 + sum_i k_i^T (exp(g_{i+1} + .. + g_last) v_i)
//
// four products on the matrix cores.  Decays are only ever exponentials of sums of g inside a block of 16 tokens and products of
// such, never a quotient, so nothing overflows and nothing is subtracted but sums inside a block, which two numbers hold to 2^-31.
//
// The gradients are products of the same form (o, S as above, do the gradient of o):
//     dr = mix(q = do, k = v, v = k; S_0 transposed)     dv = reversed mix(q = k, k = r, v = do)     dk = reversed mix(q = v, k = do, v = r)
// and that of g_t is the sum of r.dr - k.dk from t to the end of any later block plus <dS, S> there: see decay_gradient_kernel.
//
// A workgroup takes one segment of one (sequence, head) and walks its chunks.  Its eleven waves have four parts, so that one's matrix products
// run beside another's vector instructions and waits; they meet at one barrier a chunk:
//   movers     (2) bring the rows straight from memory into LDS, kStages - 1 chunks ahead, and store the read-outs of the chunk before in
//              whole rows
//   a timer    (1) forms the decays two chunks ahead
//   producers  (4) form, one chunk ahead, the part of the read-outs that needs no state: a producer takes 16 queries, P^T (keys x queries)
//              from the rows of k and q as they lie, whose accumulators are, lane by lane, the operand of v^T P^T (v through transposing
//              reads); so P never leaves the registers
//   consumers  (4) own 16 of the 64 value columns each: the state's [64][16] columns stay in registers for the whole walk, and as accumulators
//              of k^T (decayed v) they lie as S^T q^T wants them.  They add that to the producers' part, in its place in LDS
//
// What bounds it.  8 x 4096 tokens x 32 heads, bf16: 537 MB in 119 us, 4.5 TB/s, where a large copy reaches 5.1; a round (64 tokens of every
// workgroup) takes 1.85 us, of which the consumers and the last producer work 1.3, so memory and the barrier share the rest.  One prompt of 131072 tokens: 226
// us for the states and 446 to 514 for the read-outs, 3.2 GB at 4.7 TB/s (k and v are read twice).  Gradients of 8 x 4096 x 32: 394 us for 1.49 GB
// (counted: dv and dk find the rows that they share in an XCD's L2, dr runs the other way), 3.8 TB/s: three rounds of workgroups of 2.05 us a chunk.  fp32
// rows: 5.0 us for 64 tokens of every compute unit (8 x 2048 x 32 160 us), fp32 matrix instructions in series with their LDS reads.
//
// bf16 rows: products of rows are exact in fp32; the computed operands (P, S, decayed v) enter as sums of three bf16, which hold an
// fp32 value whole over its whole range, one product for each; two where only bf16 read-outs come of them.  fp32 rows: fp32 matrix instructions.
#include "head_decay.h"
#include "wkv6_lds_loads.h"
#include "wkv6_math.h"

#include <cmath>
#include <type_traits>

namespace wkv6 {
namespace {

typedef float float4v __attribute__((ext_vector_type(4)));
typedef short short4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef unsigned uint2v __attribute__((ext_vector_type(2)));
typedef unsigned uint4v __attribute__((ext_vector_type(4)));

struct Bf16 {
    short bits;
};

// What differs between the types of rows.  Raw: four consecutive contraction indices of an operand as they lie in a tile.  Fine: four
// computed ones.  A tile is kC rows of kHeadSize values in places of 16 bytes, which a row's number permutes so that the reads below
// take every bank equally often.
template <typename T>
struct Elem;

template <>
struct Elem<Bf16> {
    static constexpr int kSize = 2, kRow = kHeadSize * kSize, kPlaces = kRow / 16;
    typedef short4v Raw;
    template <int kTerms>
    struct Fine {
        short4v term[kTerms];
    };
    // reads of a place of sixteen rows, and of 32 bytes of every other one of eight, take all banks
    __device__ static __forceinline__ int swizzle(int row) { return (row & 6) | (row >> 3 & 1); }
    __device__ static __forceinline__ int at(int row, int place) { return row * kRow + 16 * (place ^ swizzle(row)); }
    // lanes are rows, contraction indices columns 16 q + 4 g4 ..
    __device__ static __forceinline__ Raw row_piece(const char* tile, int row, int q, int g4) {
        return *reinterpret_cast<const Raw*>(tile + at(row, 2 * q + (g4 >> 1)) + 8 * (g4 & 1));
    }
    // lanes are columns c0 + l16, contraction indices rows 16 b + 4 g4 ..: transposing reads, in which lane i of sixteen passes the
    // address of four columns of row i / 4 and gets column i of the four rows.  (A wave with loads into LDS on their way would wait for all
    // of them here, wherever they go: the movers have no such reads.)
    template <int kBlocks>
    __device__ static __forceinline__ void column(const char* tile, int c0, int l16, int g4, Raw (&to)[kBlocks]) {
        typedef short4v __attribute__((address_space(3))) * lds_ptr;
        const int row = 4 * g4 + (l16 >> 2), col = c0 + 4 * (l16 & 3);
        const char* from = tile + at(row, col >> 3) + 8 * (col >> 2 & 1);      // (rows sixteen apart are permuted alike)
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) to[b] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(from + 16 * b * kRow));
    }
    __device__ static __forceinline__ float4v floats(Raw r) {
        const uint2v u = __builtin_bit_cast(uint2v, r);
        return float4v{bf16_lo(u.x), bf16_hi(u.x), bf16_lo(u.y), bf16_hi(u.y)};
    }
    // x as a sum of bf16, largest first: three hold all 24 bits of it, two are 2^-17 off
    template <int kTerms>
    __device__ static __forceinline__ Fine<kTerms> fine(float4v x) {
        Fine<kTerms> f;
#pragma unroll
        for (int i = 0; i < kTerms; ++i) {
            f.term[i] = __builtin_bit_cast(short4v, __builtin_convertvector(x, bf16x4));
            if (i + 1 < kTerms) x -= floats(f.term[i]);
        }
        return f;
    }
    __device__ static __forceinline__ bf16x8 both(Raw a, Raw b) {
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
    }
    template <int kTerms>
    __device__ static __forceinline__ Raw term(const Fine<kTerms>& f, int i) { return f.term[i]; }
    // acc += A B over 32 contraction indices (two pieces)
    __device__ static __forceinline__ float4v mul(Raw a0, Raw a1, Raw b0, Raw b1, float4v acc) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(both(a0, a1), both(b0, b1), acc, 0, 0, 0);
    }
    // products of rows 16 i + l16 of one tile with a row of another
    template <int kCount, int kSize>
    __device__ static __forceinline__ void row_products(const char* ta, const char* tb, int row, int l16, int g4, float4v (&acc)[kSize]) {
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            const bf16x8 b = *reinterpret_cast<const bf16x8*>(tb + at(row, 4 * m + g4));
#pragma unroll
            for (int i = 0; i < kCount; ++i)
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(*reinterpret_cast<const bf16x8*>(ta + at(16 * i + l16, 4 * m + g4)), b,
                                                                 m == 0 ? float4v{0.f, 0.f, 0.f, 0.f} : acc[i], 0, 0, 0);
        }
    }
};

template <>
struct Elem<float> {
    static constexpr int kSize = 4, kRow = kHeadSize * kSize, kPlaces = kRow / 16;
    typedef float4v Raw;
    template <int kTerms>
    using Fine = float4v;
    __device__ static __forceinline__ int swizzle(int row) { return row & 15; }
    __device__ static __forceinline__ int at(int row, int place) { return row * kRow + 16 * (place ^ swizzle(row)); }
    __device__ static __forceinline__ Raw row_piece(const char* tile, int row, int q, int g4) {
        return *reinterpret_cast<const Raw*>(tile + at(row, 4 * q + g4));
    }
    template <int kBlocks>
    __device__ static __forceinline__ void column(const char* tile, int c0, int l16, int g4, Raw (&to)[kBlocks]) {
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int row = 16 * b + 4 * g4 + e, col = c0 + l16;
                to[b][e] = *reinterpret_cast<const float*>(tile + at(row, col >> 2) + 4 * (col & 3));
            }
    }
    __device__ static __forceinline__ float4v floats(Raw r) { return r; }
    template <int kTerms>
    __device__ static __forceinline__ float4v fine(float4v x) { return x; }
    __device__ static __forceinline__ float4v term(float4v f, int) { return f; }
    __device__ static __forceinline__ float4v mul(float4v a0, float4v a1, float4v b0, float4v b1, float4v acc) {
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a0[e], b0[e], acc, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(a1[e], b1[e], acc, 0, 0, 0);
        return acc;
    }
    template <int kCount, int kSize>
    __device__ static __forceinline__ void row_products(const char* ta, const char* tb, int row, int l16, int g4, float4v (&acc)[kSize]) {
#pragma unroll
        for (int i = 0; i < kCount; ++i) acc[i] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int q = 0; q < 4; q += 2) {
            const float4v b0 = row_piece(tb, row, q, g4), b1 = row_piece(tb, row, q + 1, g4);
#pragma unroll
            for (int i = 0; i < kCount; ++i) acc[i] = mul(row_piece(ta, 16 * i + l16, q, g4), row_piece(ta, 16 * i + l16, q + 1, g4), b0, b1, acc[i]);
        }
    }
};

constexpr int kWaves = 4, kMovers = 2, kThreads = 64 * (2 * kWaves + kMovers + 1);  // consumers, producers; movers; the timer
static_assert(kThreads == kMixThreads, "the launch");
constexpr int kDecayPlaces = 3;        // for a chunk's decays: being formed, the producers', the consumers'
constexpr int kStreamed = 2;             // cache policy of the read-outs, non-temporal: prefill 8 x 4096 x 32 117.7 -> 115.6 us, its gradients 390 -> 384
constexpr float kLowest = -128.f;      // exp(-128) is nothing beside the smallest fp32 value: -inf is taken as this

// A decay of many tokens, keep + rest, keep one or nought.  S + (w - 1) S has one rounding of the size of S where w S has two, w's and its own: with a
// decay near one, and the same every time, these would add up over what the state remembers.  A w far from one is taken as it is: w - 1 would keep
// only what it has above 2^-25
struct Factor {
    float keep, rest;
    __device__ __forceinline__ float4v times(float4v s, float4v add) const {       // w s + add, the change first
        const float4v change = s * rest + add;
        return s * keep + change;
    }
    __device__ __forceinline__ Factor then(Factor f) const {
        const float less = fmaf(rest, f.rest, rest) + f.rest;                       // of the product less one, if both are near it
        const bool both = keep * f.keep != 0.f, near_one = both && fabsf(less) < 0.5f;
        const float far = both ? 1.f + less : (keep + rest) * (f.keep + f.rest);
        return {near_one ? 1.f : 0.f, near_one ? less : far};
    }
};

// A chunk's decays by token, in LDS.  In logarithms to base 2 (high, low) or as factors (the others)
template <int kC>
struct Decays {
    float high[kC], low[kC];           // sum of g from the block's first token to this, in two parts: in multiples of 2^-10, which stay exact, and the rest
    float high_key[kC];                // high of tokens that are there, far above nought of others
    float in_block[kC];                // exp2(high + low)
    float to_block[kC];                // from behind this token to the block's end; nought for tokens that are not there
    float in_chunk[kC];                // from the chunk's first token to this
    float to_chunk[kC];                // from behind this token to the chunk's end; nought for tokens that are not there
    float block[kC / 16];              // of whole blocks
    float whole[4];                    // of the whole chunk: a Factor (two values)
};

template <typename T, typename Out, int kC, bool kStates, bool kSums>
struct Layout {
    static constexpr int kTile = kC * Elem<T>::kRow;
    static constexpr int kTiles = kStates ? 2 : 3;               // k, v, q
    static constexpr int kStage = kTile * kTiles;
    static constexpr int kStages = 4;                            // places for a chunk's tiles: the consumers', the producers', two on their way
    static constexpr int kBlocks = kC / 16;
    // terms of a bf16 operand that is no row.  What reaches fp32 results (states, gradients of decays, fp32 read-outs) keeps
    // all bits; for read-outs that are rounded to bf16, 2^-17 is far below that rounding
    static constexpr int kStateTerms = Elem<T>::kSize == 4 ? 1 : 3, kOutTerms = Elem<T>::kSize == 4 ? 1 : sizeof(Out) == 4 || kSums ? 3 : 2;
    static constexpr int kInner = kStates ? 0 : kC * kHeadSize * 4;    // a chunk's read-outs: being formed, completed, stored
    static constexpr int kOffDecays = kStages * kStage;
    static constexpr int kOffInner = kOffDecays + kDecayPlaces * static_cast<int>(sizeof(Decays<kC>));
    static constexpr int kLds = kOffInner + 3 * kInner;
    static constexpr int kLoads = kTile / 1024 / kMovers;        // of a mover and tile,
    static constexpr int kAsked = kLoads * kTiles;               // and chunk
    // stores of read-outs: lanes a row, rows of a store, stores of a mover and chunk
    static constexpr int kRowLanes = sizeof(Out) == 4 ? 16 : 8, kRowsAStore = 64 / kRowLanes, kStores = kC / kMovers / kRowsAStore;
    static constexpr int kLeft = kStates ? 0 : kSums ? 2 * kStores : kStores;      // and of their sums
    static_assert(kLds <= 160 * 1024, "LDS of a compute unit");
};

// All waves, and what they have written to LDS; loads and stores stay on their way (a fence would wait for loads into LDS).  The empty
// statements keep the compiler from moving LDS accesses across, which the barrier alone does not.
__device__ __forceinline__ void lds_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(15 | 3 << 14 | 7 << 4);         // the wave's own LDS reads and writes
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// A value that is the same in all lanes, in a scalar register: what depends on the kernel's argument or on memory through a computed
// index is not known to be, and a descriptor of such would be read lane by lane.
template <typename V>
__device__ __forceinline__ V uniform(V v) {
    if constexpr (sizeof(V) == 8) {
        const uint2v u = __builtin_bit_cast(uint2v, v);
        const uint2v same = {static_cast<unsigned>(__builtin_amdgcn_readfirstlane(u.x)), static_cast<unsigned>(__builtin_amdgcn_readfirstlane(u.y))};
        if constexpr (std::is_pointer_v<V>) {
            // device memory, which the compiler no longer sees: behind flat accesses it waits for all of a wave's LDS reads where it needs one
            typedef __attribute__((address_space(1))) std::remove_pointer_t<V>* Global;
            return (V)__builtin_bit_cast(Global, same);
        } else {
            return __builtin_bit_cast(V, same);
        }
    } else {
        return static_cast<V>(__builtin_amdgcn_readfirstlane(static_cast<int>(v)));
    }
}
__device__ __forceinline__ __amdgpu_buffer_rsrc_t descriptor(const char* base, int bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(uniform(base)), 0, uniform(bytes), 0x00020000);
}
__device__ __forceinline__ Sweep uniform_sweep(const Sweep& w) {
    Sweep u;
    u.q = uniform(w.q); u.k = uniform(w.k); u.v = uniform(w.v);
    u.q_row = uniform(w.q_row); u.k_row = uniform(w.k_row); u.v_row = uniform(w.v_row);
    u.out = uniform(w.out); u.out_row = uniform(w.out_row);
    u.with = uniform(w.with); u.with_row = uniform(w.with_row); u.sums = uniform(w.sums);
    u.state_in = uniform(w.state_in); u.state_out = uniform(w.state_out);
    u.locals = uniform(w.locals); u.anchors = uniform(w.anchors);
    u.reverse = uniform(w.reverse); u.turned = uniform(w.turned); u.locals_turned = uniform(w.locals_turned);
    return u;
}

struct Span {                          // a workgroup's tokens
    int b, h, len;                     // sequence, head, the sequence's tokens
    long long first;                   // its first row
    int seg, segs;                     // segment, and how many the sequence has
    int begin, end;                    // the segment's tokens
};

// Offsets are taken as they are as far as they lie inside the rows: nothing outside the tensors is touched, whatever they hold.
__device__ __forceinline__ Span span_of(const MixArgs& a, int unit, int seg) {
    Span s;
    s.b = uniform(unit / a.H);
    s.h = unit - s.b * a.H;
    if (a.offsets) {
        long long lo = uniform(a.offsets[s.b]), hi = uniform(a.offsets[s.b + 1]);
        lo = lo < 0 ? 0 : lo > a.rows ? a.rows : lo;
        hi = hi < lo ? lo : hi > a.rows ? a.rows : hi;
        s.first = lo;
        s.len = static_cast<int>(hi - lo > a.T ? a.T : hi - lo);
    } else {
        s.first = static_cast<long long>(s.b) * a.T;
        s.len = a.T;
    }
    s.seg = seg;
    s.segs = s.len > 0 ? (s.len - 1) / a.seg_len + 1 : 1;
    s.begin = seg * a.seg_len;
    s.end = s.begin + a.seg_len < s.len ? s.begin + a.seg_len : s.len;
    return s;
}

// The places of a sequence's anchors
struct Anchors {
    int last, last_place, first_place;                          // its last block, its place, and that of the first block if it is another one
    __device__ __forceinline__ Anchors(const MixArgs& a, const Span& s)
        : last((s.len - 1) / a.anchor_len),
          last_place(a.whole_places < 0 ? s.b * a.blocks + last : a.whole_places + s.b),
          first_place(a.whole_places < 0 ? s.b * a.blocks : static_cast<int>(s.first) / a.anchor_len) {}
    __device__ __forceinline__ float4v* of(const float* anchors, int block, const MixArgs& a, const Span& s) const {
        const long long place = block == last ? last_place : first_place + block;
        return reinterpret_cast<float4v*>(const_cast<float*>(anchors)) + (place * a.H + s.h) * (kHeadSize * kHeadSize / 4);
    }
};

// exp of a log-decay from memory
__device__ __forceinline__ float decay_factor(float g) {
    g = g < kLowest ? kLowest : g;                              // (NaN stays)
    return __builtin_amdgcn_exp2f(g * kLog2e);
}

// 2^x for x <= 0, half a unit in the last place off where v_exp_f32 is a whole one: a head's decays are often the same for all tokens, and
// so would be their error.  2^f - 1 by the series, |f| <= 1/2 (first dropped term 5e-9)
__device__ __forceinline__ float exp2_less_1(float f) {
    float q = 1.5252734e-5f;
    q = fmaf(q, f, 1.5403530e-4f);
    q = fmaf(q, f, 1.3333558e-3f);
    q = fmaf(q, f, 9.6181291e-3f);
    q = fmaf(q, f, 5.5504109e-2f);
    q = fmaf(q, f, 2.4022651e-1f);
    q = fmaf(q, f, 6.9314718e-1f);
    return q * f;
}
__device__ __forceinline__ float exp2_near(float x) {
    const float n = __builtin_rintf(x);
    return __builtin_amdgcn_ldexpf(1.f + exp2_less_1(x - n), static_cast<int>(n));
}

template <int kCtrl>
__device__ __forceinline__ float dpp(float v) {                 // (nought from lanes that are not there)
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), kCtrl, 0xf, 0xf, true));
}
// Sum over the lanes of a row of sixteen up to this one
__device__ __forceinline__ float prefix16(float v) {
    v += dpp<0x111>(v);                                         // from one, two, four, eight lanes below
    v += dpp<0x112>(v);
    v += dpp<0x114>(v);
    return v + dpp<0x118>(v);
}
// and from it on
__device__ __forceinline__ float suffix16(float v) {
    v += dpp<0x101>(v);
    v += dpp<0x102>(v);
    v += dpp<0x104>(v);
    return v + dpp<0x108>(v);
}
__device__ __forceinline__ float lane_value(float v, int lane) {
    return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane));
}

template <typename T, typename Out, int kC, bool kStates, bool kSums>
struct Walk {
    using E = Elem<T>;
    using L = Layout<T, Out, kC, kStates, kSums>;
    static constexpr int kBlocks = L::kBlocks;

    const MixArgs& a;
    const Sweep w;
    const Span s;
    char* const lds;
    const int lane, wave, l16, g4;                              // wave of its part
    const int first_chunk, chunks;                              // of the segment
    float4v state[4];                                           // consumers: S[16 i + 4 g4 + e][16 wave + l16]
    Factor total = {1.f, 0.f};                                  // kStates: decay of all chunks so far

    // token of the chunk's first place, by the chunk's number on the walk
    __device__ __forceinline__ int chunk_token(int n) const { return (first_chunk + (w.reverse ? chunks - 1 - n : n)) * kC; }

    // A mover's offsets in a chunk's rows: lanes take 16 bytes each, places permuted.  Rows behind the sequence's last token are
    // that token's again: their factors are nought
    __device__ __forceinline__ void offsets_in(int (&off)[L::kLoads], long long row_bytes, int tokens) const {
        constexpr int kRowsALoad = 1024 / E::kRow;
#pragma unroll
        for (int i = 0; i < L::kLoads; ++i) {
            const int r = (wave * L::kLoads + i) * kRowsALoad + lane / E::kPlaces;
            int t = w.reverse ? kC - 1 - r : r;
            t = t < tokens ? t : tokens - 1;
            off[i] = t * static_cast<int>(row_bytes) + 16 * ((lane % E::kPlaces) ^ E::swizzle(r));
        }
    }
    struct Offsets {                                            // of whole chunks
        int k[L::kLoads], v[L::kLoads], q[L::kLoads];
    };
    __device__ __forceinline__ Offsets whole_offsets() const {
        Offsets o;
        offsets_in(o.k, w.k_row, kC);
        offsets_in(o.v, w.v_row, kC);
        if constexpr (!kStates) offsets_in(o.q, w.q_row, kC);
        return o;
    }
    __device__ __forceinline__ void ask_tile(const char* base, long long row_bytes, int tokens, int token, int to, const int (&whole)[L::kLoads]) const {
        const __amdgpu_buffer_rsrc_t rows = descriptor(base + (s.first + token) * row_bytes + static_cast<long long>(s.h) * E::kRow,
                                                       static_cast<int>((tokens - 1) * row_bytes) + E::kRow);
        typedef __attribute__((address_space(3))) char* lds_ptr;
        char* dst = lds + to + wave * (L::kLoads * 1024);
        if (tokens == kC) {
#pragma unroll
            for (int i = 0; i < L::kLoads; ++i) __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, (lds_ptr)(dst + 1024 * i), 16, whole[i], 0, 0, 0);
        } else {
            int off[L::kLoads];
            offsets_in(off, row_bytes, tokens);
#pragma unroll
            for (int i = 0; i < L::kLoads; ++i) __builtin_amdgcn_raw_ptr_buffer_load_lds(rows, (lds_ptr)(dst + 1024 * i), 16, off[i], 0, 0, 0);
        }
    }
    __device__ __forceinline__ void ask_rows(int n, const Offsets& o) const {
        const int to = n % L::kStages * L::kStage;
        const int token = chunk_token(n), left = s.len - token, tokens = left < kC ? left : kC;
        ask_tile(w.k, w.k_row, tokens, token, to, o.k);
        ask_tile(w.v, w.v_row, tokens, token, to + L::kTile, o.v);
        if constexpr (!kStates) ask_tile(w.q, w.q_row, tokens, token, to + 2 * L::kTile, o.q);
    }
    // The timer's g, a lane a place.  In reverse a token's is that of the token behind it; places without one are cleared later
    __device__ __forceinline__ float read_g(int n) const {
        const int token = chunk_token(n < chunks ? n : chunks - 1);
        int t = token + (w.reverse ? kC - lane : lane);
        t = t < 0 ? 0 : t < s.len ? t : s.len - 1;
        return a.g[(s.first + t) * a.g_row + s.h];
    }

    __device__ __forceinline__ char* inner_of(int n) const { return lds + L::kOffInner + n % 3 * L::kInner; }
    // a lane's four of 16 queries x 16 columns: query l16, columns 4 g4 ..  The queries of a group of columns are permuted by the group, so that
    // whole rows (a lane a group) take all banks too
    __device__ __forceinline__ static int inner_place(int columns, int g, int query) { return columns * 1024 + g * 256 + ((query ^ (4 * columns + g)) & 15) * 16; }
    __device__ __forceinline__ float4v* inner_at(int n, int queries, int columns) const {
        return reinterpret_cast<float4v*>(inner_of(n) + queries * 4096 + inner_place(columns, g4, l16));
    }
    __device__ __forceinline__ char* rows_of(int n) const { return lds + n % L::kStages * L::kStage; }
    __device__ __forceinline__ Decays<kC>& decays(int n) const {
        return *reinterpret_cast<Decays<kC>*>(lds + L::kOffDecays + n % kDecayPlaces * static_cast<int>(sizeof(Decays<kC>)));
    }

    // the chunk's decays from its g, a lane a token
    __device__ __forceinline__ void form_decays(int n, float g) const {
        Decays<kC>& d = decays(n);
        const int at = lane < kC ? lane : 0, t = chunk_token(n) + (w.reverse ? kC - 1 - at : at);
        const bool there = t < s.len;
        const bool has = w.reverse ? t + 1 < s.len : there;
        g = g < kLowest ? kLowest : g;                          // (NaN stays)
        g = has ? g * kLog2e : 0.f;
        // a token that forgets nearly all takes no bits from the differences of tokens behind it: 22 bits hold sixteen parts of up to 185
        const float step = __builtin_rintf(g * 1024.f) * (1.f / 1024.f), high = prefix16(step), low = prefix16(g - step);
        const float pre = high + low, behind = dpp<0x101>(suffix16(g));         // (the factors: nothing is subtracted)
        float block = 0.f, before = 0.f, after = 0.f, all = 0.f;               // sums over this block, those in front of it and behind it
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) {
            const float sum = lane_value(pre, 16 * i + 15);
            block = i == lane >> 4 ? sum : block;
            before += i < lane >> 4 ? sum : 0.f;
            after += i > lane >> 4 ? sum : 0.f;
            all += sum;
        }
        if (lane < kC) {
            d.high[lane] = high;
            d.low[lane] = low;
            d.high_key[lane] = there ? high : 32768.f;           // 2^-32768 is nought
            d.in_block[lane] = exp2_near(pre);
            d.to_block[lane] = there ? exp2_near(behind) : 0.f;
            d.in_chunk[lane] = exp2_near(before + pre);
            d.to_chunk[lane] = there ? exp2_near(behind + after) : 0.f;
            if ((lane & 15) == 0) d.block[lane >> 4] = exp2_near(block);
            if (lane == 0) {
                const bool near_one = fabsf(all) < 0.5f;
                d.whole[0] = near_one ? 1.f : 0.f;
                d.whole[1] = near_one ? exp2_less_1(all) : exp2_near(all);
            }
        }
    }

    // A producer's part of sum_{i <= t} P_ti v_i: 16 queries (with fewer blocks than producers, of a share of the columns).  Loops run over
    // what does not depend on one another innermost, here and in advance: a product waits for the one before it in its sum
    template <int kQ>
    __device__ __forceinline__ void form_inner(int n) const {
        const int j0 = wave / kBlocks * kBlocks;                // block of columns
        const char* tile = rows_of(n);
        const Decays<kC>& d = decays(n);
        const int query = 16 * kQ + l16;
        constexpr int kKeys = kQ + 1, kEven = (kKeys + 1) / 2 * 2;           // blocks of keys, in pairs
        float4v sc[kEven];
        E::template row_products<kKeys>(tile, tile + 2 * L::kTile, query, l16, g4, sc);
        typename E::template Fine<L::kOutTerms> p[kEven];
        float f = d.in_block[query];                            // from behind a block of keys to the query
#pragma unroll
        for (int kb = kQ; kb >= 0; --kb) {
            const int key = 16 * kb + 4 * g4;
            if (kb == kQ) {
                const float4v high = d.high[query] - *reinterpret_cast<const float4v*>(&d.high_key[key]);
                const float4v low = d.low[query] - *reinterpret_cast<const float4v*>(&d.low[key]);
#pragma unroll
                for (int e = 0; e < 4; ++e) sc[kb][e] = key + e <= query ? sc[kb][e] * exp2_near(high[e] + low[e]) : 0.f;
            } else {
                sc[kb] *= *reinterpret_cast<const float4v*>(&d.to_block[key]) * f;
                f *= d.block[kb];
            }
            p[kb] = E::template fine<L::kOutTerms>(sc[kb]);
        }
        if constexpr (kEven > kKeys) p[kKeys] = {};
        typename E::Raw v[kBlocks][kEven];
        float4v acc[kBlocks];
#pragma unroll
        for (int j = 0; j < kBlocks; ++j) {
            E::column(tile + L::kTile, 16 * (j0 + j), l16, g4, v[j]);
            acc[j] = float4v{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int kb = 0; kb < kEven; kb += 2)
#pragma unroll
            for (int i = L::kOutTerms - 1; i >= 0; --i)
#pragma unroll
                for (int j = 0; j < kBlocks; ++j) acc[j] = E::mul(v[j][kb], v[j][kb + 1], E::term(p[kb], i), E::term(p[kb + 1], i), acc[j]);
#pragma unroll
        for (int j = 0; j < kBlocks; ++j) *inner_at(n, kQ, j0 + j) = acc[j];
    }
    template <int kQ>
    __device__ __forceinline__ void produce() const {
        lds_barrier();
        for (int n = 0; n < chunks; ++n) {                      // in front of barrier n
            form_inner<kQ>(n);
            lds_barrier();
        }
        lds_barrier();
    }

    // A consumer's part: the read-outs of the chunk and the state behind it
    __device__ __forceinline__ void advance(int n) {
        const char* tile = rows_of(n);
        const Decays<kC>& d = decays(n);
        // everything is asked for well before it is waited for
        typename E::Raw v[kBlocks], k[4][kBlocks];
        float4v to_chunk[kBlocks], inner[kBlocks], o[kBlocks];
        float in_chunk[kBlocks];
        typename E::Raw row[kBlocks][4];
        if constexpr (!kStates) {
            const char* q = tile + 2 * L::kTile;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int m = 0; m < 4; ++m) row[b][m] = E::row_piece(q, 16 * b + l16, m, g4);
        }
        E::column(tile + L::kTile, 16 * wave, l16, g4, v);
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) to_chunk[b] = *reinterpret_cast<const float4v*>(&d.to_chunk[16 * b + 4 * g4]);
        const Factor whole = {d.whole[0], d.whole[1]};
        __builtin_amdgcn_sched_barrier(0);
        if constexpr (!kStates) {
            typename E::template Fine<L::kOutTerms> st[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) st[i] = E::template fine<L::kOutTerms>(state[i]);
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) o[b] = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int m = 0; m < 4; m += 2)
#pragma unroll
                for (int i = L::kOutTerms - 1; i >= 0; --i)
#pragma unroll
                    for (int b = 0; b < kBlocks; ++b) o[b] = E::mul(E::term(st[m], i), E::term(st[m + 1], i), row[b][m], row[b][m + 1], o[b]);
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                inner[b] = *inner_at(n, b, wave);
                in_chunk[b] = d.in_chunk[16 * b + l16];
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) E::column(tile, 16 * i, l16, g4, k[i]);
        __builtin_amdgcn_sched_barrier(0);
        typename E::template Fine<L::kStateTerms> vd[kBlocks];
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) vd[b] = E::template fine<L::kStateTerms>(E::floats(v[b]) * to_chunk[b]);
        if constexpr (kStates) total = total.then(whole);
        if constexpr (!kStates) {
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
                *inner_at(n, b, wave) = inner[b] + o[b] * in_chunk[b];
        }
        // what the chunk changes of the state first, whose roundings are of its size, and one of the state's, which is the larger with long memories
        float4v sum[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = state[i] * whole.rest;
#pragma unroll
        for (int b = 0; b < kBlocks; b += 2)
#pragma unroll
            for (int t = L::kStateTerms - 1; t >= 0; --t)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] = E::mul(k[i][b], k[i][b + 1], E::term(vd[b], t), E::term(vd[b + 1], t), sum[i]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) state[i][e] = fmaf(state[i][e], whole.keep, sum[i][e]);
    }

    // kSums: a mover's rows that the read-outs are multiplied with, laid out like its stores
    typedef std::conditional_t<sizeof(Out) == 4, float4v, uint4v> With;
    __device__ __forceinline__ void ask_with(int n, With (&to)[L::kStores]) const {
        const int token = chunk_token(n), left = s.len - token, tokens = left < kC ? left : kC;
        const __amdgpu_buffer_rsrc_t rows = descriptor(w.with + (s.first + token) * w.with_row + static_cast<long long>(s.h) * E::kRow,
                                                       static_cast<int>((tokens - 1) * w.with_row) + E::kRow);
#pragma unroll
        for (int i = 0; i < L::kStores; ++i) {
            const int r = (wave * L::kStores + i) * L::kRowsAStore + lane / L::kRowLanes;
            int t = w.reverse ? kC - 1 - r : r;
            t = t < tokens ? t : tokens - 1;
            to[i] = __builtin_bit_cast(With, __builtin_amdgcn_raw_buffer_load_b128(rows, t * static_cast<int>(w.with_row) + lane % L::kRowLanes * 16, 0, 0));
        }
    }

    // A mover's half of the chunk's read-outs, in whole rows, and their sums.  Rows that are not there lie behind a descriptor's end: always
    // the same number of stores.
    __device__ __forceinline__ void store(int n, const With (&with)[L::kStores]) const {
        constexpr int kOutSize = sizeof(Out) == 4 ? 4 : 2;
        const int token = chunk_token(n);
        const int left = s.len - token, tokens = left < kC ? left : kC;
        const int row = static_cast<int>(w.out_row);
        const __amdgpu_buffer_rsrc_t rows = descriptor(w.out + (s.first + token) * w.out_row + static_cast<long long>(s.h) * (kHeadSize * kOutSize),
                                                       (tokens - 1) * row + kHeadSize * kOutSize);
        const __amdgpu_buffer_rsrc_t sums = descriptor(reinterpret_cast<const char*>(w.sums + s.h * a.rows + s.first + token), kSums && w.with ? 4 * tokens : 0);
        const int x = lane % L::kRowLanes;
#pragma unroll
        for (int i = 0; i < L::kStores; ++i) {
            const int r = (wave * L::kStores + i) * L::kRowsAStore + lane / L::kRowLanes, t = w.reverse ? kC - 1 - r : r;
            const char* from = inner_of(n) + (r >> 4) * 4096;
            const int off = t < tokens ? t * row + 16 * x : 0x7ffffff0;
            float sum;
            if constexpr (kOutSize == 4) {
                const float4v o = *reinterpret_cast<const float4v*>(from + inner_place(x >> 2, x & 3, r & 15));
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uint4v, o), rows, off, 0, kStreamed);
                const float4v p = o * with[i];
                sum = (p[0] + p[1]) + (p[2] + p[3]);
            } else {
                const float4v o0 = *reinterpret_cast<const float4v*>(from + inner_place(x >> 1, x % 2 * 2, r & 15));
                const float4v o1 = *reinterpret_cast<const float4v*>(from + inner_place(x >> 1, x % 2 * 2 + 1, r & 15));
                const bf16x8 o = __builtin_convertvector(__builtin_shufflevector(o0, o1, 0, 1, 2, 3, 4, 5, 6, 7), bf16x8);
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uint4v, o), rows, off, 0, kStreamed);
                const float4v p = o0 * Elem<Bf16>::floats(__builtin_bit_cast(short4v, uint2v{with[i].x, with[i].y})) +
                                  o1 * Elem<Bf16>::floats(__builtin_bit_cast(short4v, uint2v{with[i].z, with[i].w}));
                sum = (p[0] + p[1]) + (p[2] + p[3]);
            }
            if constexpr (kSums) {
                sum += dpp<0xB1>(sum);                          // over the row's lanes: neighbours, pairs, fours, eights
                sum += dpp<0x4E>(sum);
                sum += dpp<0x141>(sum);
                if constexpr (L::kRowLanes == 16) sum += dpp<0x140>(sum);
                __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, sum), sums, x == 0 && t < tokens ? 4 * t : 0x7ffffff0, 0, 0);
            }
        }
    }

    // the state's place in memory: [key][value], or turned
    __device__ __forceinline__ int state_at(int i, int e, bool turned) const {
        const int c = 16 * i + 4 * g4 + e, j = 16 * wave + l16;
        return turned ? j * kHeadSize + c : c * kHeadSize + j;
    }
    __device__ __forceinline__ void read_state(const float* from, bool turned, float4v (&to)[4]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (turned) {
                to[i] = *reinterpret_cast<const float4v*>(from + state_at(i, 0, true));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) to[i][e] = from[state_at(i, e, false)];
            }
    }
    __device__ __forceinline__ void write_state(float* to, bool turned, float factor) const {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (turned) {
                *reinterpret_cast<float4v*>(to + state_at(i, 0, true)) = state[i] * factor;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) to[state_at(i, e, false)] = state[i][e] * factor;
            }
    }
    // the state next to the end of chunk n, if a block of anchor_len tokens ends there
    __device__ __forceinline__ void keep_anchor(int n) const {
        const int end = chunk_token(n) + kC;
        if (end % a.anchor_len != 0 && end < s.len) return;
        float4v* to = Anchors(a, s).of(w.anchors, (end - 1) / a.anchor_len, a, s) + threadIdx.x;
#pragma unroll
        for (int i = 0; i < 4; ++i) to[i * 256] = state[i];
    }
};

constexpr int kStateFloats = kHeadSize * kHeadSize;

// Workgroups go to the XCDs in turn; here consecutive indices share one.
__device__ __forceinline__ int index_on_xcd() {
    const int n = gridDim.x, x = blockIdx.x & 7, each = n >> 3, rest = n & 7;
    return x * each + (x < rest ? x : rest) + (blockIdx.x >> 3);
}

// Index: unit outermost, then segment, then sweep; of packed sequences segment outermost.
template <typename T, typename Out, int kC, bool kStates, bool kSums>
__global__ __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 3))) void mix_kernel(const MixArgs a) {
    using L = Layout<T, Out, kC, kStates, kSums>;
    extern __shared__ __align__(16) char lds[];
    // Runs of units on one XCD, which read whole lines of neighbouring heads' rows: 8 x 4096 x 32 126 -> 118 us, 131072 x 32 784 -> 680.  Packed
    // sequences differ in length, and an XCD that has the long ones would work alone: in turn (37 x 12 of up to 2011 tokens,
    // fp32 read-outs, the kernel alone, 74 -> 60; 59 now)
    int at = a.offsets ? static_cast<int>(blockIdx.x) : index_on_xcd();
    const int sweep = uniform(at % a.sweeps);
    at /= a.sweeps;
    const int all_units = a.B * a.H;
    // (and the segments of a packed call one behind the other: with the units outermost the first ones, which the short sequences have too,
    // would share few XCDs: 20 x 8000 x 8 in eight 108 -> 98, in sixteen 121 -> 117)
    const int unit = uniform(a.offsets ? at % all_units : at / a.segs), seg = uniform(a.offsets ? at / all_units : at % a.segs);
    const Sweep w = uniform_sweep(a.sweep[sweep]);
    const Span s = span_of(a, unit, seg);
    if (seg >= s.segs) return;
    const int lane = threadIdx.x & 63, part = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = part % kWaves;
    const int chunks = s.end > s.begin ? (s.end - s.begin + kC - 1) / kC : 0;
    using W = Walk<T, Out, kC, kStates, kSums>;
    W walk{a, w, s, lds, lane, wave, lane & 15, lane >> 4, s.begin / kC, chunks, {}};
    const long long units = static_cast<long long>(a.B) * a.H;
    float* const locals = w.locals + unit * static_cast<long long>(kStateFloats);
    // A call in place: its last segment overwrites what others may not have read yet.  They read a copy in the place of the one segment that hands
    // nothing over, as nothing follows it on the walk.
    const int last = w.reverse ? 0 : s.segs - 1;
    const bool copied = a.segs > 1 && w.state_in && w.state_in == w.state_out;
    float4v* const copy = reinterpret_cast<float4v*>(locals + last * units * kStateFloats);
    if (kStates && (chunks == 0 || seg == last)) {
        const float4v* from = reinterpret_cast<const float4v*>(w.state_in + unit * static_cast<long long>(kStateFloats));
        if (copied && seg == last)
            for (int i = threadIdx.x; i < kStateFloats / 4; i += kThreads) copy[i] = from[i];
        return;
    }

    if (part == 2 * kWaves + kMovers) {                         // the timer
        if (chunks == 0) return;
        float g[4] = {walk.read_g(0), walk.read_g(1), walk.read_g(2), walk.read_g(3)};
        walk.form_decays(0, g[0]);
        if (chunks > 1) walk.form_decays(1, g[1]);
        lds_barrier();
        for (int n = 0; n < chunks; ++n) {
            g[0] = g[2];
            g[2] = g[3];
            g[3] = walk.read_g(n + 4);
            lds_barrier();
            if (n + 2 < chunks) walk.form_decays(n + 2, g[0]);
        }
        if constexpr (!kStates) lds_barrier();
        return;
    }
    if (part >= 2 * kWaves) {                                   // movers
        if (chunks == 0) return;
        constexpr int kAhead = L::kStages - 1;
        const typename W::Offsets offsets = walk.whole_offsets();
        for (int n = 0; n < kAhead && n < chunks; ++n) walk.ask_rows(n, offsets);
        wait_loads<0>();
        lds_barrier();
        typename W::With with[2][L::kStores];
        auto round = [&](int n, typename W::With(&asked)[L::kStores], typename W::With(&used)[L::kStores]) {
            // all rows of chunk n + 1 are there, chunk n - 1 is done with, and what the last round formed can be read
            lds_barrier();
            if constexpr (kSums)
                if (w.with) walk.ask_with(n, asked);
            __builtin_amdgcn_sched_barrier(0);
            const bool more = n + kAhead < chunks;
            if (more) walk.ask_rows(n + kAhead, offsets);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (!kStates)
                if (n > 0) walk.store(n - 1, used);
            // rows of chunk n + 2, asked for a round ago: behind them that round's and this one's stores and this one's loads
            if (!more) wait_loads<0>();
            else if (n < 2) wait_loads<L::kAsked>();
            else wait_loads<L::kAsked + 2 * L::kLeft>();
        };
        for (int n = 0; n < chunks; n += 2) {
            round(n, with[0], with[1]);
            if (n + 1 < chunks) round(n + 1, with[1], with[0]);
        }
        if constexpr (!kStates) {
            lds_barrier();
            walk.store(chunks - 1, with[(chunks - 1) & 1]);
        }
        return;
    }
    if (part >= kWaves) {                                       // producers
        if (kStates) {
            for (int n = 0; n < chunks + 1; ++n) lds_barrier();
        } else if (chunks > 0) {
            const int q = wave % L::kBlocks;
            if (q == 0) walk.template produce<0>();
            else if (q == 1) walk.template produce<1>();
            else if constexpr (L::kBlocks > 2) {
                if (q == 2) walk.template produce<2>();
                else walk.template produce<3>();
            }
        }
        return;
    }

    Factor* const totals = reinterpret_cast<Factor*>(w.locals + a.segs * units * kStateFloats) + unit;
#pragma unroll
    for (int i = 0; i < 4; ++i) walk.state[i] = float4v{0.f, 0.f, 0.f, 0.f};
    if constexpr (!kStates) {
        if (w.state_in) walk.read_state(copied ? reinterpret_cast<const float*>(copy) : w.state_in + unit * static_cast<long long>(kStateFloats), w.turned, walk.state);
        // and what the segments in front of this one hand over, in the walk's order
        const int count = w.reverse ? s.segs - 1 - seg : seg;
        constexpr int kAtOnce = 4;                              // asked for together
        for (int x0 = 0; x0 < count; x0 += kAtOnce) {
            float4v add[kAtOnce][4];
            Factor decay[kAtOnce];
#pragma unroll
            for (int x = 0; x < kAtOnce; ++x) {
                const int from = x0 + x < count ? x0 + x : count - 1, other = w.reverse ? s.segs - 1 - from : from;
                walk.read_state(locals + other * units * kStateFloats, w.locals_turned, add[x]);
                decay[x] = totals[other * units];
            }
#pragma unroll
            for (int x = 0; x < kAtOnce; ++x)
                if (x0 + x < count)
#pragma unroll
                    for (int i = 0; i < 4; ++i) walk.state[i] = decay[x].times(walk.state[i], add[x][i]);
        }
    }
    if (chunks > 0) {
        lds_barrier();
        for (int n = 0; n < chunks; ++n) {
            lds_barrier();
            if (!kStates && w.anchors && w.reverse) walk.keep_anchor(n);
            walk.advance(n);
            if (!kStates && w.anchors && !w.reverse) walk.keep_anchor(n);
        }
        if constexpr (!kStates) lds_barrier();
    }
    if constexpr (kStates) {
        walk.write_state(locals + seg * units * kStateFloats, w.locals_turned, 1.f);
        if (threadIdx.x == 0) totals[seg * units] = walk.total;
    } else if (w.state_out && seg == last) {
        float factor = 1.f;
        if (w.reverse && s.len > 0) factor = decay_factor(a.g[s.first * a.g_row + s.h]);
        walk.write_state(w.state_out + unit * static_cast<long long>(kStateFloats), w.turned, factor);
    }
}

// dg.  exp(G_t - G_i) with G the running sum of g makes dL/dG_t = r_t . dr_t - k_t . dk_t, plus <dS, S> for a state handed on, so
//     dg_t = sum_{t <= s <= a} (r_s . dr_s - k_s . dk_s) + w_{a+1} <dS_{a+1}, S_a>
// for any a >= t; dS_{a+1} is the gradient of the state behind token a + 1, and behind the last token that of state_out.  The sums nearly
// cancel, so a is the end of t's block of anchor_len tokens and not of the sequence.  r_s . dr_s and k_s . dk_s are fp32 sums of 64 fp32 products, formed
// beside the read-outs: exact products added in 64 bits there made the gradients of 8 x 4096 x 32 416 us where they took 398, packed ones of 20 x 3000 x 12
// 96 and 90.  From there on all is in 64 bits but a block's partial sum of one decay a head, which is rounded to fp32 once.  Errors of dg are
// 1.3e-7 to 2.2e-6 of its root mean square, where chunks in 32 bits with these products in 64 are 3e-7 to 4.2e-6 off.
// A workgroup per unit and block.  15 us of the 8 x 4096 x 32 gradients' 408: 24 MB, and 256 tokens at a time in series.
__global__ __launch_bounds__(kDecayGradientThreads) void decay_gradient_kernel(const MixArgs a, const float* r_sums, const float* k_sums,
                                                             const float* behind, const float* front, float* head_sums, float* dg) {
    __shared__ double part[4];
    int at = index_on_xcd();
    const int h = at % a.H;
    at /= a.H;
    const int blocks = a.blocks, b = at / blocks, block = at - b * blocks;
    const int unit = b * a.H + h;
    const Span s = span_of(a, unit, 0);
    const int t0 = block * a.anchor_len, t1 = t0 + a.anchor_len < s.len ? t0 + a.anchor_len : s.len;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (t0 >= t1) {
        if (head_sums && threadIdx.x == 0) head_sums[(static_cast<long long>(b) * blocks + block) * a.H + h] = 0.f;
        return;
    }
    const Anchors anchors(a, s);
    const float4v *x = anchors.of(behind, block, a, s), *y = anchors.of(front, block, a, s);
    double dot = 0.;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float4v p = x[i * 256 + threadIdx.x] * y[i * 256 + threadIdx.x];
        dot += static_cast<double>((p[0] + p[1]) + (p[2] + p[3]));
    }
    auto wave_sum = [](double v) {
#pragma unroll
        for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m);
        return v;
    };
    dot = wave_sum(dot);
    if (lane == 0) part[wave] = dot;
    __syncthreads();
    double after = (part[0] + part[1]) + (part[2] + part[3]);
    if (t1 < s.len) after *= static_cast<double>(decay_factor(a.g[(s.first + t1) * a.g_row + h]));
    __syncthreads();
    // from the block's end, 256 tokens at a time
    double all = 0.;
    const long long base = h * a.rows + s.first;
    for (int e = t1; e > t0; e -= 256) {
        const int t = e - 1 - static_cast<int>(threadIdx.x);
        double v = t >= t0 ? static_cast<double>(r_sums[base + t]) - static_cast<double>(k_sums[base + t]) : 0.;
#pragma unroll
        for (int m = 1; m < 64; m *= 2) {
            const double from = __shfl_up(v, m);
            if (lane >= m) v += from;
        }
        if (lane == 63) part[wave] = v;
        __syncthreads();
        double before = after;
        for (int i = 0; i < wave; ++i) before += part[i];
        after += (part[0] + part[1]) + (part[2] + part[3]);
        v += before;
        if (t >= t0) {
            if (head_sums) all += v;
            else dg[(s.first + t) * a.H + h] = static_cast<float>(v);
        }
        __syncthreads();
    }
    if (head_sums) {
        all = wave_sum(all);
        if (lane == 0) part[wave] = all;
        __syncthreads();
        if (threadIdx.x == 0)
            head_sums[(static_cast<long long>(b) * blocks + block) * a.H + h] = static_cast<float>((part[0] + part[1]) + (part[2] + part[3]));
    }
}

// dg of one decay a head: the partial sums of a head, always in the same order.  A wave a head: 4 us, a launch.
__global__ __launch_bounds__(64) void head_sums_kernel(long long count, int H, const float* head_sums, float* dg) {
    double v = 0.;
    for (long long i = threadIdx.x; i < count; i += 64) v += static_cast<double>(head_sums[i * H + blockIdx.x]);
#pragma unroll
    for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m);
    if (threadIdx.x == 0) dg[blockIdx.x] = static_cast<float>(v);
}

constexpr int kChunkBf16 = 64, kChunkF32 = 32;

// f(kernel, LDS bytes) for the kernel of these rows
template <bool kStates, bool kSums, typename F>
hipError_t with_mix(bool f32_rows, bool f32_out, F f) {
    if (f32_rows) return f(&mix_kernel<float, float, kChunkF32, kStates, kSums>, Layout<float, float, kChunkF32, kStates, kSums>::kLds);
    if constexpr (!kStates && !kSums)
        if (f32_out) return f(&mix_kernel<Bf16, float, kChunkBf16, kStates, kSums>, Layout<Bf16, float, kChunkBf16, kStates, kSums>::kLds);
    return f(&mix_kernel<Bf16, Bf16, kChunkBf16, kStates, kSums>, Layout<Bf16, Bf16, kChunkBf16, kStates, kSums>::kLds);
}

template <bool kStates, bool kSums>
hipError_t launch(const MixArgs& a, bool f32_rows, bool f32_out, hipStream_t stream) {
    const unsigned grid = static_cast<unsigned>(static_cast<long long>(a.B) * a.H * a.segs * a.sweeps);
    return with_mix<kStates, kSums>(f32_rows, f32_out, [&](auto kernel, int lds) {
        hipLaunchKernelGGL(kernel, dim3(grid), dim3(kThreads), lds, stream, a);
        return hipGetLastError();
    });
}

}  // namespace

namespace {

// What a call takes in `segs` segments, in microseconds, from what a walk takes for 64 tokens and what memory takes: a compute unit holds one workgroup of
// a walk with read-outs, two of one for the states alone.  full: sequences that the rows would be if all were `tokens` long, times heads.
// Packed sequences differ in length, so that short ones run beside the longest; segments that a short one does not have cost
// their workgroups.
double modelled(double units, double full, double tokens, int segs, bool packed, bool backward, bool f32_rows) {
    const double sweeps = backward ? 3 : 1, each = std::ceil(tokens / segs / kMixBlock), walks = full * sweeps * segs, load = walks < 256. ? walks / 256. : 1.;
    const double per = f32_rows ? (backward ? 4.6 : 4.3) + 1.2 * load : (backward ? 1.6 : 1.4) + 0.6 * load;
    const double stream = full * tokens * (f32_rows ? 256. : 128.) / 4.5e6;          // one read or write of all rows
    double whole = std::ceil(walks / 256.) * (5.5 + each * per);
    double empty = 0.;
    if (packed) {
        const double shares = full * sweeps * tokens / kMixBlock / 256.;
        whole = std::ceil(walks / 256.) * 5.5 + per * (each + std::fmax(0., shares - 0.5 * each)) + 1.6 * std::fmax(0., units * sweeps * segs / 256. - 1.);
        empty = 0.8 * std::fmax(0., units * (backward ? 2 : 1) * segs / 512. - 1.);
    }
    whole = std::fmax(whole, (backward ? 11. : 4.) * stream);
    if (segs == 1) return whole;
    const double states = std::ceil(full * (backward ? 2 : 1) * (segs - 1) / 512.) * each * (f32_rows ? 2. : 0.72) + empty;
    return whole + 4. + 0.2 * segs + std::fmax(states, (backward ? 4. : 2.) * stream * (segs - 1) / segs);
}

}  // namespace

MixPlan plan_mix(int B, int T, int H, long long packed_rows, bool backward, bool f32_rows) {
    const bool packed = packed_rows >= 0;
    const int longest = packed && packed_rows < T ? static_cast<int>(packed_rows) : T;
    const double units = static_cast<double>(B) * H, tokens = longest > 0 ? longest : 1;
    const double full = packed ? std::fmin(units, static_cast<double>(packed_rows) * H / tokens) : units;
    int segs = 1;
    // Pieces are for calls that would leave compute units idle; they read k and v (and r and dout) twice.  Measured, whole / in the planned number of
    // pieces / the best of 1 to 32, us: bf16 1 x 4096 x 32 heads 94.7 / 32.6 (8) / 32.6, 1 x 30000 x 12 659 / 84 (21) / 84 (24), 4 x 2048 x 32 53.2 / 51.0
    // (2) / 51.0; 5 x 4096 x 32 stays whole, 100, where the best cut takes 132 (6).  Gradients: 1 x 4096 x 32 114 / 89.5 (5) / 87.4 (8), 1 x 30000 x 12
    // 754 / 219 (14) / 213 (6); 4 x 2048 x 32 stays whole, 130, against 144 (2).  A modelled gain of under 7 % is left: of 52 sizes and types five are
    // more than 8 % off the best, the furthest 20 %
    // Packed, 20 sequences of up to 8000 tokens x 8 heads 173 / 98 (8) / 93 (4), fp32 rows 564 / 244 (8) / 235 (4); 9 x 1531 x 12 37.6 / 29.3 (6) / 28.4 (4),
    // gradients 51.9 whole against 58 (4), of fp32 rows 128 / 99 (4) / 99; of 40 such sizes and types most are within 8 % of the best, the
    // furthest 16 %.  With 256 units and more whole: packed 37 x 2011 x 12 (bf16 read-outs) 51.6 whole, 67 in two; sequences of one length, whole and as
    // cut by the model, bf16 9 x 4096 x 32 200 and 233, 10 x 199 and 246, 12 x 216 and 216, 9 x 8192 x 32 380 and 440, 300 x 4096 x 1 200 and 237, 33 x
    // 32768 x 8 1520 and 1556; gradients 9 x 4096 x 32 504 and 508, fp32 1250 and 1256; fp32 9 x 4096 x 32 586 and 595, 12 x 590 and 664.  The only
    // ones found that would gain are fp32 prompts of many more tokens, 33 x 8192 x 8 1158 and 1022, 33 x 32768 x 8 5200 and 3860
    if (units < kMixFewUnits) {
        const int whole_ones = packed ? plan_mix(B, T, H, -1, backward, f32_rows).segs : 32;
        const int most = whole_ones > kMixPackedSegments ? whole_ones : kMixPackedSegments;
        double least = 0.93 * modelled(units, full, tokens, 1, packed, backward, f32_rows);
        for (int n = 2; n <= most && n * kMixBlock < longest + kMixBlock; ++n) {
            const double us = modelled(units, full, tokens, n, packed, backward, f32_rows);
            if (us < least) least = us, segs = n;
        }
    }
    MixPlan p;
    const long long each = (static_cast<long long>(tokens) + segs - 1) / segs;
    p.seg_len = static_cast<int>((each + kMixBlock - 1) / kMixBlock * kMixBlock);
    p.segs = longest > 0 ? (longest - 1) / p.seg_len + 1 : 1;
    const int padded = longest > 0 ? (longest - 1) / kMixBlock * kMixBlock + kMixBlock : kMixBlock;
    p.anchor_len = padded < 1024 ? padded : 1024;
    p.blocks = longest > 0 ? (longest - 1) / p.anchor_len + 1 : 0;
    p.places = static_cast<long long>(B) * p.blocks;
    p.whole_places = -1;
    if (packed && p.blocks > 0 && packed_rows / p.anchor_len + B < p.places) {
        p.whole_places = static_cast<int>(packed_rows / p.anchor_len);
        p.places = static_cast<long long>(p.whole_places) + B;
    }
    return p;
}

hipError_t raise_mix_limits() {
    struct Raised;
    return once_per_device<Raised>([] {
        auto raise = [](auto kernel, int lds) { return set_lds_limit(kernel, lds); };
        for (int i = 0; i < 3; ++i) {
            const bool f32_rows = i == 2, f32_out = i > 0;
            hipError_t err = with_mix<false, false>(f32_rows, f32_out, raise);
            if (err == hipSuccess) err = with_mix<true, false>(f32_rows, f32_out, raise);
            if (err == hipSuccess) err = with_mix<false, true>(f32_rows, f32_out, raise);
            if (err != hipSuccess) return err;
        }
        return hipSuccess;
    });
}

hipError_t launch_mix(const MixArgs& a, bool f32_rows, bool f32_out, hipStream_t stream) {
    return a.sweeps > 1 ? launch<false, true>(a, f32_rows, f32_rows, stream) : launch<false, false>(a, f32_rows, f32_out, stream);
}

hipError_t launch_mix_locals(const MixArgs& a, int count, bool f32_rows, hipStream_t stream) {
    MixArgs part = a;
    part.sweeps = count;
    return launch<true, false>(part, f32_rows, f32_rows, stream);
}

hipError_t launch_decay_gradient(const MixArgs& a, const float* r_sums, const float* k_sums, const float* behind, const float* front,
                                 float* head_sums, float* dg, hipStream_t stream) {
    const long long count = static_cast<long long>(a.B) * a.blocks;
    if (count > 0)
        hipLaunchKernelGGL(decay_gradient_kernel, dim3(static_cast<unsigned>(count * a.H)), dim3(kDecayGradientThreads), 0, stream, a, r_sums,
                           k_sums, behind, front, a.g_row == 0 ? head_sums : nullptr, dg);
    const hipError_t err = hipGetLastError();
    return err != hipSuccess || a.g_row != 0 ? err : launch_head_sums(count, a.H, head_sums, dg, stream);
}

hipError_t launch_head_sums(long long count, int H, const float* head_sums, float* dg, hipStream_t stream) {
    hipLaunchKernelGGL(head_sums_kernel, dim3(static_cast<unsigned>(H)), dim3(64), 0, stream, count, H, head_sums, dg);
    return hipGetLastError();
}

}  // namespace wkv6
