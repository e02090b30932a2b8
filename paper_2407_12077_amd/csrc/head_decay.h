// The head-decay time mix: what its kernels are told (head_decay.hip, head_decay_step.hip) and how long axes are cut.
#pragma once
#include <hip/hip_runtime.h>

#include "wkv6_launch.h"

namespace wkv6 {

constexpr int kMixBlock = 64;          // segments and anchors are whole multiples of this many tokens
constexpr int kMixThreads = 704;       // of a workgroup

// One product of the mix, o_t = sum_{i <= t} exp(g_{i+1} + .. + g_t) (q_t . k_i) v_i + exp(g_1 + .. + g_t) q_t S_0, with the state
// S[key][value] behind it.  Rows have kHeadSize values a head; strides in bytes from token to token.
// reverse: from the last token to the first, where a token takes the decay of the token behind it in the sequence (the
// last one none), and the state that is handed on has taken the first token's decay too.
struct Sweep {
    const char *q = nullptr, *k = nullptr, *v = nullptr;
    long long q_row = 0, k_row = 0, v_row = 0;
    char* out = nullptr;
    long long out_row = 0;
    const char* with = nullptr;        // rows like q; sums[head][row] = with_t . o_t
    long long with_row = 0;
    float* sums = nullptr;
    const float* state_in = nullptr;   // [B][H][64][64]; null: zeros
    float* state_out = nullptr;        // null: not written
    float* locals = nullptr;           // states of the segments from zero, [segment][unit][64][64], and behind them
                                       // their total decays [segment][unit], two floats each
    float* anchors = nullptr;          // [place][head][4096] the states at blocks of anchor_len tokens: behind the block's last token,
                                       // in reverse in front of it; a private order
    bool reverse = false;
    bool turned = false;               // state_in and state_out hold S[value][key],
    bool locals_turned = false;        // and locals
};

struct MixArgs {
    int B, T, H;
    long long rows;                    // of the packed tensors
    const float* g;
    long long g_row;                   // floats from token to token, 0: one decay a head
    const int* offsets;                // [B + 1] or null: B sequences of T rows
    int segs, seg_len;                 // a sequence's segments; seg_len is a multiple of kMixBlock
    int anchor_len, blocks;            // blocks: of the longest sequence
    int whole_places;                  // anchors' places by rows: see MixPlan; -1: by sequence and block
    int sweeps;
    Sweep sweep[3];
};

// How the token axis is cut: segs segments of seg_len tokens; anchors every anchor_len tokens, at most `blocks` in a sequence.  Multiples of kMixBlock.
// The anchors of a head have `places` places.  A packed call whose sequences differ in length would leave most of B x blocks empty.  There a
// sequence's last block has a place of its own, whole_places + the sequence, and a block in front of it the place first row / anchor_len, below
// whole_places = rows / anchor_len: such blocks are anchor_len rows long, so no two of them that share no row start between the same multiples.
struct MixPlan {
    int segs, seg_len, anchor_len, blocks;
    int whole_places;
    long long places;
};
constexpr int kDecayGradientThreads = 256;
// packed_rows: of a call with offsets, else -1; such a call is cut into at most kMixPackedSegments, or as many as
// the same call of sequences that are all T long.
constexpr int kMixPackedSegments = 8;
constexpr int kMixFewUnits = 256;      // calls of as many or more stay whole: see plan_mix
MixPlan plan_mix(int B, int T, int H, long long packed_rows, bool backward, bool f32_rows);

hipError_t launch_mix(const MixArgs& a, bool f32_rows, bool f32_out, hipStream_t stream);

// The segments' own states, `count` sweeps of a; before launch_mix when a.segs > 1.
hipError_t launch_mix_locals(const MixArgs& a, int count, bool f32_rows, hipStream_t stream);

// dg from the sums (r . dr in r_sums, k . dk in k_sums) and the anchors of both directions.  When the decays are one a head (g_row = 0) partial sums
// [blocks][H] in head_sums are folded into dg [H], which is written without any too; otherwise dg is [rows][H].
hipError_t launch_decay_gradient(const MixArgs& a, const float* r_sums, const float* k_sums, const float* behind, const float* front,
                                 float* head_sums, float* dg, hipStream_t stream);

// dg [H] of one decay a head from `count` rows of partial sums [H]; none: nought.
hipError_t launch_head_sums(long long count, int H, const float* head_sums, float* dg, hipStream_t stream);

// Raises the dynamic LDS limits of all of these, without launching.
hipError_t raise_mix_limits();

// One token a sequence: rows row_stride elements apart.
hipError_t launch_mix_step(int B, int H, const void* r, const void* k, const void* v, long long row_stride, const float* g,
                           long long g_row, const float* state_in, void* out, float* state_out, bool f32_rows, bool f32_out,
                           hipStream_t stream);

}  // namespace wkv6
