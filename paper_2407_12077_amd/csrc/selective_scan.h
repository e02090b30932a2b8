// The selective scan: what its kernels are told (selective_scan.hip, selective_scan_step.hip, selective_scan_backward.hip) and how long axes are cut.
#pragma once
#include <hip/hip_runtime.h>

#include "scan_places.h"
#include "wkv6_launch.h"

namespace wkv6 {

constexpr int kScanChannels = 64;      // of a workgroup: a lane each
constexpr int kScanChunk = 16;         // tokens that a workgroup takes at once; segments are whole multiples of it

struct ScanArgs {
    int B, T, D, N;
    long long rows;                    // of the packed tensors
    const void *x, *delta, *z, *b, *c; // z null: no gate
    long long x_row, delta_row, z_row, bc_row;   // bytes from token to token
    const float *a, *bias, *skip;      // bias, skip may be null
    bool softplus;
    const int* offsets;                // [B + 1] or null: B sequences of T rows
    const float* state_in;             // null: zeros
    int segs, seg_len;                 // a sequence's segments
    // segs > 1: [segs][B][D][N], state_in in front of all, then what segment s - 1 leaves of nothing; behind them the segments' sums
    // of step sizes, [segs][B][D], likewise
    float* locals;
};

// segs segments of seg_len tokens, a multiple of kScanChunk.  packed_rows: of a call with offsets, else -1.
//
// By what a call is modelled to take, in microseconds: a chunk takes a workgroup `alone` if it has a compute unit to itself, and `share` of
// a unit that is full; the pieces' own states cost three quarters of the walk itself (of gradients, both ways, two fifths), and every piece adds
// up what the pieces in front of it leave.  Measured, whole and cut: 4 x 4096 x 4096 359 and 335 us (the model takes it whole), 5 x 4096 x 4096 450 and 497, 8 x 4096 x 4096 452 and 659,
// 1 x 300 x 4096 30 and 19; gradients of 4 x 2048 x 4096 672 and 588, 8 x 2048 x 4096 893 and 1120; 37 packed requests of up to 2011 x 1536 206 and 171, gradients of
// nine of up to 1531 x 768 465 and 90.
struct ScanPlan {
    int segs, seg_len;
};
constexpr int kScanMostSegments = 64;
// Of a packed call with a workgroup for every compute unit, whose pieces' states take as many times the states' memory: 16, and no more workgroups than these, empty ones
// among them.  Microseconds with at most 1, 8, 16 and 32 pieces: 37 of up to 2011 x 1536 210, 189, 175, 200 (64 states 356, 356, 494, 710: there the model cuts too
// much), 100 of up to 4096 x 1024 427, 369, 349, 354, 20 of up to 8192 x 2048 713, 474, 420, 372; gradients of 37 of up to 2011 x 1536 815, 506, 525, 524.  With twice and four times the
// workgroups 63 of 200 and one of 20000 x 2048 take 560 and 511 instead of 803, for 143 and 285 MB of workspace instead of 71; 255 of one and one of 8192 x 4096 stay at 955.
constexpr int kScanPackedSegments = 16, kScanPackedWorkgroups = 16384;
int scan_most_segments(int B, int T, int D, bool packed);
ScanPlan plan_scan(int B, int T, int D, int N, long long packed_rows, bool backward);
inline long long scan_blocks(int D) { return (D + kScanChannels - 1) / kScanChannels; }
inline long long scan_local_floats(const ScanPlan& p, long long B, long long D, int N) { return p.segs > 1 ? p.segs * B * D * (N + 1) : 0; }
constexpr int scan_threads(int N) { return 16 * N; }

// state_out may be null.  With a.segs > 1 the segments' own states first.
hipError_t launch_scan(const ScanArgs& a, void* out, float* state_out, bool f32_rows, bool f32_out, hipStream_t stream);

constexpr int kScanFoldRows = 16;      // whose shares of db and dc a workgroup adds up, a wave each

// Gradients.  Tokens whose decays and states stay in registers on the way back; the states in front of them are kept in `states`.
constexpr int scan_back_chunk(int N) { return N == 8 || N == 64 ? 8 : 16; }
struct ScanGradients {
    const void* dout;
    const float* dstate_out;
    void *dx, *ddelta, *db, *dc, *dz;
    float *da, *dskip, *dbias, *dstate_in;
    // workspace
    float* states;                     // [place][D][N] in front of every chunk but a sequence's last (chunk_place)
    float* behind;                     // segs > 1: [segs][B][D][N] what a segment hands to the one in front of it of nothing; behind
                                       // them the sums of its step sizes [segs][B][D]
    float* rows;                       // [rows][blocks][2 N]: shares of db and dc
    int* owners;                       // with offsets [rows]: the number of the sequence that has the row (owns)
    float* weights;                    // [place][D][N], then [place][2][D]: segments' shares of da, and of dskip and dbias (share_places)
    long long places;                  // of them
    long long* used;                   // how many of these segments have, where they are counted (counts_segments)
};
hipError_t launch_scan_backward(const ScanArgs& a, const ScanGradients& g, bool f32, hipStream_t stream);

// da, dskip, dbias (what is wanted of them) from g.weights; without sequences nought.
hipError_t launch_scan_weights(const ScanArgs& a, const ScanGradients& g, hipStream_t stream);

// The pieces' own states, in a.locals, and what they hand on, in g.behind (selective_scan.hip).
hipError_t launch_scan_pieces(const ScanArgs& a, const ScanGradients& g, bool f32_rows, hipStream_t stream);

// One token a sequence, or a few, one behind the other in the same lanes.  A chunk of 16 takes as long for two as for all; microseconds by chunks and
// so, 256 sequences of 2048 channels and 16 states: of 1 token 57 and 14, of 4 59 and 31, of 8 65 and 46, of 12 68 and 62; 64 of 2048 and 32 states: of 4 27 and 18,
// of 8 27.6 and 26.4, of 12 28 and 35; one of 4096 and 16 states: of 2 5.3 and 4.6, of 8 5.4 and 5.7.
constexpr int kScanFewTokens = 8;
hipError_t launch_scan_step(const ScanArgs& a, void* out, float* state_out, bool f32_rows, bool f32_out, hipStream_t stream);

}  // namespace wkv6
