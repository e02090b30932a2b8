// Where the gradients of the selective scan and of the short convolution keep what their workgroups leave for others, in sums over tokens and in states in
// front of chunks.  Sequences lie in any order (offsets may fall), and a call's memory grows with its rows and sequences, not with the longest
// sequence that may come, so places go by what no two sequences share: their rows, and their number.  Shared with a host-side check.
#pragma once

#if defined(__HIPCC__)
#define WKV6_HD __host__ __device__
#else
#define WKV6_HD
#endif

namespace wkv6 {

// A sequence's first row, and its tokens; Args has B, T, rows and offsets.
template <typename Args>
WKV6_HD inline long long first_row_of(const Args& a, int b) {
    if (!a.offsets) return static_cast<long long>(b) * a.T;
    const long long f = a.offsets[b];
    return f < 0 ? 0 : f > a.rows ? a.rows : f;
}
template <typename Args>
WKV6_HD inline int tokens_of(const Args& a, int b) {
    if (!a.offsets) return a.T;
    const long long e = a.offsets[b + 1], len = (e < 0 ? 0 : e > a.rows ? a.rows : e) - first_row_of(a, b);
    return static_cast<int>(len < 0 ? 0 : len > a.T ? a.T : len);
}

// Whether b is a sequence, and a row its own.  Whoever walks a sequence leaves its number beside its rows; what stands there of rows of nobody, whatever
// it is, is not the number of a sequence that has them.
template <typename Args>
WKV6_HD inline bool owns(const Args& a, int b, long long row) {
    if (b < 0 || b >= a.B) return false;
    const long long at = row - first_row_of(a, b);
    return at >= 0 && at < tokens_of(a, b);
}

// A sequence's segments of seg_len tokens; one of none if it has no tokens.
WKV6_HD inline int segments_of(int tokens, int seg_len) {
    return tokens <= seg_len ? 1 : static_cast<int>((static_cast<unsigned>(tokens) - 1) / static_cast<unsigned>(seg_len)) + 1;
}

// Places of the segments' sums, one behind the other: segment s of sequence b at s + the segments of the sequences in front of b.  That is b where a call has
// one segment a sequence, and b segs + s without offsets.  Sequences that do not overlap have rows / seg_len + B at most; of others, what does not fit
// is left out.
WKV6_HD constexpr long long share_places(int B, long long rows, int segs, int seg_len, bool packed) {
    return segs == 1 ? B : packed ? (B > 0 ? rows / seg_len + B : 0) : static_cast<long long>(B) * segs;
}

// The same without counting, for short workgroups: a sequence's last segment at `whole` + its number, the others, which are whole, by their first row: whole
// segments start a segment apart at least, so that no two share a place.  Of the places by row some are nobody's; whoever comes in front of them in the order of rows
// sets them to nought: a sequence with rows those behind its own, up to the first of the sequence that starts next, and number 0 those in front of all.
WKV6_HD constexpr long long whole_places(long long rows, int segs, int seg_len) { return segs == 1 ? 0 : rows / seg_len; }
WKV6_HD inline long long place_of_row(long long row, int seg_len) { return row >> __builtin_ctz(static_cast<unsigned>(seg_len)); }   // (the convolution's are powers of two)
// The first row from `row` on at which sequence b starts, if it has rows; else `rows`.
template <typename Args>
WKV6_HD inline long long start_behind(const Args& a, int b, long long row) {
    const long long first = first_row_of(a, b);
    return first >= row && tokens_of(a, b) > 0 ? first : a.rows;
}

// Places of the states in front of chunks: by the chunk's first row.  Those of whole chunks are a chunk apart at least, so that no two share one; a state in front of a
// sequence's last chunk is not kept.
WKV6_HD constexpr long long chunk_place(long long row, int chunk) { return row / chunk; }
WKV6_HD constexpr long long chunk_places(long long rows, int chunk) { return rows / chunk + 1; }

}  // namespace wkv6
