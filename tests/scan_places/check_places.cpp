// Host-side check of where the gradients of the selective scan and the short convolution keep what their workgroups leave (csrc/scan_places.h): for random
// offsets, rising or falling, outside the rows or not, that let no two sequences overlap, no two segments' sums and no two kept states share a place, all places are inside
// what a call asks memory for, and the rows that are found to be somebody's are those of the sequences.  Of offsets that overlap, that places stay inside.
#include <algorithm>
#include <cstdio>
#include <random>
#include <vector>

#include "../../paper_2407_12077_amd/csrc/scan_places.h"

struct Call {
    int B, T;
    long long rows;
    const int* offsets;
};

static int fail(const char* what, const Call& a, int seg_len) {
    std::printf("FAIL %s: rows %lld T %d seg_len %d offsets", what, a.rows, a.T, seg_len);
    for (int b = 0; a.offsets && b <= a.B; ++b) std::printf(" %d", a.offsets[b]);
    std::printf("\n");
    return 1;
}

static int check(const Call& a, long long* apart) {
    std::vector<int> owners(static_cast<size_t>(a.rows));
    bool overlap = false;
    for (int b = 0; b < a.B; ++b)
        for (int t = 0; t < wkv6::tokens_of(a, b); ++t) overlap |= owners[static_cast<size_t>(wkv6::first_row_of(a, b) + t)]++ > 0;
    *apart += !overlap;
    for (long long row = 0; row < a.rows && !overlap; ++row) {
        int owner = -1;                                        // as the walks leave it
        for (int b = 0; b < a.B; ++b)
            if (row >= wkv6::first_row_of(a, b) && row < wkv6::first_row_of(a, b) + wkv6::tokens_of(a, b)) owner = b;
        if ((owner >= 0) != (owners[static_cast<size_t>(row)] > 0)) return fail("rows", a, 0);
        for (int b = -1; b <= a.B; ++b)                        // whatever an earlier call has left
            if (wkv6::owns(a, b, row) != (b >= 0 && b == owner)) return fail("rows of somebody", a, 0);
    }
    for (const int seg_len : {16, 32, 128, a.T > 0 ? a.T : 1}) {
        const int segs = a.T > 0 ? (a.T - 1) / seg_len + 1 : 1;
        const long long places = wkv6::share_places(a.B, a.rows, segs, seg_len, a.offsets != nullptr);
        long long used = 0;
        for (int b = 0; b < a.B; ++b) {
            const int tokens = wkv6::tokens_of(a, b), mine = wkv6::segments_of(tokens, seg_len);
            if (mine < 1 || mine > segs || (mine - 1) * static_cast<long long>(seg_len) >= (tokens > 0 ? tokens : 1)) return fail("segments", a, seg_len);
            if (static_cast<long long>(mine) * seg_len < tokens) return fail("tokens in no segment", a, seg_len);
            if ((segs == 1 || !a.offsets) && used != static_cast<long long>(b) * segs) return fail("places without counting", a, seg_len);
            used += mine;
        }
        if (!overlap && used > places) return fail("sums outside their memory", a, seg_len);
        if (a.offsets && segs > 1) {                           // without counting
            const long long whole = wkv6::whole_places(a.rows, segs, seg_len);
            std::vector<int> left(static_cast<size_t>(places));
            auto next_start = [&](long long row) {
                long long start = a.rows;
                for (int i = 0; i < a.B; ++i) start = std::min(start, wkv6::start_behind(a, i, row));
                return wkv6::place_of_row(start, seg_len);
            };
            auto leave = [&](long long place) { return place >= 0 && place < places && ++left[static_cast<size_t>(place)] > 0; };
            bool inside = true;
            for (int b = 0; b < a.B; ++b) {
                const long long first = wkv6::first_row_of(a, b);
                const int tokens = wkv6::tokens_of(a, b), mine = wkv6::segments_of(tokens, seg_len);
                for (int seg = 0; seg < mine; ++seg) inside &= leave(seg == mine - 1 ? whole + b : wkv6::place_of_row(first, seg_len) + seg);
                if (b == 0)
                    for (long long i = 0, end = next_start(0); i < end; ++i) inside &= leave(i) && i < whole;
                if (tokens == 0) continue;
                const long long end = first + tokens, next = next_start(end);
                if (!overlap && b + 1 < a.B && wkv6::start_behind(a, b + 1, end) == end && next != wkv6::place_of_row(end, seg_len)) return fail("who comes next", a, seg_len);
                for (long long i = wkv6::place_of_row(first, seg_len) + mine - 1; i < next; ++i) inside &= leave(i) && i < whole;
            }
            if (!inside) return fail("a segment outside its memory", a, seg_len);
            for (const int n : left)
                if (n != 1 && !overlap) return fail("a place left by none or by two", a, seg_len);
        }
        for (const int chunk : {8, 16}) {
            if (segs > 1 && seg_len % chunk != 0) continue;
            const long long kept = wkv6::chunk_places(a.rows, chunk);
            std::vector<char> taken(static_cast<size_t>(kept));
            for (int b = 0; b < a.B; ++b)
                for (int t = 0, tokens = wkv6::tokens_of(a, b); t < tokens; t += chunk) {
                    const long long row = wkv6::first_row_of(a, b) + t, seg_row = row - t % seg_len;
                    const long long place = wkv6::chunk_place(seg_row, chunk) + t % seg_len / chunk;       // as a workgroup moves from chunk to chunk
                    if (place < 0 || place >= kept) return fail("states outside their memory", a, seg_len);
                    const int segment_end = t - t % seg_len + seg_len < tokens ? t - t % seg_len + seg_len : tokens;
                    if (t + chunk >= segment_end) continue;                                                  // the segment's last chunk: stays in registers
                    if (taken[static_cast<size_t>(place)]++ && !overlap) return fail("two states in one place", a, seg_len);
                }
        }
    }
    return 0;
}

int main() {
    std::mt19937 random(1);
    auto below = [&](int n) { return static_cast<int>(random() % static_cast<unsigned>(n)); };
    long long apart = 0;
    const std::vector<std::vector<int>> given = {{2000, 3500, 3500, 0, 1500}, {200, 0, 5000}, {100, 200, 0, 90}, {-5, 40, 30, 900, 900, 2000}, {600, 300, 500, 0, 200, 600, 601, 700}};
    for (const auto& offsets : given)
        for (const int T : {9000, 120, 1})
            if (check({static_cast<int>(offsets.size()) - 1, T, 3507, offsets.data()}, &apart)) return 1;
    for (int i = 0; i < 200000; ++i) {
        const int B = 1 + below(6), rows = below(400);
        std::vector<int> offsets(static_cast<size_t>(B) + 1);
        for (int& o : offsets) o = below(rows + 40) - 20;
        if (check({B, below(3) ? 1 + below(500) : 1 + below(40), rows, offsets.data()}, &apart)) return 1;
        if (i % 50 == 0 && check({B, rows, static_cast<long long>(B) * rows, nullptr}, &apart)) return 1;
    }
    std::printf("ok %lld calls without overlap\n", apart);
    return apart > 20000 ? 0 : 1;
}
