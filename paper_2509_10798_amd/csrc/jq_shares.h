// How the work of attention over shared prefixes is shared out among workgroups (jq_shared.hip has the kernels).  Plain integer code
// without any HIP call, so that a host compiler takes it too and a test can walk every workgroup of any call on the CPU.
#pragma once

#include "jq_sweep.h"

namespace jq {

constexpr int kTileRows = 16;  // query rows of one MFMA tile
constexpr int kSharedWaves = 8, kSharedThreads = 64 * kSharedWaves, kSharedJoinThreads = 256;
constexpr int kSharedChip = 256;  // workgroups that run at a time, one a CU

struct SharedPlan {
    int32_t prefix_tiles, own_tiles, own_groups;  // tiles of 16 query rows a workgroup takes, workgroups over the same keys
    int32_t first_groups, first_splits;           // of the first prefix
    int32_t cu_split[JQ_MAX_SEQ + 1];             // a prefix's workgroups (of a layer), summed up
    int32_t own_split[JQ_MAX_SEQ + 1];            // shares of a sequence, summed up
    int32_t cu_part[JQ_MAX_SEQ + 1];              // splits times query rows of the prefixes, summed up
    int32_t prefix_blocks, own_blocks, grid;      // shares of either sweep (of a layer), workgroups that take them
    bool fits;                                    // every launch stays below 2^32 threads
    size_t off_prefix_stats, off_prefix_part, off_own_stats, off_own_part, ws_bytes;
};

// The (share of keys, KV head) and group of query rows that a sweep's workgroup takes.  Eight units lie side by side, on eight XCDs;
// groups of query rows over the same keys eight workgroups apart, so that they meet in one XCD's L2.  Units left over lie as many apart as they
// are: no workgroup is without work, and as many are launched as the plan counts.
struct UnitAt {
    int unit, group;
};
JQ_HD UnitAt unit_at(int at, int units, int groups) {
    const int whole = units & ~7;
    int first = 0, wide = 8;
    if (at >= whole * groups) {
        at -= whole * groups;
        first = whole;
        wide = units - whole;
    }
    const int line = at / wide, octet = line / groups;
    return UnitAt{first + octet * wide + at - line * wide, line - octet * groups};
}

// Workgroups below prefix_blocks take that share of the prefixes, then as all others shares of the sequences: first those that have none of
// a prefix, then around.
JQ_HD int first_own(int bx, int prefix_blocks, int grid) { return bx - prefix_blocks + (bx < prefix_blocks ? grid : 0); }

// How the work is shared out.  Prefixes and sequences are cut into shares, either side by side, on CUs of their own, or, where there is
// much of both, one behind the other on all of them: what a CU reads in a given time is limited, some 25 GB/s, however many of its
// waves ask, so a sweep that has few CUs takes long.  Fewer shares leave fewer parts to write and to join; fewer query rows a workgroup
// (and the prefix read twice, which meets in an XCD's L2) halve them too.  In nanoseconds, fitted to calls on one MI355X: below, us a call with
// 8 KV heads of 4 query heads for all CUs, three, two and one quarter of them for the prefixes; in brackets what is chosen.
//   rows of sequences | of their prefix     query rows a workgroup          half of them
//   24 x 200 | 2048                         128: 25.4 23.9 23.9 [20.0]      64: 26.0 25.9 25.8 22.8
//   24 x 200 | 8192                         128: [30.3] 29.6 31.9 36.0      64: 31.2 32.5 35.3 41.9
//   24 x 200 | 65536                        128: [78.1] 85.8 112 195        64: 91.5 106 143 252
//   32 x 700 | 32768                        128: [64.6] 66.4 76.9 119       64: 71.7 76.4 92.5 150
//   30 x 3000 | 8192                        128: [97.0] 90.8 90.6 95.0      64: 100 94.3 95.4 104
//   92 x 200 | four of 3000 to 12000        128: [62.0] 66.2 82.0 127       64: 73.2 81.5 101 207
//   48 x 64 | 1000                          256: 25.1 25.2 25.2 25.6        128: 25.8 [23.6] 23.7 24.5
//   64 x 100 | 4096                         256: 38.8 36.4 36.8 43.5        128: [36.2] 33.8 36.1 45.7
//   64 x 300 | 32768                        256: [83.5] 86.3 106 174        128: 87.8 95.0 122 211
//   128 x 500 | 16384                       256: [119] 121 137 202          128: 125 131 155 240
//   18 x 64, 4 tokens | 9000, 5000, 3000    256: 46.3 50.0 61.8 100         128: [43.4] 48.2 61.8 115
//   16 x 500 | 131072                       64: [119] 127 154 268
//   10 x 2000 | 8192                        64: 42.6 43.0 42.4 [35.3]
//   60 x 600 | three, 13000 to 31000, 2 heads  128: 40.4 43.7 [39.3] 60.5   64: 42.7 48.3 47.9 72.7
constexpr int64_t kSharedStart = 6000, kSharedNext = 3000, kOwnRow = 22, kPartBytes = 4000;  // (the last: bytes a nanosecond, there and back)
inline int64_t prefix_row_time(int tiles) { return tiles <= 8 ? 25 : 36; }
template <class P>  // Plan, or what a test makes like it
void plan_shared(const P& p, const P& pp, const int32_t* cu_members, SharedPlan* sp) {
    const int own_tiles = (p.rows + kTileRows - 1) / kTileRows;
    sp->own_tiles = own_tiles <= 1 ? 1 : 2;
    sp->own_groups = (own_tiles + sp->own_tiles - 1) / sp->own_tiles;
    const int64_t heads = (int64_t)p.n_layers * p.h_kv;
    int32_t longest = 0, longest_own = 0, most_rows = 0;
    int32_t length[JQ_MAX_SEQ], own_length[JQ_MAX_SEQ], rows[JQ_MAX_SEQ];
    for (int i = 0; i < pp.n_seq; ++i) {
        length[i] = pp.tab.cu_seq[i + 1] - pp.tab.cu_seq[i];
        rows[i] = (cu_members[i + 1] - cu_members[i]) * p.rows;
        longest = std::max(longest, length[i]);
        most_rows = std::max(most_rows, rows[i]);
    }
    for (int s = 0; s < p.n_seq; ++s) {
        own_length[s] = p.tab.cu_seq[s + 1] - p.tab.cu_seq[s];
        longest_own = std::max(longest_own, own_length[s]);
    }
    auto split = [](int32_t rows, int64_t share) { return (int64_t)(((uint32_t)rows + (uint32_t)share - 1) / (uint32_t)share); };
    // The smallest share, in multiples of `unit` rows, that makes no more than `most` workgroups, if any does.
    auto smallest = [](auto blocks, int32_t rows, int64_t unit, int64_t most) {
        int64_t lo = 1, hi = (rows + unit - 1) / unit;
        while (lo < hi) {
            const int64_t mid = (lo + hi) / 2;
            if (blocks(mid * unit) <= most) hi = mid; else lo = mid + 1;
        }
        return lo * unit;
    };
    auto own_blocks = [&](int64_t share) {
        int64_t n = 0;
        for (int s = 0; s < p.n_seq; ++s) n += split(own_length[s], share);
        return n * heads * sp->own_groups;
    };
    constexpr int kChoices = 4;  // all CUs for both, or three, two, one quarter for the prefixes
    int64_t own_of[kChoices], own_n[kChoices];
    for (int c = 0; c < kChoices; ++c) {
        own_of[c] = smallest(own_blocks, longest_own, 256, c ? c * kSharedChip / kChoices : kSharedChip);
        own_n[c] = own_blocks(own_of[c]);
    }
    const int tiles = (most_rows + kTileRows - 1) / kTileRows, natural = tiles <= 1 ? 1 : tiles <= 2 ? 2 : tiles <= 4 ? 4 : tiles <= 8 ? 8 : 16;
    int64_t best = INT64_MAX, share = 1, own_share = 1;
    for (int each = natural; each >= std::max(natural / 2, std::min(natural, 4)); each /= 2) {
        int64_t groups[JQ_MAX_SEQ];
        for (int i = 0; i < pp.n_seq; ++i) groups[i] = (rows[i] + each * kTileRows - 1) / (each * kTileRows);
        auto prefix_blocks = [&](int64_t share) {
            int64_t n = 0;
            for (int i = 0; i < pp.n_seq; ++i) n += split(length[i], share) * groups[i];
            return n * heads;
        };
        for (int c = 0; c < kChoices; ++c) {
            const int64_t size = smallest(prefix_blocks, longest, each <= 2 ? 256 : each == 4 ? 128 : 64, kSharedChip - c * kSharedChip / kChoices);
            const int64_t n = prefix_blocks(size), m = own_n[c];
            const int64_t time = std::min(size, (int64_t)longest) * prefix_row_time(each), own_time = std::min(own_of[c], (int64_t)longest_own) * kOwnRow;
            const int64_t rounds = (n + kSharedChip - 1) / kSharedChip, own_rounds = (m + kSharedChip - 1) / kSharedChip;
            int64_t cost = n + m <= kSharedChip ? kSharedStart + std::max(time, own_time) : rounds * (kSharedStart + time) + own_rounds * (kSharedNext + own_time);
            int64_t parts = 0;
            for (int i = 0; i < pp.n_seq; ++i) parts += split(length[i], size) * rows[i];
            cost += (parts * heads + m * p.rows) * (2 * kHeadDim * (int64_t)sizeof(float)) / kPartBytes;
            if (cost < best) { best = cost; share = size; own_share = own_of[c]; sp->prefix_tiles = each; }
        }
    }
    sp->cu_split[0] = sp->cu_part[0] = sp->own_split[0] = 0;
    int64_t parts = 0, blocks = 0;
    for (int i = 0; i < pp.n_seq; ++i) {
        const int64_t ns = split(length[i], share);
        const int64_t groups = (rows[i] + sp->prefix_tiles * kTileRows - 1) / (sp->prefix_tiles * kTileRows);
        blocks += ns * p.h_kv * groups;
        if (i == 0) { sp->first_groups = (int32_t)groups; sp->first_splits = (int32_t)ns; }
        sp->cu_split[i + 1] = (int32_t)blocks;
        parts += ns * rows[i];
        sp->cu_part[i + 1] = (int32_t)parts;
    }
    for (int s = 0; s < p.n_seq; ++s) sp->own_split[s + 1] = sp->own_split[s] + (int32_t)split(own_length[s], own_share);
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    const size_t pre = (size_t)heads * (size_t)parts, own = (size_t)heads * sp->own_split[p.n_seq] * p.rows;
    sp->off_prefix_stats = 0;
    sp->off_prefix_part = up(pre * sizeof(float) * 2);
    sp->off_own_stats = sp->off_prefix_part + up(pre * kHeadDim * sizeof(float));
    sp->off_own_part = sp->off_own_stats + up(own * sizeof(float) * 2);
    sp->ws_bytes = sp->off_own_part + up(own * kHeadDim * sizeof(float));
    const int64_t own_all = (int64_t)sp->own_split[p.n_seq] * p.h_kv * sp->own_groups, all = blocks + own_all;
    const int64_t joins = (int64_t)p.n_seq * p.h_kv * p.rows;
    sp->fits = parts <= INT32_MAX && all * kSharedThreads <= UINT32_MAX && joins * kSharedJoinThreads <= UINT32_MAX;
    if (!sp->fits) return;
    sp->prefix_blocks = (int32_t)blocks;
    sp->own_blocks = (int32_t)own_all;
    // more than the CUs take at a time, with layers on top: all in one round of workgroups if the prefixes are
    const int64_t most = std::max(kSharedChip / p.n_layers, 1);
    sp->grid = (int32_t)(all <= most || blocks > most ? all : most);
}

}  // namespace jq
