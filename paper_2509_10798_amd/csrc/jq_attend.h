// Attention of a sequence's newest tokens over its (pruned) cache, the step that decoding repeats between two evictions
// (paper Section 4.3: decoding continues on the pruned cache):
//
//   s[r,j] = scale * q[r] . k[j]      r: the n_q * G query rows of one KV head, j: the live cache rows that r may see
//   p[r,j] = exp(s[r,j] - lse[r]),    lse[r] = ln sum_j exp s[r,j],    out[r] = sum_j p[r,j] v[j]
//   weights[j] += sum_r p[r,j]        (where the caller accumulates the attention every cached row receives)
//
// K and V are read once, 512 bytes a (row, KV head); the few query rows stay in registers.  One pass with a running maximum m
// and sum z per query row; workgroups that share a sequence leave (m, z, unnormalised out), which the last of them joins, or a
// second launch where that is much.  All sums and statistics are fp32.  Measured on one MI355X, whole calls, 8 KV heads of 4 query
// heads: one token over 131072 rows 97 us (5.5 TB/s; a plain read reaches 6.2), 32 sequences of 2048 rows with weights 55
// (bound by memory), one token over 1000 rows of 2 heads 11 (bound by the round trips of a join), 25 drafted tokens over eight
// paged caches of 29909 rows together 41, 64 over 32832 rows 53 (both: matrix and vector instructions, and waits in step).
//
// Layout.  Both products are v_mfma_f32_16x16x32_bf16, of which lane l holds row (or column) l % 16 and the eight products'
// terms 8 * (l / 16) .. + 7 of either operand, and of the result column l % 16 and rows 4 * (l / 16) .. + 3.  Scores are
// formed transposed, keys x query rows, out of a 16-key tile and 16 query rows: lane l then holds query row l % 16 and keys
// 4 * (l / 16) + e of the tile, which is what the second product wants of its right operand when the terms of its 32-key sum are
// numbered 8 * (l / 16) + 4 * tile + e.  So the probabilities never move between lanes.  The left operand of the second product
// is V transposed: lane l loads 16 bytes (d = 8 * (l % 16) .. + 7) of the rows 4 * (l / 16) + e, a wave's load covers whole rows, and
// byte permutes inside the lane pair the rows up: no value passes through LDS, and no workgroup barrier stands in the sweep.
// out comes out transposed too: lane l holds d = 32 * (l / 16) .. + 31 of query row l % 16, in line with m and z.
//
// The sweeps are templates of how a cache's rows lie and come into registers (Rows16 here, RowsCoded in jq_codes.h) and bodies that more
// than one kernel has (jq_shared.hip).
#pragma once
#include <type_traits>

#include "jq_common.h"

namespace jq {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint32_t au32x4 __attribute__((ext_vector_type(4)));

constexpr int kAttendWaves = 4;
constexpr int kAttendThreads = 64 * kAttendWaves;
constexpr int kOutStride = kHeadDim + 4;  // floats a row of partial output takes in LDS: rows of 128 would meet in the same banks
constexpr int kMostJoinRows = 8;  // query rows whose shares the last workgroup of a sequence joins
constexpr int kMostHeld = 65536;  // bytes of logits that a workgroup holds in LDS
constexpr float kSlack = 8.0f;  // a row's running maximum may lag this far (in powers of two) behind before its sums are rescaled
constexpr float kLargeSum = 16777216.0f;  // or, with many query rows, until a lane's share of the sum is this large

// Which cache rows a query row sees, apart from the live ones' end.
enum AttendMask { kSeeAll = 0, kSeeCausal, kSeeTree };

struct AttendArgs {
    static constexpr int kShare = 0;
    const char* Q; const char* K; const char* V;
    const int32_t* lens;   // DEVICE [n_layers][n_seq] live rows, or null: all
    const uint32_t* seen;  // kSeeTree: DEVICE [n_seq][n_q][words]
    uint16_t* out; float* lse;  // lse may be null
    float* weights;        // [n_layers][h_kv][T], may be null
    float* part;           // unnormalised outputs [n_layers][splits][h_kv][rows][d]
    float2* stats;         // their (m, z), [n_layers][splits][h_kv][rows]; m in powers of two
    float* logits;         // with weights: scale * log2(e) * q . k, [n_layers][h_kv][rows][logit_T]
    int32_t n_layers, n_seq, n_q, h_q, h_kv, group, rows, row_groups, units, n_splits, words;
    int32_t hold_keys;     // rows of the cache whose logits a workgroup holds in LDS at most (those of more than 32 query rows are not held)
    float scale2;          // scale * log2(e)
    int64_t T, logit_T;
    uint64_t* arrived;     // one launch: [n_layers][n_seq][h_kv][row_groups], `tag` and the number of workgroups done
    uint64_t tag;          // 40 bits of the call's own above 24 of zeros; 0: another launch joins
    PageMap pm;
    int32_t cu_seq[JQ_MAX_SEQ + 1];
    int32_t cu_split[JQ_MAX_SEQ + 1];
    const uint8_t* K_scale; const uint8_t* V_scale;  // of codes
};

// Sequences that continue shared prefixes (jq_shared.hip): a sweep over the prefixes, whose query rows are those of all the sequences
// that continue one, and a sweep over the sequences' own rows.  Both always leave parts.
struct PrefixArgs : AttendArgs {  // n_seq, lens, cu_seq: of prefixes; cu_split: in place of splits, their workgroups
    static constexpr int kShare = 1;
    int32_t cu_member[JQ_MAX_SEQ + 1];  // sequences that continue a prefix
    int32_t cu_part[JQ_MAX_SEQ + 1];    // parts of a prefix: splits times query rows, of each layer and KV head
};
struct OwnArgs : AttendArgs {
    static constexpr int kShare = 2;
    int32_t causal;
};

// The query rows that meet the keys of a (layer, sequence, KV head): how many, where the row of token i and head h lies among all
// calls' queries, and where the rows' part of the output begins.
__device__ __forceinline__ int query_rows(const AttendArgs& a, int) { return a.rows; }
__device__ __forceinline__ int64_t query_at(const AttendArgs& a, int layer, int s, int i, int h) { return (((int64_t)layer * a.n_seq + s) * a.n_q + i) * a.h_q + h; }
__device__ __forceinline__ int64_t part_at(const AttendArgs& a, int layer, int, int split, int, int g) {
    return (((int64_t)layer * a.n_splits + split) * a.h_kv + g) * a.rows;
}
__device__ __forceinline__ int query_rows(const PrefixArgs& a, int s) { return (a.cu_member[s + 1] - a.cu_member[s]) * a.n_q * a.group; }
__device__ __forceinline__ int64_t query_at(const PrefixArgs& a, int layer, int s, int i, int h) {
    return (((int64_t)layer * a.cu_member[a.n_seq] + a.cu_member[s]) * a.n_q + i) * a.h_q + h;
}
__device__ __forceinline__ int64_t part_at(const PrefixArgs& a, int layer, int s, int, int mine, int g) {
    const int rows = query_rows(a, s);
    return ((int64_t)layer * a.cu_part[a.n_seq] + a.cu_part[s] + (int64_t)mine * rows) * a.h_kv + (int64_t)g * rows;
}

__device__ __forceinline__ int32_t live_rows(const int32_t* lens, int n_seq, int layer, int s, int cap) {
    return lens ? min(max(lens[(int64_t)layer * n_seq + s], 0), cap) : cap;
}

// First entry of a sequence's logits in a row of logit_T: whole tiles of 32 keys have room in front of the next sequence's.
__device__ __forceinline__ int64_t logit_at(const int32_t* cu_seq, int s) { return 32 * ((int64_t)(cu_seq[s] / 32) + s); }

// What one workgroup leaves for another of the same launch: stored and loaded past the caches that the XCDs do not share.
__device__ __forceinline__ void put_pair(float* p, float x, float y) {
    __hip_atomic_store((uint64_t*)p, (uint64_t)__float_as_uint(x) | (uint64_t)__float_as_uint(y) << 32, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ float2 get_pair(const float* p) {
    const uint64_t v = __hip_atomic_load((const uint64_t*)p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

// The sequence that a split belongs to: all of the table's entries at once, where a binary search would wait for one after the other.
__device__ __forceinline__ int seq_of_split(const AttendArgs& a, int split, int lane) {
    if (a.n_seq == 1) return 0;
    int s = __popcll(__ballot(lane + 1 < a.n_seq && a.cu_split[min(lane + 1, a.n_seq)] <= split));
    if (a.n_seq > 64) s += __popcll(__ballot(lane + 65 < a.n_seq && a.cu_split[min(lane + 65, a.n_seq)] <= split));
    return s;
}

// What the workgroup `bx` of a layer does: which share of a sequence's keys it sweeps, for which KV head and group of query rows.
// Groups of query rows over the same keys lie eight workgroups apart, so that they meet in one XCD's L2.
struct KeyShare {
    int s, split, ns, mine, g, rg;  // sequence, share among all, shares of the sequence, share among these, KV head, group
};
// (Apart from the share itself: one found behind a branch is waited for field by field, in front of the first request.)
__device__ __forceinline__ bool has_share(const AttendArgs& a, int bx) { return bx / (8 * a.row_groups) * 8 + (bx & 7) < a.units; }
__device__ __forceinline__ bool has_share(const PrefixArgs&, int) { return true; }
__device__ __forceinline__ bool has_share(const OwnArgs&, int) { return true; }
__device__ __forceinline__ KeyShare key_share_of(const AttendArgs& a, int bx, int, int lane) {
    const int per = 8 * a.row_groups;
    const int u = bx / per * 8 + (bx & 7), rg = (bx % per) >> 3;
    const int split = u / a.h_kv, g = u - split * a.h_kv, s = seq_of_split(a, split, lane);
    return KeyShare{s, split, a.cu_split[s + 1] - a.cu_split[s], split - a.cu_split[s], g, rg};
}
// Prefixes have as many groups as their own rows ask for (`rows` each): with as many as the largest, workgroups that had nothing to do
// stood between the others, and some CUs were left two of these (three prefixes with 192, 80 and 16 query rows 92 us for 64).
__device__ __forceinline__ KeyShare key_share_of(const PrefixArgs& a, int bx, int rows, int lane) {
    int s = 0, ns = a.n_splits, groups = a.row_groups;  // of one prefix
    if (a.n_seq > 1) {
        s = seq_of_split(a, bx, lane);
        const int mine_rows = (a.cu_member[s + 1] - a.cu_member[s]) * a.n_q * a.group;
        ns = (a.cu_part[s + 1] - a.cu_part[s]) / mine_rows;
        groups = (mine_rows + rows - 1) / rows;
    }
    const UnitAt at = unit_at(bx - a.cu_split[s], ns * a.h_kv, groups);
    const int mine = at.unit / a.h_kv;
    return KeyShare{s, 0, ns, mine, at.unit - mine * a.h_kv, at.group};
}
__device__ __forceinline__ KeyShare key_share_of(const OwnArgs& a, int bx, int, int lane) {
    const UnitAt at = unit_at(bx, a.units, a.row_groups);
    const int split = at.unit / a.h_kv, s = seq_of_split(a, split, lane);
    return KeyShare{s, split, a.cu_split[s + 1] - a.cu_split[s], split - a.cu_split[s], at.unit - split * a.h_kv, at.group};
}

// log2 of a sum: v_log_f32 rounds towards zero and is off by more the larger its result, so it only sees the mantissa.
__device__ __forceinline__ float log2_of(float z) { return (float)__builtin_amdgcn_frexp_expf(z) + __builtin_amdgcn_logf(__builtin_amdgcn_frexp_mantf(z)); }
constexpr float kLn2 = 0.69314718055994531f;

__device__ __forceinline__ float max4(f32x4 x) { return fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])); }

// What sums are multiplied by when their row's maximum moves.  Never 0, so that an infinity among them stays one: 2^-126 of sums that
// this happens to is nothing beside the new ones.
__device__ __forceinline__ float rescale(float from, float to) { return from == to ? 1.0f : __builtin_amdgcn_exp2f(fmaxf(from - to, -126.0f)); }

// Values of V that are not finite.  They make the outputs of their own dimension, of the rows that see their key, infinite or NaN, and
// reach nothing else: log-sum-exps and weights are functions of Q and K.  In the products they would reach rows that do not see
// them (0 * inf), so tiles that some row does not see whole are cleared of them; in the others they spoil their own dimension, but a
// second part of a probability that is 0 or negative makes a NaN of an infinity.  So a wave that has cleared any, or ends with a
// sum that is not finite though its row's terms are, reads its V once more and marks those outputs by the definition alone
// (mark_kinds).  Other calls pay for the look at their sums.
// Whether all of a lane's pieces are finite: the largest exponents of the lower and the upper halves, without a branch a word (some 35 of
// them took 0.8 us of a call).
struct Exponents {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 most = {0, 0};
    __device__ __forceinline__ void add(au32x4 x) {
#pragma unroll
        for (int w = 0; w < 4; ++w) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, x[w] & 0x7F807F80u));
    }
    __device__ __forceinline__ bool finite() const { return max(most[0], most[1]) < 0x7F80; }
};
__device__ __forceinline__ au32x4 cleared(au32x4 x) {  // zeros for what is not finite
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const uint32_t low = (x[w] & 0x7F80u) == 0x7F80u ? 0u : x[w] & 0xFFFFu, high = (x[w] & 0x7F800000u) == 0x7F800000u ? 0u : x[w] & 0xFFFF0000u;
        x[w] = low | high;
    }
    return x;
}
template <int N>
__device__ __forceinline__ bool all_finite(const f32x4 (&o)[N]) {
    float x = 0.0f;
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) x = __builtin_fmaf(o[d][e], 0.0f, x);
    return x == 0.0f;
}
__device__ __forceinline__ float sum_of_row(float z) {  // over the four lanes of a query row
    z += __shfl_xor(z, 16);
    return z + __shfl_xor(z, 32);
}

// The marks of a wave's row tiles, in the layout of their sums: 0, or what stands in for the sum.  Kinds are counted by a product
// over 32 keys: 1 for a NaN, 64 for +inf, 4096 for -inf times 1 where a row sees the key, so that its sums are exact whole numbers.
// tile(i): first key of the wave's tile i, -1 behind the last; sees(r, key): of the lane's query row in row tile r; dim(d): the
// lane's dimension of the left operand in block d.
template <int RT, class Rows, class Tile, class Sees, class Dim>
__device__ __forceinline__ void mark_kinds(f32x4 (&marks)[RT][8], const Rows& rows, int n, int lane, Tile tile, Sees sees, Dim dim) {
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int d = 0; d < 8; ++d) marks[r][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int i = 0, key0 = tile(0); key0 >= 0; key0 = tile(++i)) {
        const uint32_t row0 = rows.row(key0);
        uint32_t at[8];  // the rows of the lane's eight keys; those behind the last are nobody's to see
        Exponents exponents;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            at[k] = rows.v_at(row0 + (uint32_t)min(16 * (k >> 2) + 4 * (lane >> 4) + (k & 3), n - 1 - key0));
            exponents.add(rows.v_piece(at[k], lane));
        }
        if (__all(exponents.finite())) continue;
        au32x4 seen[RT];
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int key = key0 + 16 * (k >> 2) + 4 * (lane >> 4) + (k & 3);
                const uint32_t one = sees(r, key) ? 0x3F80u : 0u;
                seen[r][k >> 1] = k & 1 ? seen[r][k >> 1] | one << 16 : one;
            }
#pragma unroll
        for (int d = 0; d < 8; ++d) {
            au32x4 kinds;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t x = rows.v_value(at[k], dim(d));
                const uint32_t kind = (x & 0x7F80u) != 0x7F80u ? 0u : x & 0x7Fu ? 0x3F80u : x & 0x8000u ? 0x4580u : 0x4280u;
                kinds[k >> 1] = k & 1 ? kinds[k >> 1] | kind << 16 : kind;
            }
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const f32x4 count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kinds), __builtin_bit_cast(bf16x8, seen[r]),
                                                                            f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int c = (int)count[e];
                    const float nan = c & 63 ? __builtin_nanf("") : 0.0f, up = c & 0xFC0 ? __builtin_inff() : 0.0f, down = c >> 12 ? __builtin_inff() : 0.0f;
                    marks[r][d][e] += nan + up - down;
                }
            }
            __builtin_amdgcn_sched_barrier(0);  // (all blocks' comparisons together do not fit the scalar registers)
        }
    }
}

// 32 keys of K and V in registers: k[t][c] is chunk c (32 of the 128 dimensions) of key 16 t + l % 16, v[t][e] 8 dimensions of key
// 16 t + 4 (l / 16) + e.
struct KvTile {
    au32x4 k[2][4], v[2][4];
    __device__ __forceinline__ au32x4 key_piece(int i, int c) const { return k[i][c]; }
    // The lane's dimensions 2 w and 2 w + 1 of its eight keys of V.
    template <int W>
    __device__ __forceinline__ void value_words(uint32_t (&x)[2][4]) const {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[i][e] = v[i][e][W];
    }
};

// One head's rows of one sequence in a bf16 cache [.., rows, KV heads, 128], dense or in pages.
struct Rows16 {
    static constexpr bool kCoded = false;
    static constexpr int waves(int, bool) { return kAttendWaves; }  // of a workgroup, by its tiles of 16 query rows and whether there are weights
    static constexpr int least_waves(int row_tiles) { return row_tiles == 1 ? 3 : 2; }  // of a SIMD that registers have to leave room for
    using Tile = KvTile;
    using Piece = au32x4;             // eight dimensions of a row
    const char* K; const char* V;
    uint32_t stride;
    const_i32_ptr table;
    int shift, n_pages;
    bool paged;

    __device__ __forceinline__ Rows16(const AttendArgs& a, int layer, int s, int g) {
        stride = (uint32_t)a.h_kv * (kHeadDim * 2);
        const int64_t first_row = a.pm.block_table ? ((int64_t)layer * a.pm.n_pages) << a.pm.page_shift : (int64_t)layer * a.T + a.cu_seq[s];
        K = a.K + first_row * stride + g * (kHeadDim * 2);
        V = a.V + first_row * stride + g * (kHeadDim * 2);
        table = (const_i32_ptr)(a.pm.block_table ? a.pm.block_table + (int64_t)s * a.pm.max_pages : nullptr);
        shift = a.pm.page_shift; n_pages = a.pm.n_pages;
        paged = a.pm.block_table != nullptr;
    }
    // The row that holds the first key of a tile; its others follow: a page holds whole tiles (page sizes are powers of two from 32 on).
    __device__ __forceinline__ uint32_t row(int key) const {
        if (!paged) return (uint32_t)key;
        return ((uint32_t)clamp_page(table[key >> shift], n_pages) << shift) + (uint32_t)(key & ((1 << shift) - 1));
    }
    // Where the lane's terms of chunk c of a row of Q lie.
    static __device__ __forceinline__ int q_at(int c, int lane) { return 64 * c + 16 * (lane >> 4); }
    // Requests the tile whose first key is row `row0`; rows past `last` (counted from row0) are taken from `last`.
    __device__ __forceinline__ void load(KvTile& t, uint32_t row0, int last, int lane) const {
        const uint32_t kb = (uint32_t)(lane >> 4) * 16u, vb = (uint32_t)(lane & 15) * 16u;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t at = row0 + (uint32_t)min(16 * i + (lane & 15), last);
            const char* k = K + (at * stride + kb);  // (the rest in the instructions)
#pragma unroll
            for (int c = 0; c < 4; ++c) t.k[i][c] = *(const au32x4*)(k + 64 * c);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t at = row0 + (uint32_t)min(16 * i + 4 * (lane >> 4) + e, last);
                t.v[i][e] = *(const au32x4*)(V + (at * stride + vb));
            }
    }
    // K's or V's rows for lanes that take the eight dimensions 8 * (lane % 16) .. of each, and the bf16 values of these.
    struct Source {
        const char* base;
        uint32_t stride;
        __device__ __forceinline__ Source(const Rows16& rows, bool is_v, int lane) : base((is_v ? rows.V : rows.K) + (lane & 15) * 16), stride(rows.stride) {}
        __device__ __forceinline__ Piece request(uint32_t at) const { return *(const au32x4*)(base + at * stride); }
        __device__ __forceinline__ au32x4 values(Piece x) const { return x; }
    };
    // A row of V by what v_at makes of its number: the same eight dimensions, one of them.
    __device__ __forceinline__ uint32_t v_at(uint32_t at) const { return at * stride; }
    __device__ __forceinline__ au32x4 v_piece(uint32_t at, int lane) const { return *(const au32x4*)(V + (at + (uint32_t)(lane & 15) * 16u)); }
    __device__ __forceinline__ uint32_t v_value(uint32_t at, int d) const { return *(const uint16_t*)(V + (at + (uint32_t)d * 2u)); }
};

// Row tiles (of 16 query rows) of one workgroup: RT.
template <int RT>
struct RowState {
    bf16x8 q[RT][4];   // query row l % 16 of tile i, dimensions 32 c + 8 (l / 16) ..
    f32x4 o[RT][8];    // unnormalised output: d = 32 (l / 16) + 8 e + r of query row l % 16 in o[i][r][e]
    float m[RT], z[RT];  // running maximum (the same in the four lanes of a row) and the lane's own share of the sum
};

// Whether a query row sees a key.  Without branches, and what depends on it is selected: of branches around stores to elements of a
// vector the compiler (ROCm 7.2) has lost the store.
template <int MASK>
__device__ __forceinline__ bool row_sees(const AttendArgs& a, int key, int n, int row_limit, const uint32_t* row_seen) {
    if (MASK == kSeeAll) return key < n;
    if (MASK == kSeeCausal) return key < min(n, row_limit);
    const int j = key - (n - a.n_q);
    const uint32_t bit = row_seen[min(max(j, 0), a.n_q - 1) >> 5] >> (j & 31) & 1u;
    return (key < n) & ((j < 0) | (bit != 0));
}

// One tile of 32 keys.  MASKED: some row may not see some key of it, or the tile reaches past the live rows.
template <int RT, bool MASKED, int MASK, bool KEEP, class Tile>
__device__ __forceinline__ void tile_step(RowState<RT>& st, Tile& t, const AttendArgs& a, int lane, int key0, int n, const int* row_limit,
                                          const uint32_t* const* row_seen, float* hold, bool* was_cleared) {
    if constexpr (MASKED) {
        Exponents exponents;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) exponents.add(t.v[i][e]);
        if (!__all(exponents.finite())) {
            Exponents live;  // (rows that are not live may hold anything, and mark nothing)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    live.add(t.v[i][e] & (key0 + 16 * i + 4 * (lane >> 4) + e < n ? 0xFFFFFFFFu : 0u));
                    t.v[i][e] = cleared(t.v[i][e]);
                }
            *was_cleared |= !__all(live.finite());
        }
    }
    f32x4 s[RT][2];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            f32x4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int c = 0; c < 4; ++c) x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, t.key_piece(i, c)), st.q[r][c], x, 0, 0, 0);
            s[r][i] = x * a.scale2;
        }
    if (MASKED) {
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int key = key0 + 16 * i + 4 * (lane >> 4) + e;
                    s[r][i][e] = row_sees<MASK>(a, key, n, row_limit[r], row_seen[r]) ? s[r][i][e] : -__builtin_inff();
                }
    }
    if (KEEP) {  // `hold`: the lane's place in the tile's part of the held logits
#pragma unroll
        for (int r = 0; r < RT; ++r)
            if (r * kTileRows + (lane & 15) < a.rows) {
#pragma unroll
                for (int i = 0; i < 2; ++i) *(f32x4*)(hold + r * kTileRows * a.hold_keys + 16 * i) = s[r][i];
            }
    }
    // Running maximum: raised, and the sums rescaled, only when a score passes it by more than kSlack; terms stay below 2^8.
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        float top = fmaxf(max4(s[r][0]), max4(s[r][1]));
        if (__any(top > st.m[r] + kSlack)) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float to = top > st.m[r] + kSlack ? top : st.m[r];  // (a row's bits do not depend on the others of its wave)
            const float f = rescale(st.m[r], to);
            st.m[r] = to;
            st.z[r] *= f;
#pragma unroll
            for (int d = 0; d < 8; ++d) st.o[r][d] *= f;
        }
    }
    // Probabilities in two bf16 parts, the rounded value and the rest, so that 2^-16 of them is lost and not 2^-8: out is then as
    // exact as its own rounding leaves it.  The second product doubles, which a call of few rows does not notice: it waits for K
    // and V.
    bf16x8 hi[RT], lo[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const float m = st.m[r] == -__builtin_inff() ? 0.0f : st.m[r];  // nothing seen so far: every term is 0
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                f32x2 p;
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    p[k] = __builtin_amdgcn_exp2f(s[r][i][e + k] - m);
                    st.z[r] += p[k];
                }
                const bf16x2 h = __builtin_convertvector(p, bf16x2);  // (two at a time: one instruction)
                const f32x2 rest = {p[0] - (float)h[0], p[1] - (float)h[1]};
                const bf16x2 l = __builtin_convertvector(rest, bf16x2);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    hi[r][4 * i + e + k] = h[k];
                    lo[r][4 * i + e + k] = l[k];
                }
            }
    }
    auto add_values = [&](auto word) {
        uint32_t x[2][4];
        t.template value_words<word.value>(x);
#pragma unroll
        for (int odd = 0; odd < 2; ++odd) {
            const int d = 2 * word.value + odd;
            au32x4 v;
            const uint32_t sel = odd ? 0x07060302u : 0x05040100u;  // the upper or the lower halves of two registers
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) v[2 * i + e] = __builtin_amdgcn_perm(x[i][2 * e + 1], x[i][2 * e], sel);
            const bf16x8 vt = __builtin_bit_cast(bf16x8, v);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                st.o[r][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, hi[r], st.o[r][d], 0, 0, 0);
                st.o[r][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, lo[r], st.o[r][d], 0, 0, 0);
            }
        }
    };
    add_values(std::integral_constant<int, 0>{});
    add_values(std::integral_constant<int, 1>{});
    add_values(std::integral_constant<int, 2>{});
    add_values(std::integral_constant<int, 3>{});
}

// Where outputs go.  What a kernel needs of its arguments while it stores is copied first: through the reference the compiler has to
// take every store for one to them, and loads them again behind it.
struct OutArgs {
    uint16_t* out; float* lse;
    int32_t n_seq, n_q, h_q, group;
    __device__ __forceinline__ OutArgs(const AttendArgs& a) : out(a.out), lse(a.lse), n_seq(a.n_seq), n_q(a.n_q), h_q(a.h_q), group(a.group) {}
};
// Four dimensions of a query row's output out of its sums; a row that has seen nothing: zeros, and -inf for its log-sum-exp.
__device__ __forceinline__ void store_out(const OutArgs& a, int layer, int s, int g, int row, int d, f32x4 o, float m, float z) {
    const int i = row / a.group, h = g * a.group + row - i * a.group;
    const int64_t q_row = (((int64_t)layer * a.n_seq + s) * a.n_q + i) * a.h_q + h;
    const float inv = z == 0.0f ? 0.0f : 1.0f / z;
    __bf16 y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (__bf16)(o[e] * inv);
    *(uint2*)(a.out + q_row * kHeadDim + d) = *(const uint2*)y;
    if (a.lse && d == 0) a.lse[q_row] = z == 0.0f ? -__builtin_inff() : (m + log2_of(z)) * kLn2;
}

// weights[j] += sum_r 2^(x[r,j] - lse2[r]) for the rows j from `begin` to `end` of the cache, all threads of the workgroup together;
// the logits may have been left by other workgroups of the launch.  A thread takes four pairs of rows at a time, so that sixteen
// loads are under way; the first of them may have been requested earlier (request()).
template <int THREADS>
struct Weigher {
    static constexpr int kPairs = 4;
    const float* x;
    float* w;
    int64_t logit_T;
    int rows, end, j0;
    float2 y[kPairs][4], old[kPairs];

    __device__ __forceinline__ Weigher(const AttendArgs& a, int layer, int s, int g, int begin, int end_)
        : x(a.logits + ((int64_t)layer * a.h_kv + g) * a.rows * a.logit_T + logit_at(a.cu_seq, s)),
          w(a.weights + ((int64_t)layer * a.h_kv + g) * a.T + a.cu_seq[s]), logit_T(a.logit_T), rows(a.rows), end(end_),
          j0(begin + 2 * (int)threadIdx.x) {}
    __device__ __forceinline__ int row(int k) const { return j0 + 2 * k * THREADS; }
    __device__ __forceinline__ void request(int r0) {
        if (j0 >= end) return;
#pragma unroll
        for (int k = 0; k < kPairs; ++k) {
            const int j = row(k) < end ? row(k) : j0;
#pragma unroll
            for (int r = 0; r < 4; ++r) y[k][r] = get_pair(x + min(r0 + r, rows - 1) * logit_T + j);
            if (r0 == 0) old[k] = make_float2(w[j], j + 1 < end ? w[j + 1] : 0.0f);
        }
    }
    __device__ __forceinline__ void add(const float* lse2, bool requested) {
        for (; j0 < end; j0 += 2 * kPairs * THREADS) {
            float2 sum[kPairs];
            for (int r0 = 0; r0 < rows; r0 += 4) {
                if (!requested) request(r0);
                requested = false;
                if (r0 == 0) {
#pragma unroll
                    for (int k = 0; k < kPairs; ++k) sum[k] = make_float2(0.0f, 0.0f);
                }
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (r0 + r < rows) {
                        const float l = lse2[r0 + r];
#pragma unroll
                        for (int k = 0; k < kPairs; ++k) {
                            sum[k].x += __builtin_amdgcn_exp2f(y[k][r].x - l);
                            sum[k].y += __builtin_amdgcn_exp2f(y[k][r].y - l);
                        }
                    }
            }
#pragma unroll
            for (int k = 0; k < kPairs; ++k) {
                if (row(k) < end) w[row(k)] = old[k].x + sum[k].x;
                if (row(k) + 1 < end) w[row(k) + 1] = old[k].y + sum[k].y;
            }
        }
    }
};

// A kernel's only argument, where it lies: read through a reference to the parameter itself, stores in between make the compiler (ROCm
// 7.2) load and divide by its fields once more for every four dimensions of output.
template <class Args>
__device__ __forceinline__ const Args& kernel_args() { return *(const Args*)__builtin_amdgcn_kernarg_segment_ptr(); }

// bx, layer: the workgroup's place in the grid.
template <class Rows, int RT, int MASK, bool KEEP, int WAVES, class Args>
__device__ __forceinline__ void attend_few_rows(const Args& a, int bx, int layer) {
    extern __shared__ __align__(16) float lds[];  // [waves][16 RT][kOutStride], then (m, z) [waves][16 RT]
    constexpr int kThreads = 64 * WAVES;
    constexpr bool kParts = Args::kShare != 0;
    static_assert(!(KEEP && kParts), "weights are those of one sweep");
    float2* lds_stats = (float2*)(lds + WAVES * RT * kTileRows * kOutStride);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    if (!has_share(a, bx)) return;
    const KeyShare share = key_share_of(a, bx, RT * kTileRows, lane);
    const int split = share.split, g = share.g, s = share.s, rg = share.rg, ns = share.ns, mine = share.mine;
    const int row0 = rg * RT * kTileRows;

    // Tiles of 32 keys, dealt to the sequence's waves in turn, so that all of them sweep one moving window of the cache.
    const Rows rows(a, layer, s, g);
    // The first tile is requested before anything else is looked at, the live count too, which only decides whether it matters: rows
    // that are not live yet are the caller's as well, and masked.
    const int step = 32 * WAVES * ns, cap = a.cu_seq[s + 1] - a.cu_seq[s];
    int key = 32 * (WAVES * mine + wave);
    typename Rows::Tile t;
    if (key < cap) rows.load(t, rows.row(key), cap - 1 - key, lane);
    RowState<RT> st;
    int row_limit[RT];
    const uint32_t* row_seen[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = min(row0 + r * kTileRows + (lane & 15), query_rows(a, s) - 1);  // rows past the last repeat it and are not stored
        const int i = row / a.group, h = g * a.group + row - i * a.group;
        const char* q = a.Q + query_at(a, layer, s, i, h) * (kHeadDim * 2);
#pragma unroll
        for (int c = 0; c < 4; ++c) st.q[r][c] = __builtin_bit_cast(bf16x8, *(const au32x4*)(q + Rows::q_at(c, lane)));
#pragma unroll
        for (int d = 0; d < 8; ++d) st.o[r][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        st.m[r] = -__builtin_inff();
        st.z[r] = 0.0f;
        row_limit[r] = i + 1;  // (and the rows in front of the queries' own, below)
        if constexpr (Args::kShare == 2) row_limit[r] = a.causal ? i + 1 : a.n_q;
        row_seen[r] = MASK == kSeeTree ? a.seen + ((int64_t)s * a.n_q + i) * a.words : nullptr;
    }

    const int n = live_rows(a.lens, a.n_seq, layer, s, cap);
    // keys from `open` on are not seen by every row
    int open = MASK == kSeeAll ? n : max(n - a.n_q + (MASK == kSeeCausal ? 1 : 0), 0);
    if constexpr (Args::kShare == 2) open = a.causal ? open : n;
#pragma unroll
    for (int r = 0; r < RT; ++r) row_limit[r] += n - a.n_q;
    // The sequence's count of finished workgroups starts at zero for this call: it holds the call's tag or is given it here.
    uint64_t* arrived = a.arrived + (((int64_t)layer * a.n_seq + s) * a.h_kv + g) * a.row_groups + rg;
    if (RT == 1 && !kParts && a.tag && ns > 1 && threadIdx.x == 0) {
        uint64_t was = __hip_atomic_load(arrived, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if ((was ^ a.tag) >> 24) __hip_atomic_compare_exchange_strong(arrived, &was, a.tag, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    // With weights every row's logits stay in LDS until its sums are known, [rows][hold_keys], a wave's tiles four apart.  (Written
    // out as they are formed they kept reads from being under way: 32 sequences of 2048 rows 71.7 us a call, without weights 58.3.)
    float* held = (float*)(lds_stats + WAVES * RT * kTileRows);
    float* hold = KEEP ? held + (lane & 15) * a.hold_keys + 32 * wave + 4 * (lane >> 4) : nullptr;
    bool was_cleared = false;
    // One tile, and the request of the one that takes its place.
    auto step_of = [&](auto masked, auto& tile) {
        tile_step<RT, masked.value, MASK, KEEP>(st, tile, a, lane, key, n, row_limit, row_seen, hold, &was_cleared);
        if (KEEP) hold += 32 * WAVES;
        key += step;
    };
    if constexpr (Rows::kCoded) {
        // Whole tiles are requested from uniform addresses; where the wave's last one is not whole, the last that is stands in for it
        // until it is known which it is: a branch between two ways of requesting a tile cost a move for each of its registers.
        const int last_whole = (cap & ~31) - 32;
        const bool turns = key + 32 <= open;
        while (key + 32 <= open) {
            step_of(std::false_type{}, t);
            if (key < n) rows.load_whole(t, rows.row(min(key, last_whole)), lane);
        }
        if (turns && key < n && key > last_whole) rows.load(t, rows.row(key), n - 1 - key, lane);
        while (key < n) {
            KvTile values;
            Rows::unpack(values, t, lane);
            step_of(std::true_type{}, values);
            if (key < n) rows.load(t, rows.row(key), n - 1 - key, lane);
        }
    } else {
        while (key + 32 <= open) {
            step_of(std::false_type{}, t);
            if (key < n) rows.load(t, rows.row(key), n - 1 - key, lane);
        }
        while (key < n) {
            step_of(std::true_type{}, t);
            if (key < n) rows.load(t, rows.row(key), n - 1 - key, lane);
        }
    }

    bool marked = was_cleared;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        st.z[r] = sum_of_row(st.z[r]);
        marked |= st.z[r] < __builtin_inff() && !all_finite(st.o[r]);
    }
    if (__any(marked)) {
        f32x4 marks[RT][8];
        auto tile = [&](int i) { const int k = 32 * (WAVES * mine + wave) + i * step; return k < n ? k : -1; };
        auto sees = [&](int r, int k) { return row_sees<MASK>(a, k, n, row_limit[r], row_seen[r]); };
        mark_kinds<RT>(marks, rows, n, lane, tile, sees, [&](int d) { return 8 * (lane & 15) + d; });
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int d = 0; d < 8; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) st.o[r][d][e] = marks[r][d][e] == 0.0f ? st.o[r][d][e] : marks[r][d][e];
    }

    // The waves' sums, in wave order.
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        if (lane < 16) lds_stats[(wave * RT + r) * kTileRows + lane] = make_float2(st.m[r], st.z[r]);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        float m = -__builtin_inff();
#pragma unroll
        for (int w = 0; w < WAVES; ++w) m = fmaxf(m, lds_stats[(w * RT + r) * kTileRows + (lane & 15)].x);
        const float f = rescale(st.m[r], m);
        float* to = lds + ((wave * RT + r) * kTileRows + (lane & 15)) * kOutStride + 32 * (lane >> 4);
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                f32x4 x;
#pragma unroll
                for (int d = 0; d < 4; ++d) x[d] = st.o[r][4 * half + d][e] * f;
                *(f32x4*)(to + 8 * e + 4 * half) = x;
            }
    }
    __syncthreads();
    const int64_t part_row = part_at(a, layer, s, split, mine, g);
    const int rows_here = min(query_rows(a, s) - row0, RT * kTileRows);
    const OutArgs outs(a);
    float* const parts_to = a.part + part_row * kHeadDim;
    float2* const stats_to = a.stats + part_row;
    float* const logits_to = KEEP ? a.logits + ((int64_t)layer * a.h_kv + g) * a.rows * a.logit_T + logit_at(a.cu_seq, s) : nullptr;
    const int64_t logit_T = a.logit_T;
    const int rows_all = a.rows, hold_keys = a.hold_keys;
    for (int item = threadIdx.x; item < rows_here * 32; item += kThreads) {
        const int r = item >> 5, d = (item & 31) * 4, row = row0 + r;
        float m = -__builtin_inff(), z = 0.0f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) m = fmaxf(m, lds_stats[w * RT * kTileRows + r].x);
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float2 mz = lds_stats[w * RT * kTileRows + r];
            z += mz.x == m ? mz.y : mz.y * __builtin_amdgcn_exp2f(mz.x - m);
            o += *(const f32x4*)(lds + (w * RT * kTileRows + r) * kOutStride + d);
        }
        if (ns == 1 && !kParts) {
            store_out(outs, layer, s, g, row, d, o, m, z);
        } else {
            float* to = parts_to + row * kHeadDim + d;
            put_pair(to, o[0], o[1]);
            put_pair(to + 2, o[2], o[3]);
        }
        if (d == 0 && (ns > 1 || KEEP || kParts)) put_pair((float*)(stats_to + row), m, z);
    }
    if (KEEP && ns == 1) {  // all of the sequence is here
        float* lse2 = lds;  // (the sums above have been read by the threads that wait here)
        __syncthreads();
        if ((int)threadIdx.x < rows_all) {
            float m = -__builtin_inff(), z = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) m = fmaxf(m, lds_stats[w * RT * kTileRows + threadIdx.x].x);
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float2 mz = lds_stats[w * RT * kTileRows + threadIdx.x];
                z += mz.x == m ? mz.y : mz.y * __builtin_amdgcn_exp2f(mz.x - m);
            }
            lse2[threadIdx.x] = z == 0.0f ? 0.0f : m + log2_of(z);
        }
        __syncthreads();
        float* w = a.weights + ((int64_t)layer * a.h_kv + g) * a.T + a.cu_seq[s];
        for (int j = threadIdx.x; j < n; j += kThreads) {  // (one workgroup: row j of the cache is held at j)
            float sum = 0.0f;
            for (int r = 0; r < rows_all; ++r) sum += __builtin_amdgcn_exp2f(held[r * hold_keys + j] - lse2[r]);
            w[j] += sum;
        }
        return;
    }
    if (KEEP) {  // the whole share's logits at once, to where the workgroup that weighs finds them
        const int pairs = hold_keys / 2;
        for (int item = threadIdx.x; item < rows_all * pairs; item += kThreads) {
            const int r = item / pairs, j = (item - r * pairs) * 2;
            const uint32_t tile = (uint32_t)j >> 5;
            const int at = (int)(tile / WAVES * ns + mine) * 32 * WAVES + 32 * (int)(tile % WAVES) + (j & 31);
            if (at < ((n + 31) & ~31)) put_pair(logits_to + r * logit_T + at, held[r * hold_keys + j], held[r * hold_keys + j + 1]);
        }
    }
    if (RT > 1 || kParts || !a.tag || ns == 1) return;

    // Whoever completes a sequence joins it; nobody waits.  Data first, then the count of those that have left theirs.
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    int* last = (int*)lds_stats;
    if (threadIdx.x == 0) *last = (int)(__hip_atomic_fetch_add(arrived, 1ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) & 0xFFFFFF) + 1 == ns;
    __syncthreads();
    if (!*last) return;
    if (threadIdx.x == 0) __hip_atomic_store(arrived, 0ull, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);  // a replay of the call counts from here
    // What the join begins with is requested together, statistics, sums and logits: each of them is a round trip past the caches.
    // Sixteen bytes of output a thread; where there are few rows several threads take shares of the shares.
    const int64_t first = (((int64_t)layer * a.n_splits + a.cu_split[s]) * a.h_kv + g) * a.rows + row0, next_share = (int64_t)a.h_kv * a.rows;
    static_assert(kMostJoinRows * 32 <= kThreads, "a thread or more for every four sums");
    const int items = rows_here * 32, part = (int)threadIdx.x / items, item = (int)threadIdx.x - part * items;
    int parts = 1;
    while (2 * parts * items <= kThreads && parts < 8) parts *= 2;
    constexpr int kBatch = 8;
    float2 lo[kBatch], hi[kBatch];
    auto request = [&](int i) {  // shares i, i + parts, ... of the thread's sums
        const float* from = a.part + (first + (item >> 5)) * kHeadDim + (item & 31) * 4;
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const float* p = from + min(i + k * parts, ns - 1) * next_share * kHeadDim;
            lo[k] = get_pair(p);
            hi[k] = get_pair(p + 2);
        }
    };
    request(part);
    Weigher<kThreads> weigher(a, layer, s, g, 0, n);
    if (KEEP) weigher.request(0);
    // Factors of all shares' sums, [rows_here][ns], and the rows' (m, z).
    float* factor = lds;
    float* sums = factor + (rows_here * ns + 3) / 4 * 4;  // [parts][items] outputs of four, at multiples of sixteen bytes
    float* lse2 = (float*)(lds_stats + rows_here);
    __syncthreads();
    for (int r = wave; r < rows_here; r += WAVES) {  // a wave a row, a lane a share (there are 20 at most)
        const float2 mz = lane < ns ? get_pair((const float*)(a.stats + first + r + lane * next_share)) : make_float2(-__builtin_inff(), 0.0f);
        float m = mz.x;
#pragma unroll
        for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
        const float f = rescale(mz.x, m);
        float z = mz.y * f;
#pragma unroll
        for (int d = 32; d; d >>= 1) z += __shfl_xor(z, d);
        if (lane < ns) factor[r * ns + lane] = f;
        if (lane == 0) {
            lds_stats[r] = make_float2(m, z);
            lse2[r] = z == 0.0f ? 0.0f : m + log2_of(z);  // nothing seen: all its logits are -inf
        }
    }
    __syncthreads();
    const int r = item >> 5, d = (item & 31) * 4;
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    if (part < parts) {
        for (int i = part; i < ns; i += kBatch * parts) {
            if (i > part) request(i);
#pragma unroll
            for (int k = 0; k < kBatch; ++k) {
                const bool there = i + k * parts < ns;  // (nothing times 0: a sum may be infinite)
                const float f = factor[there ? r * ns + i + k * parts : 0];
                o += f32x4{there ? lo[k].x : 0.0f, there ? lo[k].y : 0.0f, there ? hi[k].x : 0.0f, there ? hi[k].y : 0.0f} * f;
            }
        }
    }
    if (parts > 1) {
        if (part < parts) *(f32x4*)(sums + 4 * (int)threadIdx.x) = o;
        __syncthreads();
        if (part == 0)
            for (int k = 1; k < parts; ++k) o += *(const f32x4*)(sums + 4 * (k * items + item));
    }
    if (part == 0) store_out(outs, layer, s, g, row0 + r, d, o, lds_stats[r].x, lds_stats[r].y);
    if (KEEP) weigher.add(lse2, true);
}

template <class Rows, int RT, int MASK, bool KEEP, int WAVES>
__global__ __launch_bounds__(64 * WAVES, Rows::least_waves(RT)) void jq_attend_kernel(AttendArgs a) {
    attend_few_rows<Rows, RT, MASK, KEEP, WAVES>(kernel_args<AttendArgs>(), (int)blockIdx.x, (int)blockIdx.y);
}

// Many query rows (more than 32 a KV head).  A wave still holds 32 of them, but the eight waves of a workgroup share the keys: R waves
// over all rows of a group times KW over keys of their own.  K and V go through LDS, where every wave reads all of its keys' rows:
// requested into registers stages ahead, written to one of two buffers, one barrier a stage.  (Every wave reading K and V for itself
// took 117 us for 128 rows behind four prompts, 58 this way.)
// K's rows are read sixteen lanes a row of 256 bytes, piece p of row k at p ^ (k & 15), so that eight lanes' pieces meet in eight
// different bank groups; V is read transposed (ds_read_b64_tr_b16: a lane receives four keys' values of one dimension out of four
// rows of sixteen), piece p of row k at p ^ 2 (k & 7) for the same reason (no bank conflicts are counted).
// What bounds it: waits.  By the counters, us at 2.4 GHz, of a wave's life / of matrix instructions / of vector instructions a SIMD, and the
// share of wave time that waits: 100 rows over eight caches 26 / 6 / 8, 40 %; 128 behind four prompts 40 / 11 / 12, 39 %; 256 over 32832 38 / 14 / 13,
// 32 %.  With R = 4 and 8 a wave has one tile between two barriers (64 keys a stage), so the two waves of a SIMD go through the same chain in
// step: deposit, barrier, reads from LDS, first product, terms, second product.  Tried without gain: four stages ahead, two tiles' terms together, more of V's reads early,
// wave priorities, half of the waves held back behind each barrier.
template <int R>
struct Wide {
    static constexpr int kWaves = 8, kThreads = 64 * kWaves, kRows = 32 * R;
    static constexpr int KW = kWaves / R;                      // waves over the same rows, each with keys of its own
    static constexpr int kKeys = KW == 4 ? 128 : 64;           // of a stage
    static constexpr int kTiles = kKeys / 32 / KW;             // of 32 keys, a wave and stage
    static constexpr int kAhead = KW == 4 ? 1 : 2;             // stages requested ahead: 64 KB
    // Probabilities in one bf16 part, off by 2^-8 of each at most, or in two, 2^-16, for which the second product doubles.  With one, out is
    // off by 1.4 times its own rounding (2-norm against 64 bits 0.0023, 0.0017 with two).  Us a call with one / two: 64 rows over 32832
    // 39.3 / 40.4, 128 behind four prompts 58.8 / 65.2, 100 over eight caches 41.5 / 45.3, 256 over 32832 56 / 68: two while they cost 3 percent, and
    // over shared prefixes always (kExact below says why; 32 sequences behind 32768 rows 59 / 63).
    static constexpr bool kExact = R == 2;
    static constexpr int kEarly = 2;                           // blocks of V requested ahead of their use
    static constexpr int kRequests = kKeys / 2 / kWaves;       // of 1 KB, a wave and stage
    static constexpr int kBuffer = 2 * kKeys * 256;            // K, then V
    static constexpr int kMerge = (kWaves - R) * 32 * (kOutStride * 4 + 8);
    static constexpr int kFlags = 2 * kBuffer > kMerge ? 2 * kBuffer : kMerge;  // behind the buffers a byte a wave
    static constexpr int kLds = kFlags + 16;
};
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;

template <class Rows, int R, int MASK, bool KEEP, class Args>
__device__ __forceinline__ void attend_many_rows(const Args& a, int bx, int layer) {
    extern __shared__ __align__(16) char wide_lds[];
    using W = Wide<R>;
    constexpr int KW = W::KW;
    constexpr bool kParts = Args::kShare != 0;
    // Shared prefixes: most of the query rows are other sequences', and a sequence's outputs do not lose a part to their number.
    constexpr bool kExact = W::kExact || kParts;
    uint8_t* marked = (uint8_t*)wide_lds + W::kFlags;  // [kWaves]: the wave has cleared values of V, or has sums that are not finite
    bool was_cleared = false;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    if (!has_share(a, bx)) return;
    const KeyShare share = key_share_of(a, bx, W::kRows, lane);
    const int split = share.split, g = share.g, s = share.s, rg = share.rg, ns = share.ns, mine = share.mine;
    const int cap = a.cu_seq[s + 1] - a.cu_seq[s];
    const int rw = wave % R, kw = wave / R;
    const int row0 = rg * W::kRows + 32 * rw;

    const Rows rows(a, layer, s, g);

    // This wave's requests of a stage: kRequests times four rows of K or of V, all in one tile of 32 keys.
    constexpr int kPerTile = 8 / W::kRequests;  // waves that share the requests of a tile
    const bool is_v = wave >= W::kWaves / 2;
    const int in_half = wave % (W::kWaves / 2), my_tile = in_half / kPerTile;
    const int my_row = in_half % kPerTile * W::kRequests * 4 + (lane >> 4);  // the first request's row within the tile, 4 apart
    const typename Rows::Source source(rows, is_v, lane);
    // where the requests go: the pieces of rows 4 apart are exchanged by amounts that differ
    int to_lds[W::kRequests];
#pragma unroll
    for (int i = 0; i < W::kRequests; ++i) {
        const int row = my_row + 4 * i, piece = is_v ? (lane & 15) ^ 2 * (row & 7) : (lane & 15) ^ (row & 15);
        to_lds[i] = (is_v ? W::kKeys * 256 : 0) + (my_tile * 32 + row) * 256 + piece * 16;
    }
    auto request = [&](typename Rows::Piece* to, int stage, int live) {  // `live`: rows that may be read
        int key = (mine + stage * ns) * W::kKeys + 32 * my_tile;
        key = min(key, (live - 1) & ~31);  // (a stage may reach past the last tile)
        const int last = live - 1 - key;
        const uint32_t row0 = rows.row(key);
#pragma unroll
        for (int i = 0; i < W::kRequests; ++i) to[i] = source.request(row0 + (uint32_t)min(my_row + 4 * i, last));
    };
    // The first stages are requested before anything else is looked at, the live count too: rows that are not live yet are the
    // caller's as well, and masked.  (What follows, mostly instructions that the cache does not hold yet, takes some 3 us.)
    typename Rows::Piece ahead[W::kAhead][W::kRequests];
#pragma unroll
    for (int i = 0; i < W::kAhead; ++i) request(ahead[i], i, cap);
    const int n = live_rows(a.lens, a.n_seq, layer, s, cap);
    const int open = MASK == kSeeAll ? n : max(n - a.n_q + (MASK == kSeeCausal ? 1 : 0), 0);
    bf16x8 q[2][4];
    f32x4 o[2][8];  // d = 16 r + 4 (l / 16) + e of query row l % 16 in o[i][r][e]
    float m[2], z[2];
    int token[2];   // the query rows' tokens
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int row = min(row0 + r * kTileRows + (lane & 15), query_rows(a, s) - 1);
        const int i = row / a.group, h = g * a.group + row - i * a.group;
        const char* from = a.Q + query_at(a, layer, s, i, h) * (kHeadDim * 2);
#pragma unroll
        for (int c = 0; c < 4; ++c) q[r][c] = __builtin_bit_cast(bf16x8, *(const au32x4*)(from + 64 * c + 16 * (lane >> 4)));
#pragma unroll
        for (int d = 0; d < 8; ++d) o[r][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        m[r] = -__builtin_inff();
        z[r] = 0.0f;
        token[r] = i;
    }

    // Addresses of a wave's reads in buffer 0: K by chunk of the dimensions (16 keys further on: + 4096), V by block of sixteen.
    int k_at[4], v_at[8];
    {
        const int vrow = 4 * (lane >> 4) + ((lane & 15) >> 2);
#pragma unroll
        for (int c = 0; c < 4; ++c) k_at[c] = kw * W::kTiles * 8192 + (lane & 15) * 256 + ((4 * c + (lane >> 4)) ^ (lane & 15)) * 16;
#pragma unroll
        for (int d = 0; d < 8; ++d)
            v_at[d] = W::kKeys * 256 + kw * W::kTiles * 8192 + vrow * 256 + ((2 * d + ((lane & 3) >> 1)) ^ 2 * (vrow & 7)) * 16 + (lane & 1) * 8;
    }
    auto deposit = [&](typename Rows::Piece* pieces, int stage, int buf) {
        au32x4 from[W::kRequests];
#pragma unroll
        for (int k = 0; k < W::kRequests; ++k) from[k] = source.values(pieces[k]);
        if (is_v && (mine + stage * ns) * W::kKeys + W::kKeys > open) {  // some row does not see some key: cleared of what is not finite
            Exponents exponents;
#pragma unroll
            for (int k = 0; k < W::kRequests; ++k) exponents.add(from[k]);
            if (!__all(exponents.finite())) {
                Exponents live;  // (rows that are not live may hold anything, and mark nothing)
                const int key = (mine + stage * ns) * W::kKeys + 32 * my_tile + my_row;
#pragma unroll
                for (int k = 0; k < W::kRequests; ++k) {
                    live.add(from[k] & (key + 4 * k < n ? 0xFFFFFFFFu : 0u));
                    from[k] = cleared(from[k]);
                }
                was_cleared |= !__all(live.finite());
            }
        }
#pragma unroll
        for (int k = 0; k < W::kRequests; ++k) *(au32x4*)(wide_lds + buf * W::kBuffer + to_lds[k]) = from[k];
    };
    auto sees = [&](int r, int key) {
        return row_sees<MASK>(a, key, n, n - a.n_q + token[r] + 1, MASK == kSeeTree ? a.seen + ((int64_t)s * a.n_q + token[r]) * a.words : nullptr);
    };
    auto work = [&](int key0, int at) {  // the 32 keys from key0; `at`: their place in LDS behind the wave's first ones
        // LDS answers late: all of K's rows are requested together, and half of V's ahead of the terms.
        bf16x8 k[4][2];
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 2; ++i) k[c][i] = *(const bf16x8*)(wide_lds + k_at[c] + at + i * 4096);
        __builtin_amdgcn_sched_barrier(0);
        f32x4 x[2][2];  // by row tile, half tile
#pragma unroll
        for (int c = 0; c < 4; ++c)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int r = 0; r < 2; ++r)
                    x[r][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[c][i], q[r][c], c ? x[r][i] : f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0);
        s16x4 v[8][2];
        auto read_v = [&](int d) {
#pragma unroll
            for (int i = 0; i < 2; ++i) v[d][i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(wide_lds + v_at[d] + at + i * 4096));
        };
#pragma unroll
        for (int d = 0; d < W::kEarly; ++d) read_v(d);
        __builtin_amdgcn_sched_barrier(0);
        if (key0 + 32 > open) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = key0 + 16 * i + 4 * (lane >> 4) + e;
                        x[r][i][e] = sees(r, key) ? x[r][i][e] : -__builtin_inff();
                    }
            }
        }
        if (KEEP) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int row = row0 + r * kTileRows + (lane & 15);
                float* to = a.logits + (((int64_t)layer * a.h_kv + g) * a.rows + row) * a.logit_T + logit_at(a.cu_seq, s) + key0 + 4 * (lane >> 4);
                if (row < a.rows) {
                    *(f32x4*)to = x[r][0] * a.scale2;
                    *(f32x4*)(to + 16) = x[r][1] * a.scale2;
                }
            }
        }
        // The running maximum only has to keep the terms in range, so it is set by the first keys and looked at again when a row's sum
        // has grown past 2^24 (it cannot by its number of keys alone) or is not a number: then the tile's terms are formed anew.
        // (Finding the maximum of every tile took a sixth of the instructions.)
        bf16x8 p[2], rest[2];
        float sum[2];
        auto terms = [&]() {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const float mm = m[r] == -__builtin_inff() ? 0.0f : m[r];
                sum[r] = z[r];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(x[r][i][e], a.scale2, -mm));
                        sum[r] += y;
                        p[r][4 * i + e] = (__bf16)y;
                        if (kExact) rest[r][4 * i + e] = (__bf16)(y - (float)p[r][4 * i + e]);
                    }
            }
        };
        terms();
        if (__any(!(fmaxf(sum[0], sum[1]) <= kLargeSum) || fminf(m[0], m[1]) == -__builtin_inff())) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float to = fmaxf(max4(x[r][0]), max4(x[r][1])) * a.scale2;
                to = fmaxf(to, __shfl_xor(to, 16));
                to = fmaxf(m[r], fmaxf(to, __shfl_xor(to, 32)));
                int late = !(sum[r] <= kLargeSum) || m[r] == -__builtin_inff();
                late |= __shfl_xor(late, 16);
                late |= __shfl_xor(late, 32);
                if (!late) to = m[r];  // a row's bits do not depend on the others of its wave
                const float f = rescale(m[r], to);
                m[r] = to;
                z[r] *= f;
#pragma unroll
                for (int d = 0; d < 8; ++d) o[r][d] *= f;
            }
            terms();
        }
#pragma unroll
        for (int r = 0; r < 2; ++r) z[r] = sum[r];
#pragma unroll
        for (int d = 0; d < 8; ++d) {
            if (d + W::kEarly < 8) read_v(d + W::kEarly);
            __builtin_amdgcn_sched_barrier(0);
            const bf16x8 vt = __builtin_bit_cast(bf16x8, __builtin_shufflevector(v[d][0], v[d][1], 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int r = 0; r < 2; ++r) o[r][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, p[r], o[r][d], 0, 0, 0);
            if (kExact) {
#pragma unroll
                for (int r = 0; r < 2; ++r) o[r][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, rest[r], o[r][d], 0, 0, 0);
            }
        }
    };
    // Stages are dealt to the sequence's workgroups in turn; those with keys that not every row sees come last.
    const int stages = (n + W::kKeys - 1) / W::kKeys, n_mine = stages > mine ? (stages - mine - 1) / ns + 1 : 0;
    if (n_mine > 0) {
        for (int i0 = 0; i0 < n_mine; i0 += 2) {
#pragma unroll
            for (int buf = 0; buf < 2; ++buf) {
                const int i = i0 + buf;
                if (i >= n_mine) break;  // (uniform)
                deposit(ahead[buf % W::kAhead], i, buf);
                request(ahead[buf % W::kAhead], i + W::kAhead, n);  // (past the last stage: its last tile again, which costs less than a branch)
                lds_barrier();
#pragma unroll
                for (int t = 0; t < W::kTiles; ++t) {
                    const int key0 = (mine + i * ns) * W::kKeys + 32 * (W::kTiles * kw + t);
                    if (key0 < n) work(key0, buf * W::kBuffer + t * 8192);
                }
            }
        }
    }

#pragma unroll
    for (int r = 0; r < 2; ++r) {
        z[r] = sum_of_row(z[r]);
        was_cleared |= z[r] < __builtin_inff() && !all_finite(o[r]);
    }
    if (lane == 0) marked[wave] = 0;
    if (was_cleared) marked[wave] = 1;
    lds_barrier();
    if (__any(marked[lane % W::kWaves])) {
        f32x4 marks[2][8];
        auto tile = [&](int i) {
            const int key = (mine + i / W::kTiles * ns) * W::kKeys + 32 * (W::kTiles * kw + i % W::kTiles);
            return key < n ? key : -1;
        };
        mark_kinds<2>(marks, rows, n, lane, tile, sees, [&](int d) { return 16 * d + (lane & 15); });
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int d = 0; d < 8; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[r][d][e] = marks[r][d][e] == 0.0f ? o[r][d][e] : marks[r][d][e];
    }
    const int64_t part_row = part_at(a, layer, s, split, mine, g);
    const OutArgs outs(a);
    if (KW > 1) {  // the waves over other keys of the same rows
        float* sums = (float*)wide_lds;                                         // [kWaves - R][32][kOutStride]
        float2* stats = (float2*)(sums + (W::kWaves - R) * 32 * kOutStride);    // [kWaves - R][32]
        __syncthreads();
        if (kw > 0) {
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int at = (wave - R) * 32 + r * kTileRows + (lane & 15);
                if (lane < 16) stats[at] = make_float2(m[r], z[r]);
#pragma unroll
                for (int d = 0; d < 8; ++d) *(f32x4*)(sums + at * kOutStride + 4 * (lane >> 4) + 16 * d) = o[r][d];
            }
        }
        __syncthreads();
        if (kw > 0) return;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const float mine_m = m[r];
#pragma unroll
            for (int w = 0; w < KW - 1; ++w) m[r] = fmaxf(m[r], stats[(w * R + rw) * 32 + r * kTileRows + (lane & 15)].x);
            float f = rescale(mine_m, m[r]);
            z[r] *= f;
#pragma unroll
            for (int d = 0; d < 8; ++d) o[r][d] *= f;
#pragma unroll
            for (int w = 0; w < KW - 1; ++w) {
                const int at = (w * R + rw) * 32 + r * kTileRows + (lane & 15);
                const float2 mz = stats[at];
                f = rescale(mz.x, m[r]);
                z[r] += mz.y * f;
#pragma unroll
                for (int d = 0; d < 8; ++d) o[r][d] += *(const f32x4*)(sums + at * kOutStride + 16 * d + 4 * (lane >> 4)) * f;
            }
        }
    }
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int row = row0 + r * kTileRows + (lane & 15);
        if (row >= query_rows(a, s)) continue;
        if (lane < 16 && (ns > 1 || KEEP || kParts)) a.stats[part_row + row] = make_float2(m[r], z[r]);
#pragma unroll
        for (int d = 0; d < 8; ++d) {
            const int at = 16 * d + 4 * (lane >> 4);
            if (ns == 1 && !kParts) store_out(outs, layer, s, g, row, at, o[r][d], m[r], z[r]);
            else *(f32x4*)(a.part + (part_row + row) * kHeadDim + at) = o[r][d];
        }
    }
}

template <class Rows, int R, int MASK, bool KEEP>
__global__ __launch_bounds__(Wide<R>::kThreads, 2) void jq_attend_wide_kernel(AttendArgs a) {
    attend_many_rows<Rows, R, MASK, KEEP>(kernel_args<AttendArgs>(), (int)blockIdx.x, (int)blockIdx.y);
}

// ---- launches ----------------------------------------------------------------------------------------------------------------

template <class Rows, int RT, int MASK, bool KEEP, int WAVES>
static hipError_t launch_sweep(const AttendArgs& a, dim3 grid, hipStream_t st) {
    constexpr int sums = WAVES * RT * kTileRows * (kOutStride * 4 + 8);
    constexpr int most = sums + (KEEP ? kMostHeld + (WAVES - kAttendWaves) * 32 * kTileRows * RT * 4 : 0);  // (whole turns of all waves are held)
    const int lds = sums + (KEEP ? a.rows * a.hold_keys * 4 : 0);
    if (most > 65536) {
        static std::atomic<uint64_t> done{0};
        const hipError_t e = allow_dynamic_lds((const void*)jq_attend_kernel<Rows, RT, MASK, KEEP, WAVES>, most, done);
        if (e != hipSuccess) return e;
    }
    return launch_kernel(jq_attend_kernel<Rows, RT, MASK, KEEP, WAVES>, grid, dim3(64 * WAVES), lds, st, nullptr, -1, a);
}

template <class Rows, int R, int MASK, bool KEEP>
static hipError_t launch_wide(const AttendArgs& a, dim3 grid, hipStream_t st) {
    constexpr int lds = Wide<R>::kLds;
    if (lds > 65536) {
        static std::atomic<uint64_t> done{0};
        const hipError_t e = allow_dynamic_lds((const void*)jq_attend_wide_kernel<Rows, R, MASK, KEEP>, lds, done);
        if (e != hipSuccess) return e;
    }
    return launch_kernel(jq_attend_wide_kernel<Rows, R, MASK, KEEP>, grid, dim3(Wide<R>::kThreads), lds, st, nullptr, -1, a);
}

template <class Rows, int MASK, bool KEEP>
static hipError_t launch_rows(const AttendArgs& a, int row_tiles, int waves, dim3 grid, hipStream_t st) {
    constexpr int kWaves1 = Rows::waves(1, KEEP), kWaves2 = Rows::waves(2, KEEP);
    switch (row_tiles) {
        case 1:
            if (waves == kAttendWaves) return launch_sweep<Rows, 1, MASK, KEEP, kAttendWaves>(a, grid, st);
            return launch_sweep<Rows, 1, MASK, KEEP, kWaves1>(a, grid, st);
        case 2: return launch_sweep<Rows, 2, MASK, KEEP, kWaves2>(a, grid, st);
        case 4: return launch_wide<Rows, 2, MASK, KEEP>(a, grid, st);
        case 8: return launch_wide<Rows, 4, MASK, KEEP>(a, grid, st);
        default:  // more than 128 query rows: without weights
            if constexpr (KEEP) return hipErrorInvalidValue;
            else return launch_wide<Rows, 8, MASK, KEEP>(a, grid, st);
    }
}

// The sweep of a call over caches of one kind.  (One new token sees every live row, its own among them: no mask either way.)
template <class Rows>
hipError_t launch_sweeps(const AttendArgs& a, int row_tiles, int waves, bool causal, dim3 grid, hipStream_t st) {
    const bool weights = a.weights != nullptr;
    if (a.seen) return launch_rows<Rows, kSeeTree, false>(a, row_tiles, waves, grid, st);
    if (causal) return weights ? launch_rows<Rows, kSeeCausal, true>(a, row_tiles, waves, grid, st) : launch_rows<Rows, kSeeCausal, false>(a, row_tiles, waves, grid, st);
    return weights ? launch_rows<Rows, kSeeAll, true>(a, row_tiles, waves, grid, st) : launch_rows<Rows, kSeeAll, false>(a, row_tiles, waves, grid, st);
}

}  // namespace jq
