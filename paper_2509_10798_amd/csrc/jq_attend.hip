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
// paged caches of 29909 rows together 41, 64 over 32832 rows 53 (matrix and vector instructions, which take turns).
//
// Layout.  Both products are v_mfma_f32_16x16x32_bf16, of which lane l holds row (or column) l % 16 and the eight products'
// terms 8 * (l / 16) .. + 7 of either operand, and of the result column l % 16 and rows 4 * (l / 16) .. + 3.  Scores are
// formed transposed, keys x query rows, out of a 16-key tile and 16 query rows: lane l then holds query row l % 16 and keys
// 4 * (l / 16) + e of the tile, which is what the second product wants of its right operand when the terms of its 32-key sum are
// numbered 8 * (l / 16) + 4 * tile + e.  So the probabilities never move between lanes.  The left operand of the second product
// is V transposed: lane l loads 16 bytes (d = 8 * (l % 16) .. + 7) of the rows 4 * (l / 16) + e, a wave's load covers whole rows, and
// byte permutes inside the lane pair the rows up: no value passes through LDS, and no workgroup barrier stands in the sweep.
// out comes out transposed too: lane l holds d = 32 * (l / 16) .. + 31 of query row l % 16, in line with m and z.
#include <type_traits>

#include "jq_common.h"

namespace jq {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t au32x4 __attribute__((ext_vector_type(4)));

constexpr int kAttendWaves = 4;
constexpr int kAttendThreads = 64 * kAttendWaves;
constexpr int kTileRows = 16;   // query rows of one MFMA tile
constexpr int kOutStride = kHeadDim + 4;  // floats a row of partial output takes in LDS: rows of 128 would meet in the same banks
constexpr int kMostJoinRows = 8;  // query rows whose shares the last workgroup of a sequence joins
constexpr int kMostHeld = 65536;  // bytes of logits that a workgroup holds in LDS
constexpr float kSlack = 8.0f;  // a row's running maximum may lag this far (in powers of two) behind before its sums are rescaled
constexpr float kLargeSum = 16777216.0f;  // or, with many query rows, until a lane's share of the sum is this large

// Which cache rows a query row sees, apart from the live ones' end.
enum AttendMask { kSeeAll = 0, kSeeCausal, kSeeTree };

struct AttendArgs {
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
};

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
// tile(i): first key of the wave's tile i, -1 behind the last; row(key): its row of V; sees(r, key): of the lane's query row in
// row tile r; dim(d): the lane's dimension of the left operand in block d.
template <int RT, class Tile, class Row, class Sees, class Dim>
__device__ __forceinline__ void mark_kinds(f32x4 (&marks)[RT][8], const char* V, uint32_t stride, int n, int lane, Tile tile, Row row, Sees sees, Dim dim) {
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
        for (int d = 0; d < 8; ++d) marks[r][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    for (int i = 0, key0 = tile(0); key0 >= 0; key0 = tile(++i)) {
        const uint32_t row0 = row(key0);
        uint32_t at[8];  // the rows of the lane's eight keys; those behind the last are nobody's to see
        Exponents exponents;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            at[k] = (row0 + (uint32_t)min(16 * (k >> 2) + 4 * (lane >> 4) + (k & 3), n - 1 - key0)) * stride;
            exponents.add(*(const au32x4*)(V + (at[k] + (uint32_t)(lane & 15) * 16u)));
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
                const uint32_t x = *(const uint16_t*)(V + (at[k] + (uint32_t)dim(d) * 2u));
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
};

// Requests the tile whose first key is row `row0` of the base pointers; rows past `last` (counted from row0) are taken from `last`.
__device__ __forceinline__ void load_tile(KvTile& t, const char* K, const char* V, uint32_t row0, int last, uint32_t stride, int lane) {
    const uint32_t kb = (uint32_t)(lane >> 4) * 16u, vb = (uint32_t)(lane & 15) * 16u;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t row = row0 + (uint32_t)min(16 * i + (lane & 15), last);
#pragma unroll
        for (int c = 0; c < 4; ++c) t.k[i][c] = *(const au32x4*)(K + (row * stride + kb + 64u * c));
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t row = row0 + (uint32_t)min(16 * i + 4 * (lane >> 4) + e, last);
            t.v[i][e] = *(const au32x4*)(V + (row * stride + vb));
        }
}

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
template <int RT, bool MASKED, int MASK, bool KEEP>
__device__ __forceinline__ void tile_step(RowState<RT>& st, KvTile& t, const AttendArgs& a, int lane, int key0, int n, const int* row_limit,
                                          const uint32_t* const* row_seen, float* hold, bool* was_cleared) {
    if (MASKED) {
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
            for (int c = 0; c < 4; ++c) x = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, t.k[i][c]), st.q[r][c], x, 0, 0, 0);
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
            for (int e = 0; e < 4; ++e) {
                const float p = __builtin_amdgcn_exp2f(s[r][i][e] - m);
                st.z[r] += p;
                hi[r][4 * i + e] = (__bf16)p;
                lo[r][4 * i + e] = (__bf16)(p - (float)hi[r][4 * i + e]);
            }
    }
#pragma unroll
    for (int d = 0; d < 8; ++d) {
        au32x4 v;
        const uint32_t sel = d & 1 ? 0x07060302u : 0x05040100u;  // the upper or the lower halves of two registers
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) v[2 * i + e] = __builtin_amdgcn_perm(t.v[i][2 * e + 1][d >> 1], t.v[i][2 * e][d >> 1], sel);
        const bf16x8 vt = __builtin_bit_cast(bf16x8, v);
#pragma unroll
        for (int r = 0; r < RT; ++r) {
            st.o[r][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, hi[r], st.o[r][d], 0, 0, 0);
            st.o[r][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vt, lo[r], st.o[r][d], 0, 0, 0);
        }
    }
}

// Four dimensions of a query row's output out of its sums; a row that has seen nothing: zeros, and -inf for its log-sum-exp.
__device__ __forceinline__ void store_out(const AttendArgs& a, int layer, int s, int g, int row, int d, f32x4 o, float m, float z) {
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
    __device__ __forceinline__ int row(int k) const { return j0 + 2 * k * kAttendThreads; }
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
        for (; j0 < end; j0 += 2 * kPairs * kAttendThreads) {
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

template <int RT, int MASK, bool KEEP>
__global__ __launch_bounds__(kAttendThreads, RT == 1 ? 3 : 2) void jq_attend_kernel(AttendArgs a) {
    extern __shared__ __align__(16) float lds[];  // [waves][16 RT][kOutStride], then (m, z) [waves][16 RT]
    float2* lds_stats = (float2*)(lds + kAttendWaves * RT * kTileRows * kOutStride);
    // blockIdx.x: groups of query rows over the same keys eight apart, so that they meet in one XCD's L2
    const int per = 8 * a.row_groups;
    const int u = (int)blockIdx.x / per * 8 + ((int)blockIdx.x & 7), rg = ((int)blockIdx.x % per) >> 3;
    if (u >= a.units) return;
    const int layer = blockIdx.y, split = u / a.h_kv, g = u - split * a.h_kv;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int s = seq_of_split(a, split, lane);
    const int ns = a.cu_split[s + 1] - a.cu_split[s], mine = split - a.cu_split[s];
    const int row0 = rg * RT * kTileRows;

    // Tiles of 32 keys, dealt to the sequence's waves in turn, so that all of them sweep one moving window of the cache.
    const uint32_t stride = (uint32_t)a.h_kv * (kHeadDim * 2);
    const int64_t first_row = a.pm.block_table ? ((int64_t)layer * a.pm.n_pages) << a.pm.page_shift : (int64_t)layer * a.T + a.cu_seq[s];
    const char* K = a.K + first_row * stride + g * (kHeadDim * 2);
    const char* V = a.V + first_row * stride + g * (kHeadDim * 2);
    const_i32_ptr table = (const_i32_ptr)(a.pm.block_table ? a.pm.block_table + (int64_t)s * a.pm.max_pages : nullptr);
    const int shift = a.pm.page_shift, n_pages = a.pm.n_pages;
    const bool paged = a.pm.block_table != nullptr;
    auto tile_row = [&](int key) {  // a page holds whole tiles: page sizes are powers of two from 32 on
        if (!paged) return (uint32_t)key;
        return ((uint32_t)clamp_page(table[key >> shift], n_pages) << shift) + (uint32_t)(key & ((1 << shift) - 1));
    };
    // The first tile is requested before anything else is looked at, the live count too, which only decides whether it matters: rows
    // that are not live yet are the caller's as well, and masked.
    const int step = 32 * kAttendWaves * ns, cap = a.cu_seq[s + 1] - a.cu_seq[s];
    int key = 32 * (kAttendWaves * mine + wave);
    KvTile t;
    if (key < cap) load_tile(t, K, V, tile_row(key), cap - 1 - key, stride, lane);
    RowState<RT> st;
    int row_limit[RT];
    const uint32_t* row_seen[RT];
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        const int row = min(row0 + r * kTileRows + (lane & 15), a.rows - 1);  // rows past the last repeat it and are not stored
        const int i = row / a.group, h = g * a.group + row - i * a.group;
        const char* q = a.Q + ((((int64_t)layer * a.n_seq + s) * a.n_q + i) * a.h_q + h) * (kHeadDim * 2);
#pragma unroll
        for (int c = 0; c < 4; ++c) st.q[r][c] = __builtin_bit_cast(bf16x8, *(const au32x4*)(q + 64 * c + 16 * (lane >> 4)));
#pragma unroll
        for (int d = 0; d < 8; ++d) st.o[r][d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        st.m[r] = -__builtin_inff();
        st.z[r] = 0.0f;
        row_limit[r] = i + 1;  // (and the rows in front of the queries' own, below)
        row_seen[r] = MASK == kSeeTree ? a.seen + ((int64_t)s * a.n_q + i) * a.words : nullptr;
    }

    const int n = live_rows(a.lens, a.n_seq, layer, s, cap);
    // keys from `open` on are not seen by every row
    const int open = MASK == kSeeAll ? n : max(n - a.n_q + (MASK == kSeeCausal ? 1 : 0), 0);
#pragma unroll
    for (int r = 0; r < RT; ++r) row_limit[r] += n - a.n_q;
    // The sequence's count of finished workgroups starts at zero for this call: it holds the call's tag or is given it here.
    uint64_t* arrived = a.arrived + (((int64_t)layer * a.n_seq + s) * a.h_kv + g) * a.row_groups + rg;
    if (RT == 1 && a.tag && ns > 1 && threadIdx.x == 0) {
        uint64_t was = __hip_atomic_load(arrived, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if ((was ^ a.tag) >> 24) __hip_atomic_compare_exchange_strong(arrived, &was, a.tag, __ATOMIC_RELAXED, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    // With weights every row's logits stay in LDS until its sums are known, [rows][hold_keys], a wave's tiles four apart.  (Written
    // out as they are formed they kept reads from being under way: 32 sequences of 2048 rows 71.7 us a call, without weights 58.3.)
    float* held = (float*)(lds_stats + kAttendWaves * RT * kTileRows);
    float* hold = KEEP ? held + (lane & 15) * a.hold_keys + 32 * wave + 4 * (lane >> 4) : nullptr;
    bool was_cleared = false;
    while (key + 32 <= open) {
        tile_step<RT, false, MASK, KEEP>(st, t, a, lane, key, n, row_limit, row_seen, hold, &was_cleared);
        if (KEEP) hold += 32 * kAttendWaves;
        key += step;
        if (key < n) load_tile(t, K, V, tile_row(key), n - 1 - key, stride, lane);
    }
    while (key < n) {
        tile_step<RT, true, MASK, KEEP>(st, t, a, lane, key, n, row_limit, row_seen, hold, &was_cleared);
        if (KEEP) hold += 32 * kAttendWaves;
        key += step;
        if (key < n) load_tile(t, K, V, tile_row(key), n - 1 - key, stride, lane);
    }

    bool marked = was_cleared;
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        st.z[r] = sum_of_row(st.z[r]);
        marked |= st.z[r] < __builtin_inff() && !all_finite(st.o[r]);
    }
    if (__any(marked)) {
        f32x4 marks[RT][8];
        auto tile = [&](int i) { const int k = 32 * (kAttendWaves * mine + wave) + i * step; return k < n ? k : -1; };
        auto sees = [&](int r, int k) { return row_sees<MASK>(a, k, n, row_limit[r], row_seen[r]); };
        mark_kinds<RT>(marks, V, stride, n, lane, tile, tile_row, sees, [&](int d) { return 8 * (lane & 15) + d; });
#pragma unroll
        for (int r = 0; r < RT; ++r)
#pragma unroll
            for (int d = 0; d < 8; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) st.o[r][d][e] = marks[r][d][e] == 0.0f ? st.o[r][d][e] : marks[r][d][e];
    }

    // The four waves' sums, in wave order.
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        if (lane < 16) lds_stats[(wave * RT + r) * kTileRows + lane] = make_float2(st.m[r], st.z[r]);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        float m = -__builtin_inff();
#pragma unroll
        for (int w = 0; w < kAttendWaves; ++w) m = fmaxf(m, lds_stats[(w * RT + r) * kTileRows + (lane & 15)].x);
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
    const int64_t part_row = (((int64_t)layer * a.n_splits + split) * a.h_kv + g) * a.rows;
    const int rows_here = min(a.rows - row0, RT * kTileRows);
    for (int item = threadIdx.x; item < rows_here * 32; item += kAttendThreads) {
        const int r = item >> 5, d = (item & 31) * 4, row = row0 + r;
        float m = -__builtin_inff(), z = 0.0f;
#pragma unroll
        for (int w = 0; w < kAttendWaves; ++w) m = fmaxf(m, lds_stats[w * RT * kTileRows + r].x);
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < kAttendWaves; ++w) {
            const float2 mz = lds_stats[w * RT * kTileRows + r];
            z += mz.x == m ? mz.y : mz.y * __builtin_amdgcn_exp2f(mz.x - m);
            o += *(const f32x4*)(lds + (w * RT * kTileRows + r) * kOutStride + d);
        }
        if (ns == 1) {
            store_out(a, layer, s, g, row, d, o, m, z);
        } else {
            float* to = a.part + (part_row + row) * kHeadDim + d;
            put_pair(to, o[0], o[1]);
            put_pair(to + 2, o[2], o[3]);
        }
        if (d == 0 && (ns > 1 || KEEP)) put_pair((float*)(a.stats + part_row + row), m, z);
    }
    if (KEEP && ns == 1) {  // all of the sequence is here
        float* lse2 = lds;  // (the sums above have been read by the threads that wait here)
        __syncthreads();
        if ((int)threadIdx.x < a.rows) {
            float m = -__builtin_inff(), z = 0.0f;
#pragma unroll
            for (int w = 0; w < kAttendWaves; ++w) m = fmaxf(m, lds_stats[w * RT * kTileRows + threadIdx.x].x);
#pragma unroll
            for (int w = 0; w < kAttendWaves; ++w) {
                const float2 mz = lds_stats[w * RT * kTileRows + threadIdx.x];
                z += mz.x == m ? mz.y : mz.y * __builtin_amdgcn_exp2f(mz.x - m);
            }
            lse2[threadIdx.x] = z == 0.0f ? 0.0f : m + log2_of(z);
        }
        __syncthreads();
        float* w = a.weights + ((int64_t)layer * a.h_kv + g) * a.T + a.cu_seq[s];
        for (int j = threadIdx.x; j < n; j += kAttendThreads) {  // (one workgroup: row j of the cache is held at j)
            float sum = 0.0f;
            for (int r = 0; r < a.rows; ++r) sum += __builtin_amdgcn_exp2f(held[r * a.hold_keys + j] - lse2[r]);
            w[j] += sum;
        }
        return;
    }
    if (KEEP) {  // the whole share's logits at once, to where the workgroup that weighs finds them
        const int64_t to = ((int64_t)layer * a.h_kv + g) * a.rows * a.logit_T + logit_at(a.cu_seq, s);
        const int pairs = a.hold_keys / 2;
        for (int item = threadIdx.x; item < a.rows * pairs; item += kAttendThreads) {
            const int r = item / pairs, j = (item - r * pairs) * 2, tile = j >> 5;
            const int at = ((tile >> 2) * ns + mine) * 32 * kAttendWaves + 32 * (tile & 3) + (j & 31);
            if (at < ((n + 31) & ~31)) put_pair(a.logits + to + r * a.logit_T + at, held[r * a.hold_keys + j], held[r * a.hold_keys + j + 1]);
        }
    }
    if (RT > 1 || !a.tag || ns == 1) return;

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
    static_assert(kMostJoinRows * 32 <= kAttendThreads, "a thread or more for every four sums");
    const int items = rows_here * 32, part = (int)threadIdx.x / items, item = (int)threadIdx.x - part * items;
    int parts = 1;
    while (2 * parts * items <= kAttendThreads && parts < 8) parts *= 2;
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
    Weigher weigher(a, layer, s, g, 0, n);
    if (KEEP) weigher.request(0);
    // Factors of all shares' sums, [rows_here][ns], and the rows' (m, z).
    float* factor = lds;
    float* sums = factor + (rows_here * ns + 3) / 4 * 4;  // [parts][items] outputs of four, at multiples of sixteen bytes
    float* lse2 = (float*)(lds_stats + rows_here);
    __syncthreads();
    for (int r = wave; r < rows_here; r += kAttendWaves) {  // a wave a row, a lane a share (there are 20 at most)
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
    if (part == 0) store_out(a, layer, s, g, row0 + r, d, o, lds_stats[r].x, lds_stats[r].y);
    if (KEEP) weigher.add(lse2, true);
}

// Many query rows (more than 32 a KV head).  A wave still holds 32 of them, but the eight waves of a workgroup share the keys: R waves
// over all rows of a group times KW over keys of their own.  K and V go through LDS, where every wave reads all of its keys' rows:
// requested into registers stages ahead, written to one of two buffers, one barrier a stage.  (Every wave reading K and V for itself
// took 117 us for 128 rows behind four prompts, 58 this way.)
// K's rows are read sixteen lanes a row of 256 bytes, piece p of row k at p ^ (k & 15), so that eight lanes' pieces meet in eight
// different bank groups; V is read transposed (ds_read_b64_tr_b16: a lane receives four keys' values of one dimension out of four
// rows of sixteen), piece p of row k at p ^ 2 (k & 7) for the same reason (no bank conflicts are counted).
// What bounds it: with 128 rows a group memory, and the 20 us that two launches of this size cost whatever they do; with 256 the
// instructions of a tile of 32 keys and 32 rows, 512 cycles of the matrix cores and some 420 of the vector ALU, which add up
// also across the two waves of a SIMD.  Tried without gain: four stages ahead, two tiles' terms together, more of V's reads early,
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
    // 39.3 / 40.4, 128 behind four prompts 58.8 / 65.2, 100 over eight caches 41.5 / 45.3, 256 over 32832 56 / 68: two while they cost 3 percent.
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

template <int R, int MASK, bool KEEP>
__global__ __launch_bounds__(Wide<R>::kThreads, 2) void jq_attend_wide_kernel(AttendArgs a) {
    using W = Wide<R>;
    constexpr int KW = W::KW;
    extern __shared__ __align__(16) char wide_lds[];
    uint8_t* marked = (uint8_t*)wide_lds + W::kFlags;  // [kWaves]: the wave has cleared values of V, or has sums that are not finite
    bool was_cleared = false;
    const int per = 8 * a.row_groups;
    const int u = (int)blockIdx.x / per * 8 + ((int)blockIdx.x & 7), rg = ((int)blockIdx.x % per) >> 3;
    if (u >= a.units) return;
    const int layer = blockIdx.y, split = u / a.h_kv, g = u - split * a.h_kv;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int s = seq_of_split(a, split, lane);
    const int ns = a.cu_split[s + 1] - a.cu_split[s], mine = split - a.cu_split[s];
    const int cap = a.cu_seq[s + 1] - a.cu_seq[s];
    const int rw = wave % R, kw = wave / R;
    const int row0 = rg * W::kRows + 32 * rw;

    const uint32_t stride = (uint32_t)a.h_kv * (kHeadDim * 2);
    const int64_t first_row = a.pm.block_table ? ((int64_t)layer * a.pm.n_pages) << a.pm.page_shift : (int64_t)layer * a.T + a.cu_seq[s];
    const_i32_ptr table = (const_i32_ptr)(a.pm.block_table ? a.pm.block_table + (int64_t)s * a.pm.max_pages : nullptr);
    const int shift = a.pm.page_shift, n_pages = a.pm.n_pages;
    const bool paged = a.pm.block_table != nullptr;

    // This wave's requests of a stage: kRequests times four rows of K or of V, all in one tile of 32 keys.
    constexpr int kPerTile = 8 / W::kRequests;  // waves that share the requests of a tile
    const bool is_v = wave >= W::kWaves / 2;
    const int in_half = wave % (W::kWaves / 2), my_tile = in_half / kPerTile;
    const int my_row = in_half % kPerTile * W::kRequests * 4 + (lane >> 4);  // the first request's row within the tile, 4 apart
    const char* base = (is_v ? a.V : a.K) + first_row * stride + g * (kHeadDim * 2) + (lane & 15) * 16;
    // where the requests go: the pieces of rows 4 apart are exchanged by amounts that differ
    int to_lds[W::kRequests];
#pragma unroll
    for (int i = 0; i < W::kRequests; ++i) {
        const int row = my_row + 4 * i, piece = is_v ? (lane & 15) ^ 2 * (row & 7) : (lane & 15) ^ (row & 15);
        to_lds[i] = (is_v ? W::kKeys * 256 : 0) + (my_tile * 32 + row) * 256 + piece * 16;
    }
    auto tile_row = [&](int key) {
        return !paged ? (uint32_t)key : ((uint32_t)clamp_page(table[key >> shift], n_pages) << shift) + (uint32_t)(key & ((1 << shift) - 1));
    };
    auto request = [&](au32x4* to, int stage, int rows) {  // `rows`: those that may be read
        int key = (mine + stage * ns) * W::kKeys + 32 * my_tile;
        key = min(key, (rows - 1) & ~31);  // (a stage may reach past the last tile)
        const int last = rows - 1 - key;
        const uint32_t row0 = tile_row(key);
#pragma unroll
        for (int i = 0; i < W::kRequests; ++i) to[i] = *(const au32x4*)(base + (row0 + (uint32_t)min(my_row + 4 * i, last)) * stride);
    };
    // The first stages are requested before anything else is looked at, the live count too: rows that are not live yet are the
    // caller's as well, and masked.  (What follows, mostly instructions that the cache does not hold yet, takes some 3 us.)
    au32x4 ahead[W::kAhead][W::kRequests];
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
        const int row = min(row0 + r * kTileRows + (lane & 15), a.rows - 1);
        const int i = row / a.group, h = g * a.group + row - i * a.group;
        const char* from = a.Q + ((((int64_t)layer * a.n_seq + s) * a.n_q + i) * a.h_q + h) * (kHeadDim * 2);
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
    auto deposit = [&](au32x4* from, int stage, int buf) {
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
                        if (W::kExact) rest[r][4 * i + e] = (__bf16)(y - (float)p[r][4 * i + e]);
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
            if (W::kExact) {
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
        mark_kinds<2>(marks, a.V + first_row * stride + g * (kHeadDim * 2), stride, n, lane, tile, tile_row, sees, [&](int d) { return 16 * d + (lane & 15); });
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int d = 0; d < 8; ++d)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[r][d][e] = marks[r][d][e] == 0.0f ? o[r][d][e] : marks[r][d][e];
    }
    const int64_t part_row = (((int64_t)layer * a.n_splits + split) * a.h_kv + g) * a.rows;
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
        if (row >= a.rows) continue;
        if (lane < 16 && (ns > 1 || KEEP)) a.stats[part_row + row] = make_float2(m[r], z[r]);
#pragma unroll
        for (int d = 0; d < 8; ++d) {
            const int at = 16 * d + 4 * (lane >> 4);
            if (ns == 1) store_out(a, layer, s, g, row, at, o[r][d], m[r], z[r]);
            else *(f32x4*)(a.part + (part_row + row) * kHeadDim + at) = o[r][d];
        }
    }
}

// A row's statistics over the ns shares of its sequence, a lane a share: (m, z) in every lane, and the lane's own factor (of share
// `lane`; those of further shares are formed where they are needed).
__device__ __forceinline__ float2 merge_stats(const float2* from, int64_t step, int ns, int lane, float* factor) {
    const float2 own = lane < ns ? from[lane * step] : make_float2(-__builtin_inff(), 0.0f);
    float m = own.x;
    for (int i = lane + 64; i < ns; i += 64) m = fmaxf(m, from[i * step].x);
#pragma unroll
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    *factor = rescale(own.x, m);
    float z = own.y * *factor;
    for (int i = lane + 64; i < ns; i += 64) {
        const float2 mz = from[i * step];
        z += mz.x == m ? mz.y : mz.y * __builtin_amdgcn_exp2f(mz.x - m);
    }
#pragma unroll
    for (int d = 32; d; d >>= 1) z += __shfl_xor(z, d);
    return make_float2(m, z);
}

// Calls whose last workgroups would have too much to join or weigh: a second launch does it.  The first `joins` workgroups of a
// layer take four (sequence, head, query row) each, a wave a row; the others 1024 rows of the cache of a (sequence, head).
constexpr int kWeighKeys = 1024;
__global__ __launch_bounds__(kAttendThreads) void jq_attend_finish_kernel(AttendArgs a, int joins, int blocks_per_seq) {
    __shared__ float lse2[kMaxWeighRows];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), layer = blockIdx.y;
    const int64_t step = (int64_t)a.h_kv * a.rows;
    if ((int)blockIdx.x < joins) {
        const int item = (int)blockIdx.x * kAttendWaves + wave;
        if (item >= a.n_seq * a.h_kv * a.rows) return;
        const int unit = item / a.rows, row = item - unit * a.rows, s = unit / a.h_kv, g = unit - s * a.h_kv;
        const int first = a.cu_split[s], ns = a.cu_split[s + 1] - first;
        if (ns == 1) return;
        const int64_t at = (((int64_t)layer * a.n_splits + first) * a.h_kv + g) * a.rows + row;
        // two shares at a time, 16 bytes a lane; the first sixteen are requested ahead of the statistics
        const int half = lane >> 5, d = (lane & 31) * 4;
        const float* part = a.part + at * kHeadDim + d;
        constexpr int kFirst = 8;
        f32x4 x[kFirst];
#pragma unroll
        for (int k = 0; k < kFirst; ++k) x[k] = *(const f32x4*)(part + min(half + 2 * k, ns - 1) * step * kHeadDim);
        float factor;
        const float2 mz = merge_stats(a.stats + at, step, ns, lane, &factor);
        f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int k = 0; k < kFirst; ++k) {
            const float f = __shfl(factor, half + 2 * k);
            const bool there = half + 2 * k < ns;  // (nothing times 0: a sum may be infinite)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += there ? x[k][e] * f : 0.0f;
        }
        for (int i0 = 2 * kFirst; i0 < ns; i0 += 2 * kFirst) {
#pragma unroll
            for (int k = 0; k < kFirst; ++k) x[k] = *(const f32x4*)(part + min(i0 + half + 2 * k, ns - 1) * step * kHeadDim);
#pragma unroll
            for (int k = 0; k < kFirst; ++k) {
                const int i = i0 + half + 2 * k;
                float f = __shfl(factor, i & 63);
                if (i >= 64) {
                    const float mi = a.stats[at + min(i, ns - 1) * step].x;
                    f = rescale(mi, mz.x);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] += i < ns ? x[k][e] * f : 0.0f;
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], 32);
        if (lane < 32) store_out(a, layer, s, g, row, d, o, mz.x, mz.y);
        return;
    }
    const int b = ((int)blockIdx.x - joins) % blocks_per_seq, unit = ((int)blockIdx.x - joins) / blocks_per_seq;
    const int s = unit / a.h_kv, g = unit - s * a.h_kv;
    const int n = live_rows(a.lens, a.n_seq, layer, s, a.cu_seq[s + 1] - a.cu_seq[s]);
    if (b * kWeighKeys >= n) return;
    const int first = a.cu_split[s], ns = a.cu_split[s + 1] - first;
    if (ns == 1 && a.hold_keys) return;  // weighed by the workgroup that swept it
    const int64_t at = (((int64_t)layer * a.n_splits + first) * a.h_kv + g) * a.rows;
    for (int r = wave; r < a.rows; r += kAttendWaves) {
        float factor;
        const float2 mz = merge_stats(a.stats + at + r, step, ns, lane, &factor);
        if (lane == 0) lse2[r] = mz.y == 0.0f ? 0.0f : mz.x + log2_of(mz.y);  // nothing seen: all its logits are -inf
    }
    __syncthreads();
    Weigher(a, layer, s, g, b * kWeighKeys, min((b + 1) * kWeighKeys, n)).add(lse2, false);
}

// ---- host ------------------------------------------------------------------------------------------------------------------

// How many workgroups share each sequence.  Asked for more than one workgroup per CU, memory answers no faster, and there are more
// sums to join (us a call, workgroups 256 / 512 / 768): one token over 131072 rows 97 / 100 / 108, 32 tokens behind four prompts of
// 52296 rows together 59 / 70 / 80, a tree of 64 over 32832 rows 56 / 71 / 92.  So the smallest share is looked for that makes
// no more workgroups than there are CUs -- not a share of the rows rounded up for every sequence, which makes 288 for eight ragged
// ones (63 us against 47).  Where sequences and heads alone are more than that, whole sequences leave CUs idle behind the longest, and
// smaller shares in two to four rounds of the chip may be ahead; a round costs its share and a start, which is dearer where sums of
// many query rows have to be joined afterwards.  In rows of the cache, fitted to (whole sequences / as chosen) one token, 40 x 4099 rows
// 158 / 133 us, 36 x 2000 78 / 65, 64 ragged sequences of 80 to 7000 203 / 128; trees of 20 over those 257 / 161, 12 x 40 x 4099 189 /
// 177, and as they are 25 x 40 x 2099 103 (125 in smaller shares), 64 x 40 x 1099 96 (133).
constexpr int kChip = 256, kRounds = 4;
constexpr int kStart = 320, kWideStart = 1500;
// What a sequence's last workgroup joins, and weighs, instead of a second launch.  Its time grows with the shares, whose statistics and
// sums it waits for, and with the rows times them, while the second launch costs some 1.7 us whatever there is (2 with weights).  Us a call
// of 8 KV heads, joined / in a second launch, by shares of 128 rows of the cache:
//   shares:          8            12           16           20           24           32
//    1 query row  10.0 / 11.6  10.5 / 11.7  10.9 / 11.6  11.5 / 11.6  12.1 / 11.3  14.3 / 11.4
//    4            10.0 / 11.7  10.4 / 11.7  10.8 / 11.6  12.2 / 11.6  12.8 / 11.3  15.0 / 11.4
//    8            10.5 / 11.6  11.8 / 11.6  12.3 / 11.7  13.7 / 11.5  14.2 / 11.3  17.3 / 11.5
//   16, 2 shares 12.4 / 11.5; 32, 2 shares 18.9 / 11.7
//   1, weights    11.4 / 13.2  11.9 / 13.3  12.4 / 13.3               14.6 / 13.2
//   4             11.7 / 13.3  12.2 / 13.3  12.6 / 13.3               16.1 / 13.1
//   8, 4 shares   13.0 / 13.3; 8 13.4 / 13.3; 12 14.7 / 13.4; 16, 2 shares 16.7 / 15.4
constexpr int kMostJoined = 20;          // shares (a lane each in the join)
constexpr int kMostSums = 64;            // shares times query rows
constexpr int64_t kMostWeighed = 8192;   // logits of a (sequence, head)
static void plan_splits(const Plan& p, bool weights, AttendPlan* ap) {
    const int row_tiles = (p.rows + kTileRows - 1) / kTileRows;
    ap->row_tiles = row_tiles <= 1 ? 1 : row_tiles <= 2 ? 2 : row_tiles <= 4 ? 4 : row_tiles <= 8 ? 8 : 16;
    ap->row_groups = (row_tiles + ap->row_tiles - 1) / ap->row_tiles;
    // Shares are counted in what a workgroup takes at a time; workgroups left over go to the sequences with the largest.
    const int64_t heads = (int64_t)p.n_layers * p.h_kv * ap->row_groups, unit = ap->row_tiles > 4 ? 64 : 128;
    int32_t units[JQ_MAX_SEQ];
    for (int s = 0; s < p.n_seq; ++s) units[s] = (int32_t)(((int64_t)p.tab.cu_seq[s + 1] - p.tab.cu_seq[s] + unit - 1) / unit);
    auto workgroups = [&](int64_t share) {
        int64_t n = 0;
        for (int s = 0; s < p.n_seq; ++s) n += ((uint32_t)units[s] + (uint32_t)share - 1) / (uint32_t)share;
        return n;
    };
    int64_t most = (p.T + unit - 1) / unit;
    if (weights && row_tiles <= 2) most = std::min(most, (int64_t)kMostHeld / (p.rows * 4) / unit);  // its logits have to fit the LDS that is theirs
    int64_t share = most, best = INT64_MAX, slots = 0;
    const int64_t start = ap->row_tiles > 2 ? kWideStart : kStart;
    for (int rounds = 1; rounds <= (p.n_seq * heads > kChip ? kRounds : 1); ++rounds) {
        int64_t lo = 1, hi = most;
        while (lo < hi) {
            const int64_t mid = (lo + hi) / 2;
            if (workgroups(mid) * heads <= rounds * kChip) hi = mid; else lo = mid + 1;
        }
        const int64_t n = workgroups(lo) * heads, cost = (n + kChip - 1) / kChip * (lo * unit + start);
        if (cost < best) { best = cost; share = lo; slots = rounds * kChip / heads; }
    }
    int32_t ns[JQ_MAX_SEQ];
    for (int s = 0; s < p.n_seq; ++s) ns[s] = (int32_t)((units[s] + share - 1) / share);
    if (p.n_seq > 1)
        for (int64_t left = slots - workgroups(share); left > 0; --left) {
            int at = 0;
            for (int s = 1; s < p.n_seq; ++s)
                if ((int64_t)units[s] * ns[at] > (int64_t)units[at] * ns[s]) at = s;
            if (units[at] <= ns[at]) break;
            ++ns[at];
        }
    ap->cu_split[0] = 0;
    int64_t most_L = 0, tiles = 0;
    int32_t most_ns = 0;
    for (int s = 0; s < p.n_seq; ++s) {
        const int64_t L = p.tab.cu_seq[s + 1] - p.tab.cu_seq[s];
        ap->cu_split[s + 1] = ap->cu_split[s] + ns[s];
        most_L = std::max(most_L, L);
        most_ns = std::max(most_ns, ns[s]);
        tiles = std::max(tiles, ((L + 31) / 32 + 4 * ns[s] - 1) / (4 * ns[s]));  // of 32 keys, a wave
    }
    ap->hold_keys = weights && row_tiles <= 2 ? (int32_t)(tiles * 32 * kAttendWaves) : 0;
    // (without shares there is nothing to join, and the weights are the sweep's)
    ap->one_launch = row_tiles <= 2 && (most_ns == 1 || (p.rows <= kMostJoinRows && most_ns <= kMostJoined && most_ns * p.rows <= kMostSums &&
                                                         (!weights || most_L * p.rows <= kMostWeighed)));
}

// 40 bits that no other call of the process has, above 24 of zeros; never 0.
static uint64_t next_tag() {
    static std::atomic<uint64_t> calls{0};
    uint64_t x = (calls.fetch_add(1, std::memory_order_relaxed) + 1) * 0x9E3779B97F4A7C15ull;  // (odd: 64-bit numbers stay distinct)
    x &= 0xFFFFFFFFFFull;
    return (x ? x : 1) << 24;
}

void plan_attend(const Plan& p, bool weights, AttendPlan* ap) {
    plan_splits(p, weights, ap);
    const size_t parts = (size_t)p.n_layers * ap->cu_split[p.n_seq] * p.h_kv * p.rows;
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    ap->logit_T = 32 * (p.T / 32 + p.n_seq);
    ap->off_arrived = 0;
    ap->off_stats = up((size_t)p.n_layers * p.n_seq * p.h_kv * ap->row_groups * sizeof(uint64_t));
    ap->off_part = ap->off_stats + up(parts * sizeof(float2));
    ap->off_logits = ap->off_part + up(parts * kHeadDim * sizeof(float));
    ap->ws_bytes = ap->off_logits + (weights ? up((size_t)p.n_layers * p.h_kv * p.rows * ap->logit_T * sizeof(float)) : 0);
}

// Workgroups of a layer's sweep, and of the launch behind it: those that join, blocks of weights a (sequence, head).
static int64_t sweep_groups(const Plan& p, const AttendPlan& ap) { return ((int64_t)ap.cu_split[p.n_seq] * p.h_kv + 7) / 8 * 8 * ap.row_groups; }
struct Finish {
    int64_t joins, blocks, groups;
};
static Finish finish_groups(const Plan& p, const AttendPlan& ap, bool weights) {
    int32_t most = 0;
    for (int s = 0; s < p.n_seq; ++s) most = std::max(most, p.tab.cu_seq[s + 1] - p.tab.cu_seq[s]);
    const int64_t heads = (int64_t)p.n_seq * p.h_kv;
    Finish f;
    f.joins = ap.cu_split[p.n_seq] > p.n_seq ? (heads * p.rows + kAttendWaves - 1) / kAttendWaves : 0;
    f.blocks = (most + kWeighKeys - 1) / kWeighKeys;
    f.groups = ap.one_launch ? 0 : f.joins + (weights ? f.blocks * heads : 0);
    return f;
}
bool attend_fits(const Plan& p, const AttendPlan& ap, bool weights) {
    return sweep_groups(p, ap) * (ap.row_tiles > 2 ? 512 : kAttendThreads) <= UINT32_MAX && finish_groups(p, ap, weights).groups * kAttendThreads <= UINT32_MAX;
}

template <int RT, int MASK, bool KEEP>
static hipError_t launch_sweep(const AttendArgs& a, dim3 grid, hipStream_t st) {
    constexpr int most = kAttendWaves * RT * kTileRows * (kOutStride * 4 + 8) + (KEEP ? kMostHeld : 0);
    const int lds = kAttendWaves * RT * kTileRows * (kOutStride * 4 + 8) + (KEEP ? a.rows * a.hold_keys * 4 : 0);
    if (most > 65536) {
        static std::atomic<uint64_t> done{0};
        const hipError_t e = allow_dynamic_lds((const void*)jq_attend_kernel<RT, MASK, KEEP>, most, done);
        if (e != hipSuccess) return e;
    }
    return launch_kernel(jq_attend_kernel<RT, MASK, KEEP>, grid, dim3(kAttendThreads), lds, st, nullptr, -1, a);
}

template <int R, int MASK, bool KEEP>
static hipError_t launch_wide(const AttendArgs& a, dim3 grid, hipStream_t st) {
    constexpr int lds = Wide<R>::kLds;
    if (lds > 65536) {
        static std::atomic<uint64_t> done{0};
        const hipError_t e = allow_dynamic_lds((const void*)jq_attend_wide_kernel<R, MASK, KEEP>, lds, done);
        if (e != hipSuccess) return e;
    }
    return launch_kernel(jq_attend_wide_kernel<R, MASK, KEEP>, grid, dim3(Wide<R>::kThreads), lds, st, nullptr, -1, a);
}

template <int MASK, bool KEEP>
static hipError_t launch_rows(const AttendArgs& a, int row_tiles, dim3 grid, hipStream_t st) {
    switch (row_tiles) {
        case 1: return launch_sweep<1, MASK, KEEP>(a, grid, st);
        case 2: return launch_sweep<2, MASK, KEEP>(a, grid, st);
        case 4: return launch_wide<2, MASK, KEEP>(a, grid, st);
        case 8: return launch_wide<4, MASK, KEEP>(a, grid, st);
        default:  // more than 128 query rows: without weights
            if constexpr (KEEP) return hipErrorInvalidValue;
            else return launch_wide<8, MASK, KEEP>(a, grid, st);
    }
}

hipError_t launch_attend(const Plan& p, const AttendPlan& ap, const int32_t* lens, const uint32_t* seen, const void* Q, const void* K, const void* V,
                         void* out, float* lse, float* weights, char* ws, hipStream_t st) {
    AttendArgs a{};
    a.Q = (const char*)Q; a.K = (const char*)K; a.V = (const char*)V;
    a.lens = lens; a.seen = seen; a.out = (uint16_t*)out; a.lse = lse; a.weights = weights;
    a.stats = (float2*)(ws + ap.off_stats);
    a.part = (float*)(ws + ap.off_part);
    a.logits = (float*)(ws + ap.off_logits);
    a.n_layers = p.n_layers; a.n_seq = p.n_seq; a.n_q = p.n_q; a.h_q = p.h_q; a.h_kv = p.h_kv; a.group = p.group; a.rows = p.rows;
    a.row_groups = ap.row_groups;
    a.n_splits = ap.cu_split[p.n_seq];
    a.units = a.n_splits * p.h_kv;
    a.words = (p.n_q + 31) / 32;
    a.hold_keys = ap.hold_keys;
    a.scale2 = (float)(p.scale * 1.4426950408889634);
    a.T = p.T; a.logit_T = ap.logit_T;
    a.arrived = (uint64_t*)(ws + ap.off_arrived);
    a.tag = ap.one_launch ? next_tag() : 0;
    a.pm = p.page_map();
    for (int s = 0; s <= p.n_seq; ++s) { a.cu_seq[s] = p.tab.cu_seq[s]; a.cu_split[s] = ap.cu_split[s]; }
    // one new token sees every live row, its own among them: no mask either way
    const dim3 grid((unsigned)sweep_groups(p, ap), (unsigned)p.n_layers);
    hipError_t e;
    if (seen) e = launch_rows<kSeeTree, false>(a, ap.row_tiles, grid, st);
    else if (p.window && p.n_q > 1) e = weights ? launch_rows<kSeeCausal, true>(a, ap.row_tiles, grid, st) : launch_rows<kSeeCausal, false>(a, ap.row_tiles, grid, st);
    else e = weights ? launch_rows<kSeeAll, true>(a, ap.row_tiles, grid, st) : launch_rows<kSeeAll, false>(a, ap.row_tiles, grid, st);
    if (e != hipSuccess) return e;
    const Finish f = finish_groups(p, ap, weights != nullptr);
    if (f.groups == 0) return e;
    return launch_kernel(jq_attend_finish_kernel, dim3((unsigned)f.groups, (unsigned)p.n_layers), dim3(kAttendThreads), 0, st, nullptr, -1, a, (int)f.joins,
                         (int)f.blocks);
}

}  // namespace jq
