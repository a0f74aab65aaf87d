// Attention of a sequence's newest tokens over its (pruned) cache, the step that decoding repeats between two evictions
// (paper Section 4.3: decoding continues on the pruned cache):
//
//   s[r,j] = scale * q[r] . k[j]      r: the n_q * G query rows of one KV head, j: the live cache rows that r may see
//   p[r,j] = exp(s[r,j] - lse[r]),    lse[r] = ln sum_j exp s[r,j],    out[r] = sum_j p[r,j] v[j]
//   weights[j] += sum_r p[r,j]        (where the caller accumulates the attention every cached row receives)
//
// K and V are read once, 512 bytes a (row, KV head); the few query rows stay in registers.  One pass with a running maximum m
// and sum z per query row; workgroups that share a sequence leave (m, z, unnormalised out) which a second launch joins.
//
// Layout.  Both products are v_mfma_f32_16x16x32_bf16, of which lane l holds row (or column) l % 16 and the eight products'
// terms 8 * (l / 16) .. + 7 of either operand, and of the result column l % 16 and rows 4 * (l / 16) .. + 3.  Scores are
// formed transposed, keys x query rows, out of a 16-key tile and 16 query rows: lane l then holds query row l % 16 and keys
// 4 * (l / 16) + e of the tile, which is what the second product wants of its right operand when the terms of its 32-key sum are
// numbered 8 * (l / 16) + 4 * tile + e.  So the probabilities never move between lanes.  The left operand of the second product
// is V transposed: lane l loads 16 bytes (d = 8 * (l % 16) .. + 7) of the rows 4 * (l / 16) + e, a wave's load covers whole rows, and
// byte permutes inside the lane pair the rows up: no value passes through LDS, and no workgroup barrier stands in the sweep.
// out comes out transposed too: lane l holds d = 32 * (l / 16) .. + 31 of query row l % 16, in line with m and z.
#include "jq_common.h"

namespace jq {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t au32x4 __attribute__((ext_vector_type(4)));

constexpr int kAttendWaves = 4;
constexpr int kAttendThreads = 64 * kAttendWaves;
constexpr int kTileRows = 16;   // query rows of one MFMA tile
constexpr int kOutStride = kHeadDim + 4;  // floats a row of partial output takes in LDS: rows of 128 would meet in the same banks
constexpr float kSlack = 8.0f;  // a row's running maximum may lag this far (in powers of two) behind before its sums are rescaled

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
    float scale2;          // scale * log2(e)
    int64_t T, logit_T;
    PageMap pm;
    int32_t cu_seq[JQ_MAX_SEQ + 1];
    int32_t cu_split[JQ_MAX_SEQ + 1];
};

__device__ __forceinline__ int32_t live_rows(const int32_t* lens, int n_seq, int layer, int s, int cap) {
    return lens ? min(max(lens[(int64_t)layer * n_seq + s], 0), cap) : cap;
}

// First entry of a sequence's logits in a row of logit_T: whole tiles of 32 keys have room in front of the next sequence's.
__device__ __forceinline__ int64_t logit_at(const int32_t* cu_seq, int s) { return 32 * ((int64_t)(cu_seq[s] / 32) + s); }

__device__ __forceinline__ float max4(f32x4 x) { return fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])); }

__device__ __forceinline__ bool finite_pair(uint32_t x) {  // neither bf16 of the pair is infinite or NaN
    return (x & 0x7F80u) != 0x7F80u && (x & 0x7F800000u) != 0x7F800000u;
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

// One tile of 32 keys.  MASKED: some row may not see some key of it, or the tile reaches past the live rows.
template <int RT, bool MASKED, int MASK, bool KEEP>
__device__ __forceinline__ void tile_step(RowState<RT>& st, KvTile& t, const AttendArgs& a, int lane, int key0, int n, const int* row_limit,
                                          const uint32_t* const* row_seen, float* const* row_logits) {
    uint32_t bad[2][4];  // keys whose V is not finite, by the lanes that hold their 16 pieces
    if (MASKED) {
        // What a query row does not see must not reach it, not even times zero: such values count as zeros, and every row
        // that does see the key gets a NaN for its score instead.
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                bool ok = true;
#pragma unroll
                for (int w = 0; w < 4; ++w) ok = ok && finite_pair(t.v[i][e][w]);
                const uint64_t votes = __ballot(!ok);
                bad[i][e] = (uint32_t)(votes >> (16 * (lane >> 4))) & 0xFFFFu;
                if (bad[i][e])
                    t.v[i][e] = au32x4{0u, 0u, 0u, 0u};
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
                    bool see = key < n;
                    if (MASK == kSeeCausal) see = key < row_limit[r];
                    if (MASK == kSeeTree) {
                        const int j = key - (n - a.n_q);
                        if (see && j >= 0) see = (row_seen[r][j >> 5] >> (j & 31)) & 1u;
                    }
                    s[r][i][e] = see ? (bad[i][e] ? __builtin_nanf("") : s[r][i][e]) : -__builtin_inff();
                }
    }
    if (KEEP) {
#pragma unroll
        for (int r = 0; r < RT; ++r)
            if (row_logits[r]) {
#pragma unroll
                for (int i = 0; i < 2; ++i) *(f32x4*)(row_logits[r] + key0 + 16 * i + 4 * (lane >> 4)) = s[r][i];
            }
    }
    // Running maximum: raised, and the sums rescaled, only when a score passes it by more than kSlack; terms stay below 2^8.
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        float top = fmaxf(max4(s[r][0]), max4(s[r][1]));
        if (__any(top > st.m[r] + kSlack)) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float to = fmaxf(st.m[r], top);
            const float f = st.m[r] == to ? 1.0f : __builtin_amdgcn_exp2f(st.m[r] - to);  // (-inf stays -inf: no 0 * inf)
            st.m[r] = to;
            st.z[r] *= f;
#pragma unroll
            for (int d = 0; d < 8; ++d) st.o[r][d] *= f;
        }
    }
    // Probabilities in two bf16 parts, the rounded value and the rest (2^-17 of it): out is then as exact as its own rounding
    // leaves it.  The second product doubles, which a call of few rows does not notice: it waits for K and V.
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

template <int RT, int MASK, bool KEEP>
__global__ __launch_bounds__(kAttendThreads, RT == 1 ? 3 : 2) void jq_attend_kernel(AttendArgs a) {
    extern __shared__ __align__(16) float lds[];  // [waves][16 RT][kOutStride], then (m, z) [waves][16 RT]
    float2* lds_stats = (float2*)(lds + kAttendWaves * RT * kTileRows * kOutStride);
    // blockIdx.x: groups of query rows over the same keys eight apart, so that they meet in one XCD's L2
    const int per = 8 * a.row_groups;
    const int u = (int)blockIdx.x / per * 8 + ((int)blockIdx.x & 7), rg = ((int)blockIdx.x % per) >> 3;
    if (u >= a.units) return;
    const int layer = blockIdx.y, split = u / a.h_kv, g = u - split * a.h_kv;
    const int s = find_seq(a.cu_split, a.n_seq, split);
    const int ns = a.cu_split[s + 1] - a.cu_split[s], mine = split - a.cu_split[s];
    const int n = live_rows(a.lens, a.n_seq, layer, s, a.cu_seq[s + 1] - a.cu_seq[s]);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const int row0 = rg * RT * kTileRows;

    RowState<RT> st;
    int row_limit[RT];
    const uint32_t* row_seen[RT];
    float* row_logits[RT];
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
        row_limit[r] = n - a.n_q + i + 1;
        row_seen[r] = MASK == kSeeTree ? a.seen + ((int64_t)s * a.n_q + i) * a.words : nullptr;
        row_logits[r] = nullptr;
        if (KEEP && row0 + r * kTileRows + (lane & 15) < a.rows)
            row_logits[r] = a.logits + (((int64_t)layer * a.h_kv + g) * a.rows + row) * a.logit_T + logit_at(a.cu_seq, s);
    }

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
    // keys from `open` on are not seen by every row
    const int open = MASK == kSeeAll ? n : max(n - a.n_q + (MASK == kSeeCausal ? 1 : 0), 0);
    const int step = 32 * kAttendWaves * ns;
    int key = 32 * (kAttendWaves * mine + wave);
    // One tile at a time: the waves of a SIMD take turns waiting, and together they ask for far more than memory needs to be asked for.
    KvTile t;
    for (; key + 32 <= open; key += step) {
        load_tile(t, K, V, tile_row(key), 31, stride, lane);
        tile_step<RT, false, MASK, KEEP>(st, t, a, lane, key, n, row_limit, row_seen, row_logits);
    }
    for (; key < n; key += step) {
        load_tile(t, K, V, tile_row(key), n - 1 - key, stride, lane);
        tile_step<RT, true, MASK, KEEP>(st, t, a, lane, key, n, row_limit, row_seen, row_logits);
    }

    // The four waves' sums, in wave order.
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        st.z[r] += __shfl_xor(st.z[r], 16);
        st.z[r] += __shfl_xor(st.z[r], 32);
        if (lane < 16) lds_stats[(wave * RT + r) * kTileRows + lane] = make_float2(st.m[r], st.z[r]);
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < RT; ++r) {
        float m = -__builtin_inff();
#pragma unroll
        for (int w = 0; w < kAttendWaves; ++w) m = fmaxf(m, lds_stats[(w * RT + r) * kTileRows + (lane & 15)].x);
        const float f = st.m[r] == m ? 1.0f : __builtin_amdgcn_exp2f(st.m[r] - m);
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
    for (int item = threadIdx.x; item < RT * kTileRows * 32; item += kAttendThreads) {
        const int r = item >> 5, d = (item & 31) * 4, row = row0 + r;
        if (row >= a.rows) break;
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
        if (ns > 1 || KEEP) {
            if (ns > 1) *(f32x4*)(a.part + (part_row + row) * kHeadDim + d) = o;
            if (d == 0) a.stats[part_row + row] = make_float2(m, z);
        }
        if (ns == 1) {
            const int i = row / a.group, h = g * a.group + row - i * a.group;
            const int64_t q_row = (((int64_t)layer * a.n_seq + s) * a.n_q + i) * a.h_q + h;
            const float inv = z == 0.0f ? 0.0f : 1.0f / z;  // a row that sees nothing: zeros, and -inf for its log-sum-exp
            __bf16 y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = (__bf16)(o[e] * inv);
            *(uint2*)(a.out + q_row * kHeadDim + d) = *(const uint2*)y;
            if (a.lse && d == 0) a.lse[q_row] = z == 0.0f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(z)) * 0.69314718055994531f;
        }
    }
}

// Joins the workgroups of every sequence that has several: out and lse of all query rows.  Eight rows a workgroup.
constexpr int kJoinRows = 8;
__global__ __launch_bounds__(kJoinRows * 32) void jq_attend_join_kernel(AttendArgs a) {
    const int chunks = (a.rows + kJoinRows - 1) / kJoinRows;
    const int unit = (int)blockIdx.x / chunks, row = ((int)blockIdx.x - unit * chunks) * kJoinRows + (int)(threadIdx.x >> 5);
    const int s = unit / a.h_kv, g = unit - s * a.h_kv, layer = blockIdx.y, d = (threadIdx.x & 31) * 4;
    const int first = a.cu_split[s], ns = a.cu_split[s + 1] - first;
    if (ns == 1 || row >= a.rows) return;
    const int64_t at = (((int64_t)layer * a.n_splits + first) * a.h_kv + g) * a.rows + row, step = (int64_t)a.h_kv * a.rows;
    float m = -__builtin_inff(), z = 0.0f;
    for (int i = 0; i < ns; ++i) m = fmaxf(m, a.stats[at + i * step].x);
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int i = 0; i < ns; ++i) {
        const float2 mz = a.stats[at + i * step];
        const float f = mz.x == m ? 1.0f : __builtin_amdgcn_exp2f(mz.x - m);
        z += mz.y * f;
        o += *(const f32x4*)(a.part + (at + i * step) * kHeadDim + d) * f;
    }
    const int i = row / a.group, h = g * a.group + row - i * a.group;
    const int64_t q_row = (((int64_t)layer * a.n_seq + s) * a.n_q + i) * a.h_q + h;
    const float inv = z == 0.0f ? 0.0f : 1.0f / z;
    __bf16 y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (__bf16)(o[e] * inv);
    *(uint2*)(a.out + q_row * kHeadDim + d) = *(const uint2*)y;
    if (a.lse && d == 0) a.lse[q_row] = z == 0.0f ? -__builtin_inff() : (m + __builtin_amdgcn_logf(z)) * 0.69314718055994531f;
}

// weights[j] += sum_r p[r,j], from the logits that the sweep has kept: 1024 rows of the cache a workgroup.
constexpr int kWeighKeys = 1024;
__global__ __launch_bounds__(256) void jq_attend_weigh_kernel(AttendArgs a, int blocks_per_seq) {
    __shared__ float lse2[kMaxWeighRows];
    const int b = (int)blockIdx.x % blocks_per_seq, unit = (int)blockIdx.x / blocks_per_seq;
    const int s = unit / a.h_kv, g = unit - s * a.h_kv, layer = blockIdx.y;
    const int n = live_rows(a.lens, a.n_seq, layer, s, a.cu_seq[s + 1] - a.cu_seq[s]);
    if (b * kWeighKeys >= n) return;
    const int first = a.cu_split[s], ns = a.cu_split[s + 1] - first;
    const int64_t at = (((int64_t)layer * a.n_splits + first) * a.h_kv + g) * a.rows, step = (int64_t)a.h_kv * a.rows;
    if ((int)threadIdx.x < a.rows) {
        float m = -__builtin_inff(), z = 0.0f;
        for (int i = 0; i < ns; ++i) m = fmaxf(m, a.stats[at + threadIdx.x + i * step].x);
        for (int i = 0; i < ns; ++i) {
            const float2 mz = a.stats[at + threadIdx.x + i * step];
            z += mz.x == m ? mz.y : mz.y * __builtin_amdgcn_exp2f(mz.x - m);
        }
        lse2[threadIdx.x] = z == 0.0f ? 0.0f : m + __builtin_amdgcn_logf(z);  // nothing seen: all its logits are -inf
    }
    __syncthreads();
    const float* x = a.logits + ((int64_t)layer * a.h_kv + g) * a.rows * a.logit_T + logit_at(a.cu_seq, s);
    float* w = a.weights + ((int64_t)layer * a.h_kv + g) * a.T + a.cu_seq[s];
    for (int j = b * kWeighKeys + threadIdx.x; j < min((b + 1) * kWeighKeys, n); j += 256) {
        float sum = 0.0f;
        for (int r = 0; r < a.rows; ++r) sum += __builtin_amdgcn_exp2f(x[r * a.logit_T + j] - lse2[r]);
        w[j] += sum;
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------------

// How many workgroups share each sequence: as many as make some two per CU over the whole call, none with fewer than 128 rows of
// the cache to itself.
static void plan_splits(const Plan& p, AttendPlan* ap) {
    const int row_tiles = (p.rows + kTileRows - 1) / kTileRows;
    ap->row_tiles = row_tiles <= 1 ? 1 : 2;
    ap->row_groups = (row_tiles + ap->row_tiles - 1) / ap->row_tiles;
    const int64_t heads = (int64_t)p.n_layers * p.h_kv * ap->row_groups;
    const int64_t rows_per = std::max<int64_t>(128, (p.T * heads + 511) / 512);
    ap->cu_split[0] = 0;
    for (int s = 0; s < p.n_seq; ++s) {
        const int64_t L = p.tab.cu_seq[s + 1] - p.tab.cu_seq[s];
        ap->cu_split[s + 1] = ap->cu_split[s] + (int32_t)((L + rows_per - 1) / rows_per);
    }
}

void plan_attend(const Plan& p, bool weights, AttendPlan* ap) {
    plan_splits(p, ap);
    const size_t parts = (size_t)p.n_layers * ap->cu_split[p.n_seq] * p.h_kv * p.rows;
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    ap->logit_T = 32 * (p.T / 32 + p.n_seq);
    ap->off_stats = 0;
    ap->off_part = up(parts * sizeof(float2));
    ap->off_logits = ap->off_part + up(parts * kHeadDim * sizeof(float));
    ap->ws_bytes = ap->off_logits + (weights ? up((size_t)p.n_layers * p.h_kv * p.rows * ap->logit_T * sizeof(float)) : 0);
}

bool attend_fits(const Plan& p, const AttendPlan& ap) {
    const int64_t most = UINT32_MAX;
    const int64_t sweep = ((int64_t)ap.cu_split[p.n_seq] * p.h_kv + 8) * ap.row_groups * kAttendThreads;
    const int64_t join = (int64_t)p.n_seq * p.h_kv * ((p.rows + kJoinRows - 1) / kJoinRows) * (kJoinRows * 32);
    return sweep <= most && join <= most;
}

template <int RT, int MASK, bool KEEP>
static hipError_t launch_sweep(const AttendArgs& a, hipStream_t st) {
    constexpr int lds = kAttendWaves * RT * kTileRows * (kOutStride * 4 + 8);
    if (lds > 65536) {
        static std::atomic<uint64_t> done{0};
        const hipError_t e = allow_dynamic_lds((const void*)jq_attend_kernel<RT, MASK, KEEP>, lds, done);
        if (e != hipSuccess) return e;
    }
    const dim3 grid((unsigned)((a.units + 7) / 8 * 8 * a.row_groups), (unsigned)a.n_layers);
    return launch_kernel(jq_attend_kernel<RT, MASK, KEEP>, grid, dim3(kAttendThreads), lds, st, nullptr, -1, a);
}

template <int MASK, bool KEEP>
static hipError_t launch_rows(const AttendArgs& a, int row_tiles, hipStream_t st) {
    return row_tiles == 1 ? launch_sweep<1, MASK, KEEP>(a, st) : launch_sweep<2, MASK, KEEP>(a, st);
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
    a.scale2 = (float)(p.scale * 1.4426950408889634);
    a.T = p.T; a.logit_T = ap.logit_T;
    a.pm = p.page_map();
    for (int s = 0; s <= p.n_seq; ++s) { a.cu_seq[s] = p.tab.cu_seq[s]; a.cu_split[s] = ap.cu_split[s]; }
    // one new token sees every live row, its own among them: no mask either way
    hipError_t e;
    if (seen) e = launch_rows<kSeeTree, false>(a, ap.row_tiles, st);
    else if (p.window && p.n_q > 1) e = weights ? launch_rows<kSeeCausal, true>(a, ap.row_tiles, st) : launch_rows<kSeeCausal, false>(a, ap.row_tiles, st);
    else e = weights ? launch_rows<kSeeAll, true>(a, ap.row_tiles, st) : launch_rows<kSeeAll, false>(a, ap.row_tiles, st);
    if (e != hipSuccess) return e;
    if (a.n_splits > p.n_seq) {
        const dim3 grid((unsigned)(p.n_seq * p.h_kv * ((p.rows + kJoinRows - 1) / kJoinRows)), (unsigned)p.n_layers);
        e = launch_kernel(jq_attend_join_kernel, grid, dim3(kJoinRows * 32), 0, st, nullptr, -1, a);
        if (e != hipSuccess) return e;
    }
    if (weights) {
        int32_t most = 0;
        for (int s = 0; s < p.n_seq; ++s) most = std::max(most, p.tab.cu_seq[s + 1] - p.tab.cu_seq[s]);
        const int blocks = (most + kWeighKeys - 1) / kWeighKeys;
        e = launch_kernel(jq_attend_weigh_kernel, dim3((unsigned)(blocks * p.n_seq * p.h_kv), (unsigned)p.n_layers), dim3(256), 0, st, nullptr, -1, a, blocks);
    }
    return e;
}

}  // namespace jq
