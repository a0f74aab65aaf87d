// Eviction by accumulated attention weight (the accumulated-attention baseline that Section 5.1 compares with): every cached row
// carries the sum of the attention it has received (jq_attend adds to it) and the position of the token it came from.
//
//   jq_evict_weight        many rows at once: the B heaviest rows of a (layer, sequence, KV head) move to the front of the
//                          sequence's segment, in order, their weights and positions with them
//   jq_replace_lightest    one token: its row takes the slot of the lightest one
//
// Rows of the first keep_first positions and of the newest keep_last are never taken, whatever they weigh.
#include <type_traits>

#include "jq_common.h"

namespace jq {

typedef uint32_t wu32x4 __attribute__((ext_vector_type(4)));

struct WeightArgs {
    const char* K; const char* V;
    char* K_out; char* V_out;
    const float* weights; float* weights_out;  // [n_layers][h_kv][T]
    const int32_t* pos; int32_t* pos_out;      // the same; pos null: a row's number is its position; pos_out may be null
    const int32_t* lens;                       // DEVICE [n_layers][n_seq] live rows, or null: all
    int32_t* idx;                              // [n_layers][h_kv][TB]
    // long sequences, in pieces of kPieceRows rows: each piece's largest position [n_layers][h_kv][n_pieces], and the rows that its
    // selection kept [n_layers][h_kv][n_cand] (weight, position, number), piece after piece
    int32_t* newest;
    float* cand_w; int32_t* cand_pos; int32_t* cand_row;
    int32_t n_pieces, n_cand;
    int64_t first_item;                        // of a launch of the copy: (layer, kept row, head)
    int32_t own_newest;                        // every piece looks through all of its sequence's positions: no launch for `newest`
    int32_t cu_piece[JQ_MAX_SEQ + 1], cu_cand[JQ_MAX_SEQ + 1];
    const int32_t* layer_budgets;
    int32_t n_layers, h_kv, keep_first, keep_last;
    int64_t T, TB;
    PageMap pm;
    SeqTab tab;
};

__device__ __forceinline__ int live_of(const int32_t* lens, int n_seq, int layer, int s, int cap) {
    return lens ? min(max(lens[(int64_t)layer * n_seq + s], 0), cap) : cap;
}

// What a row is ranked by: its weight, and above every weight, a NaN of all ones too, the rows that stay.
constexpr uint32_t kStays = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t free_key(float w) { return min(sortable_key(w), kStays - 1u); }
__device__ __forceinline__ uint32_t weight_key(float w, int pos, int keep_first, int64_t recent) {
    return pos < keep_first || pos > recent ? kStays : free_key(w);
}

// One workgroup per (layer, sequence, KV head): exact radix select over the weights' keys, 11, 11 and 10 bits, then the kept rows
// in ascending order with their weights and positions.  Each of the sixteen waves owns a run of rows, 256 of them (four a lane) a
// round; up to ROUNDS rounds are held in registers with their keys, which the whole selection then works on, and longer runs are read
// again in every pass, four rounds at a time.  It is one chain of waits and of instructions that four waves of a SIMD take turns
// with (7 ns each): every level has a histogram of its own, cleared while the first rows are on their way, and three barriers; a row
// costs some thirty instructions, places being counted by ballots, wave by wave, with one barrier around the waves' totals.
// In place every slot written is at or before the row it comes from: what is held in registers has been read by then (one barrier),
// and longer runs are moved by one wave after the other, each of its rounds read before it is written.
constexpr int kWeightThreads = 1024, kWeightWaves = kWeightThreads / 64, kRoundRows = 256;
constexpr int kWeightBins = 2048;
constexpr int kFirstCopies = 4, kRestCopies = 2;  // of histograms, by lane: adds to one address take turns
constexpr int kHistWords = kWeightBins * (kFirstCopies + 2 * kRestCopies);
typedef float any_float4 __attribute__((ext_vector_type(4), aligned(4)));
typedef int32_t any_int4 __attribute__((ext_vector_type(4), aligned(4)));

// Four rows' weights and positions, and their keys where they are ranked.
struct FourRows {
    float w[4];
    int32_t pos[4];
    uint32_t key[4];
    // the rows from j on, of which there are n; without positions they are the rows' numbers, `base` for the first
    __device__ __forceinline__ void load(const float* from_w, const int32_t* from_pos, int j, int n, int base) {
        if (j + 4 <= n) {
            *(any_float4*)w = *(const any_float4*)(from_w + j);
            if (from_pos) *(any_int4*)pos = *(const any_int4*)(from_pos + j);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                w[e] = j + e < n ? from_w[j + e] : 0.0f;
                if (from_pos) pos[e] = j + e < n ? from_pos[j + e] : 0;
            }
        }
        if (!from_pos) {
#pragma unroll
            for (int e = 0; e < 4; ++e) pos[e] = base + j + e;
        }
    }
    // Keys: above every weight's those of rows from position keep_first + inner on, and, as the difference wraps, below keep_first; 0
    // behind the last row.  A row may have that key too; it comes before those, and never are more rows asked for than there are.
    __device__ __forceinline__ void rank(int j, int n, int keep_first, uint32_t inner) {
#pragma unroll
        for (int e = 0; e < 4; ++e) key[e] = (uint32_t)pos[e] - (uint32_t)keep_first >= inner ? kStays : free_key(w[e]);
        if (j + 4 > n) {
#pragma unroll
            for (int e = 0; e < 4; ++e) key[e] = j + e < n ? key[e] : 0u;
        }
    }
};

// STAGE: a sequence of many times as many rows as it keeps is selected from twice, so that more than one workgroup reads it:
// kPieces, its pieces of kPieceRows rows leave a budget's worth of rows each, and kRest, the budget's rows are chosen from those.
// Whatever the sequence keeps, its piece keeps; pieces and rows stay in order, so equal weights still go to the lower row.
enum WeightStage { kAllRows = 0, kPieces, kRest };
constexpr int kPieceRows = 4 * kWeightWaves * kRoundRows;  // what a workgroup holds

// The largest position of every piece.
__global__ __launch_bounds__(kWeightThreads) void jq_weight_newest_kernel(WeightArgs a) {
    __shared__ uint32_t most[kWeightWaves];
    const int piece = (int)blockIdx.x / a.h_kv, g = (int)blockIdx.x - piece * a.h_kv, layer = blockIdx.y, tid = threadIdx.x;
    const int s = find_seq(a.cu_piece, a.tab.n_seq, piece), base = (piece - a.cu_piece[s]) * kPieceRows;
    const int n = min(live_of(a.lens, a.tab.n_seq, layer, s, a.tab.cu_seq[s + 1] - a.tab.cu_seq[s]) - base, kPieceRows);
    const int32_t* pos = a.pos + ((int64_t)layer * a.h_kv + g) * a.T + a.tab.cu_seq[s] + base;
    int newest = INT32_MIN;
#pragma unroll 4
    for (int j = tid; j < n; j += kWeightThreads) newest = max(newest, pos[j]);
    const uint32_t top = wave_max((uint32_t)newest ^ 0x80000000u);
    if ((tid & 63) == 0) most[tid >> 6] = top;
    __syncthreads();
    if (tid < 64) {
        const uint32_t x = wave_max(most[tid & (kWeightWaves - 1)]);
        if (tid == 0) a.newest[((int64_t)layer * a.h_kv + g) * a.n_pieces + piece] = (int32_t)(x ^ 0x80000000u);
    }
}

template <int ROUNDS, bool HELD, int STAGE>
__global__ __launch_bounds__(kWeightThreads) void jq_weight_select_kernel(WeightArgs a) {
    extern __shared__ __align__(16) uint32_t hist[];
    __shared__ uint32_t scan[3][kWeightWaves];
    __shared__ uint2 totals[kWeightWaves];
    __shared__ uint32_t picked[3][3];
    const int unit = (int)blockIdx.x / a.h_kv, g = (int)blockIdx.x - unit * a.h_kv, layer = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int s = STAGE == kPieces ? find_seq(a.cu_piece, a.tab.n_seq, unit) : unit;
    const int cap = a.tab.cu_seq[s + 1] - a.tab.cu_seq[s];
    const int64_t head = (int64_t)layer * a.h_kv + g, row0 = head * a.T + a.tab.cu_seq[s];
    // Where the rows come from.  What is held is requested before the live count and the budget are known: rows up to the capacity are
    // the caller's.
    const float* w = a.weights + row0;
    const int32_t* pos = a.pos ? a.pos + row0 : nullptr;
    const int piece = STAGE == kPieces ? unit - a.cu_piece[s] : 0, base = piece * kPieceRows;
    int room = STAGE == kPieces ? min(cap - base, kPieceRows) : cap;
    if (STAGE == kPieces) {
        w += base;
        if (pos) pos += base;
    }
    FourRows held[ROUNDS];
    int rounds, first;  // of a wave
    auto read = [&](int i0) {
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i)
            if (i0 + i < rounds) held[i].load(w, pos, first + (i0 + i) * kRoundRows, room, base);
    };
    auto divide = [&]() {
        rounds = (room + kWeightWaves * kRoundRows - 1) / (kWeightWaves * kRoundRows);
        first = wave * rounds * kRoundRows + 4 * lane;
    };
    if (HELD && STAGE != kRest) {
        divide();
        read(0);
    }
    const int live = live_of(a.lens, a.tab.n_seq, layer, s, cap);
    const uint32_t B = budget_of(a.layer_budgets, a.tab, layer, s, a.keep_first + a.keep_last);
    // how many there are, and where those that are kept go
    const int32_t* number = nullptr;  // the rows' numbers; null: 0, 1, ...
    float* w_to = a.weights_out + row0;
    int32_t* pos_to = a.pos_out ? a.pos_out + row0 : nullptr;
    int32_t* number_to = a.idx + head * a.TB + a.tab.cu_bud[s];
    int n = live;
    const int per_piece = (int)min((uint32_t)kPieceRows, B);  // rows that a whole piece leaves
    const bool pieced = live > kPieceRows && (uint32_t)live > B;
    if (STAGE == kPieces) {
        if (!pieced) return;
        n = min(live - base, kPieceRows);
        if (n <= 0) return;
        const int64_t to = head * a.n_cand + a.cu_cand[s] + (int64_t)piece * per_piece;
        w_to = a.cand_w + to;
        pos_to = a.cand_pos + to;
        number_to = a.cand_row + to;
    }
    if (STAGE == kRest && pieced) {
        const int64_t from = head * a.n_cand + a.cu_cand[s];
        w = a.cand_w + from;
        pos = a.cand_pos + from;
        number = a.cand_row + from;
        n = live / kPieceRows * per_piece + min(live % kPieceRows, per_piece);
    }
    if (!HELD || STAGE == kRest) {
        room = n;
        divide();
        if (HELD) read(0);
    }
    const bool all = (uint32_t)n <= B;
    uint32_t inner = 0;  // positions between those that stay
    auto rank = [&](int i0) {
#pragma unroll
        for (int i = 0; i < ROUNDS; ++i)
            if (i0 + i < rounds) held[i].rank(first + (i0 + i) * kRoundRows, n, a.keep_first, inner);
    };
    auto visit = [&](bool ranked, auto f) {  // f(row, four rows from it) for every round of the wave
        for (int i0 = 0; i0 < (HELD ? 1 : rounds); i0 += ROUNDS) {
            if (!HELD) read(i0);
            if (!HELD && ranked) rank(i0);
#pragma unroll
            for (int i = 0; i < ROUNDS; ++i)
                if (i0 + i < rounds) f(first + (i0 + i) * kRoundRows, held[i]);
        }
    };
    if (!all || STAGE == kPieces) {  // (a piece that leaves all its rows still tells the newest)
        for (int i = tid; i < kHistWords / 4; i += kWeightThreads) ((uint4*)hist)[i] = make_uint4(0u, 0u, 0u, 0u);
        int newest = live - 1;  // without positions
        if (a.keep_last > 0 && a.pos) {
            int top = INT32_MIN;
            if (STAGE != kAllRows && pieced && !(STAGE == kPieces && a.own_newest)) {
                const int pieces = (live + kPieceRows - 1) / kPieceRows;
                for (int i = lane; i < pieces; i += 64) top = max(top, a.newest[head * a.n_pieces + a.cu_piece[s] + i]);
            } else {
                auto raise = [&](int j, const FourRows& r) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) top = j + e < n ? max(top, r.pos[e]) : top;
                };
                visit(false, raise);
                if (STAGE == kPieces) {  // the other pieces' positions
                    const int32_t* from = pos - base;
#pragma unroll 4
                    for (int j = 4 * tid; j + 4 <= live; j += 4 * kWeightThreads) {
                        const any_int4 x = *(const any_int4*)(from + j);
                        top = max(max(max(top, x[0]), max(x[1], x[2])), x[3]);
                    }
                    if (tid < live % 4) top = max(top, from[live - 1 - tid]);
                }
                const uint32_t in_wave = wave_max((uint32_t)top ^ 0x80000000u);
                if (lane == 0) scan[2][wave] = in_wave;
                lds_barrier();
                top = (int)(scan[2][lane & (kWeightWaves - 1)] ^ 0x80000000u);
            }
            newest = (int)(wave_max((uint32_t)top ^ 0x80000000u) ^ 0x80000000u);
            if (STAGE == kPieces && a.own_newest && tid == 0) a.newest[head * a.n_pieces + unit] = newest;
        }
        // (all rows' positions are at most `newest` where any stay for being new, so none is keep_first + inner by wrapping)
        const int64_t between = (int64_t)newest - a.keep_last - a.keep_first + 1;
        inner = all ? 0u : a.keep_last == 0 ? 0x80000000u - (uint32_t)a.keep_first : (uint32_t)max(between, (int64_t)0);
    }
    if (HELD) rank(0);
    uint32_t tau = 0, ties = 0;  // every key above tau is kept, and the first `ties` rows of key tau
    if (!all) {
        uint32_t left = B;  // places left among the keys that agree with tau under the levels' bits so far
        lds_barrier();      // histograms are clear
        auto level = [&](auto which) {  // true: no row of the bin that is found goes
            constexpr int L = decltype(which)::value, shift = L == 0 ? 21 : L == 1 ? 10 : 0, copies = L == 0 ? kFirstCopies : kRestCopies;
            constexpr uint32_t bins = L == 2 ? 1024 : 2048, mask = L == 0 ? 0u : L == 1 ? 0xFFE00000u : 0xFFFFFC00u;
            uint32_t* h = hist + (L == 0 ? 0 : kWeightBins * (kFirstCopies + (L - 1) * kRestCopies)), *mine = h + (lane & (copies - 1));
            visit(true, [&](int j, const FourRows& r) {
                if (j < n) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (L == 0 || (r.key[e] & mask) == tau) atomicAdd(mine + ((r.key[e] >> shift) & (bins - 1)) * copies, 1u);
                }
            });
            lds_barrier();
            // two bins a thread, from the largest down: the one in which the running count passes `left`
            uint32_t c[2] = {0, 0};
#pragma unroll
            for (int i = 0; i < copies; ++i) {
                const uint32_t* two = h + (kWeightBins - 2 - 2 * tid) * copies;
                c[0] += two[copies + i];
                c[1] += two[i];
            }
            auto add = [](uint32_t x, uint32_t y) { return x + y; };
            const uint32_t in_wave = wave_scan(c[0] + c[1], 0u, add);
            if (lane == 63) scan[L & 1][wave] = in_wave;
            lds_barrier();
            const uint32_t waves = row_scan(lane < kWeightWaves ? scan[L & 1][lane] : 0u, 0u, add);
            const uint32_t upto = in_wave + (wave > 0 ? (uint32_t)__builtin_amdgcn_readlane((int)waves, wave > 0 ? wave - 1 : 0) : 0u), before = upto - c[0] - c[1];
            if (before < left && left <= upto) {
                const bool upper = left <= before + c[0];
                picked[L][0] = kWeightBins - 1 - (2 * tid + (upper ? 0 : 1));
                picked[L][1] = left - before - (upper ? 0u : c[0]);
                picked[L][2] = c[upper ? 0 : 1];
            }
            lds_barrier();
            tau |= picked[L][0] << shift;
            left = picked[L][1];
            return left == picked[L][2] && tau;
        };
        // The whole bin stays, as it mostly does from the second level on: it often holds one row.
        if (level(std::integral_constant<int, 0>()) || level(std::integral_constant<int, 1>()) || level(std::integral_constant<int, 2>())) {
            tau -= 1;
            left = 0;
        }
        ties = left;
    }
    // What every wave keeps for certain, and its ties.
    uint32_t sure = 0, tied = 0;
    visit(true, [&](int, const FourRows& r) {
#pragma unroll
        for (int e = 0; e < 4; ++e) sure += (uint32_t)__popcll(__ballot(r.key[e] > tau));
        if (ties > 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) tied += (uint32_t)__popcll(__ballot(r.key[e] == tau));
        }
    });
    if (lane == 0) totals[wave] = make_uint2(sure, tied);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // what is held has been read, by every wave
    __syncthreads();
    uint32_t sure_before = 0, ties_before = 0;
#pragma unroll
    for (int i = 0; i < kWeightWaves; ++i) {
        const uint2 t = totals[i];
        sure_before += i < wave ? t.x : 0u;
        ties_before += i < wave ? t.y : 0u;
    }
    auto lower = [](uint64_t votes, uint32_t from) {  // `from` and the votes of lower lanes
        return __builtin_amdgcn_mbcnt_hi((uint32_t)(votes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)votes, from));
    };
    auto emit = [&](int j, const FourRows& r) {
        uint32_t s0 = sure_before, t0 = ties_before;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint64_t votes = __ballot(r.key[e] > tau);
            s0 = lower(votes, s0);
            sure_before += (uint32_t)__popcll(votes);
        }
        if (ties > 0) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint64_t votes = __ballot(r.key[e] == tau);
                t0 = lower(votes, t0);
                ties_before += (uint32_t)__popcll(votes);
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const bool surely = r.key[e] > tau, tie = r.key[e] == tau;
            const uint32_t to = 4 * (s0 + min(t0, ties));  // (32 bits: fewer than 2^30 rows fit 4 GiB of keys)
            if (surely || (tie && t0 < ties)) {
                *(int32_t*)((char*)number_to + to) = number ? number[j + e] : base + j + e;
                *(float*)((char*)w_to + to) = r.w[e];
                if (pos_to) *(int32_t*)((char*)pos_to + to) = r.pos[e];
            }
            s0 += surely;
            t0 += tie;
        }
    };
    if (HELD || w_to != w) {
        visit(true, emit);
        return;
    }
    for (int turn = 0; turn < kWeightWaves; ++turn) {
        // (a visit reads its next rounds before it writes into earlier rows only)
        if (turn == wave) visit(true, emit);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    }
}

// The kept rows of K and V, out of one cache into another: sixteen bytes a lane, sixteen lanes a row.  Bound by memory where rows lie side
// by side (2048 of 2560 rows in 32 layers 91 us, 5.9 TB/s), by each lane's chain of four reads where they do not (16 paged sequences 34 us, 4 TB/s).
constexpr int kMoveThreads = 256;
__global__ __launch_bounds__(kMoveThreads) void jq_weight_copy_kernel(WeightArgs a) {
    const int64_t item = a.first_item + ((int64_t)blockIdx.x * kMoveThreads + threadIdx.x) / 16;  // (layer, kept row, head), heads fastest
    if (item >= (int64_t)a.n_layers * a.TB * a.h_kv) return;
    const int g = (int)(item % a.h_kv), part = threadIdx.x & 15;
    const int64_t tb = item / a.h_kv % a.TB;
    const int layer = (int)(item / a.h_kv / a.TB);
    const int s = find_seq(a.tab.cu_bud, a.tab.n_seq, tb), b = (int)(tb - a.tab.cu_bud[s]);
    const int n = live_of(a.lens, a.tab.n_seq, layer, s, a.tab.cu_seq[s + 1] - a.tab.cu_seq[s]);
    if (b >= n || (uint32_t)b >= budget_of(a.layer_budgets, a.tab, layer, s, a.keep_first + a.keep_last)) return;
    const int j = a.idx[((int64_t)layer * a.h_kv + g) * a.TB + tb];
    const int64_t src = (kv_row(a.pm, a.tab.cu_seq, a.T, layer, s, j) * a.h_kv + g) * (kHeadDim * 2) + part * 16;
    const int64_t dst = (kv_row(a.pm, a.tab.cu_seq, a.T, layer, s, b) * a.h_kv + g) * (kHeadDim * 2) + part * 16;
    const wu32x4 k = *(const wu32x4*)(a.K + src), v = *(const wu32x4*)(a.V + src);
    __builtin_nontemporal_store(k, (wu32x4*)(a.K_out + dst));
    __builtin_nontemporal_store(v, (wu32x4*)(a.V_out + dst));
}

// The same within one cache.  A workgroup moves one 64-byte column of one head's K or V, front to back: a slot lies at or before
// the row that goes there and rows are in ascending order, so what a chunk overwrites has been read by it or by an earlier one.
// Columns have nothing to do with each other, so a (layer, sequence, head) is the work of eight workgroups.  Bound by its chunks, one
// after the other: 2048 of 2560 rows in 32 layers 162 us (the copy 101), 2048 of 65536 in one 26 (the copy 6).
constexpr int kShiftRows = 4 * kMoveThreads / 4;  // rows of a chunk: four lanes a row, four rows a lane
__global__ __launch_bounds__(kMoveThreads) void jq_weight_shift_kernel(WeightArgs a) {
    const int column = blockIdx.x & 3, g = (int)blockIdx.x >> 3, s = blockIdx.y, layer = blockIdx.z;
    char* base = (blockIdx.x & 4 ? a.V_out : a.K_out) + g * (kHeadDim * 2) + column * 64 + (threadIdx.x & 3) * 16;
    const int n = live_of(a.lens, a.tab.n_seq, layer, s, a.tab.cu_seq[s + 1] - a.tab.cu_seq[s]);
    const int B = (int)min((uint32_t)n, budget_of(a.layer_budgets, a.tab, layer, s, a.keep_first + a.keep_last));
    const int32_t* idx = a.idx + ((int64_t)layer * a.h_kv + g) * a.TB + a.tab.cu_bud[s];
    const int64_t stride = (int64_t)a.h_kv * (kHeadDim * 2);
    for (int b0 = 0; b0 < B; b0 += kShiftRows) {
        wu32x4 x[4];
        int from[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int b = b0 + i * (kMoveThreads / 4) + (int)(threadIdx.x >> 2);
            from[i] = b < B ? idx[b] : b;  // (a row that stays where it is is left alone)
            if (from[i] != b) x[i] = *(const wu32x4*)(base + kv_row(a.pm, a.tab.cu_seq, a.T, layer, s, from[i]) * stride);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // every row of the chunk has arrived before any is overwritten
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int b = b0 + i * (kMoveThreads / 4) + (int)(threadIdx.x >> 2);
            if (from[i] != b) *(wu32x4*)(base + kv_row(a.pm, a.tab.cu_seq, a.T, layer, s, b) * stride) = x[i];
        }
    }
}

struct ReplaceArgs {
    const char* k_new; const char* v_new;  // [n_layers][n_seq][h_kv][d]
    const int32_t* token;                  // DEVICE [n_seq]: the new rows' positions
    char* K; char* V;
    float* weights; int32_t* pos;
    const int32_t* lens;
    int32_t* slot;                         // [n_layers][n_seq][h_kv], may be null
    int32_t h_kv, keep_first, keep_last;
    int64_t T;
    PageMap pm;
    SeqTab tab;
};

// One workgroup per (layer, sequence, KV head): the row of least key (the lowest of equals) by a reduction, then the new row.  What
// it has to read is 8 bytes a row, so it waits more than it reads: four rows a lane and four requests at a time, the first of them
// ahead of the live count, which only decides whether they matter (rows up to the capacity are the caller's).
constexpr int kReplaceThreads = 256, kReplaceAhead = 4;
__global__ __launch_bounds__(kReplaceThreads) void jq_replace_kernel(ReplaceArgs a) {
    __shared__ uint64_t least[kReplaceThreads / 64];
    const int g = blockIdx.x, s = blockIdx.y, layer = blockIdx.z, tid = threadIdx.x;
    const int cap = a.tab.cu_seq[s + 1] - a.tab.cu_seq[s];
    const int64_t row0 = ((int64_t)layer * a.h_kv + g) * a.T + a.tab.cu_seq[s];
    const float* w = a.weights + row0;
    const int32_t* pos = a.pos + row0;
    FourRows rows[kReplaceAhead];
    auto read = [&](int base) {
#pragma unroll
        for (int i = 0; i < kReplaceAhead; ++i) {
            const int j = base + (i * kReplaceThreads + tid) * 4;
            if (j < cap) rows[i].load(w, pos, j, cap, 0);
        }
    };
    read(0);
    // the new row: sixteen lanes for K, sixteen for V
    const int part = tid & 15;
    wu32x4 fresh;
    if (tid < 32) {
        const int64_t from = (((int64_t)layer * a.tab.n_seq + s) * a.h_kv + g) * (kHeadDim * 2) + part * 16;
        fresh = *(const wu32x4*)((tid < 16 ? a.k_new : a.v_new) + from);
    }
    const int token = a.token[s], n = live_of(a.lens, a.tab.n_seq, layer, s, cap);
    int slot = n;  // room left: the next row
    if (n == cap) {
        const int64_t recent = (int64_t)token - a.keep_last;  // the new token counts among the newest
        uint64_t best = UINT64_MAX;
        for (int base = 0; base < n; base += 4 * kReplaceAhead * kReplaceThreads) {
            if (base > 0) read(base);
#pragma unroll
            for (int i = 0; i < kReplaceAhead; ++i) {
                const int j = base + (i * kReplaceThreads + tid) * 4;
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (j + e < n) {
                        const uint64_t k = (uint64_t)weight_key(rows[i].w[e], rows[i].pos[e], a.keep_first, recent) << 32 | (uint32_t)(j + e);
                        best = k < best ? k : best;
                    }
            }
        }
        // the least key of the wave, then the lowest row that has it
        const uint32_t key = (uint32_t)(best >> 32), top = wave_min(key), row = wave_min(key == top ? (uint32_t)best : 0xFFFFFFFFu);
        if ((tid & 63) == 0) least[tid >> 6] = (uint64_t)top << 32 | row;
        __syncthreads();
        best = least[0];
#pragma unroll
        for (int i = 1; i < kReplaceThreads / 64; ++i) best = least[i] < best ? least[i] : best;
        slot = (int)(uint32_t)best;
    }
    if (tid < 32) {
        const int64_t to = (kv_row(a.pm, a.tab.cu_seq, a.T, layer, s, slot) * a.h_kv + g) * (kHeadDim * 2) + part * 16;
        *(wu32x4*)((tid < 16 ? a.K : a.V) + to) = fresh;
    }
    if (tid == 32) {
        a.weights[row0 + slot] = 0.0f;
        a.pos[row0 + slot] = token;
        if (a.slot) a.slot[((int64_t)layer * a.tab.n_seq + s) * a.h_kv + g] = slot;
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------------

// Pieces or not: with pieces the last selection reads pieces * budget rows of every long sequence instead of all.  They are taken where
// that at least halves what it reads (65536 rows, 2048 kept, 8 heads: 30 us a call with pieces, 66 without).
void plan_evict_weight(const Plan& p, WeightPlan* wp) {
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    wp->cu_piece[0] = wp->cu_cand[0] = 0;
    wp->most_rows = 0;
    bool pays = false, costs = false;
    int64_t cand = 0;
    for (int s = 0; s < p.n_seq; ++s) {
        const int64_t L = p.tab.cu_seq[s + 1] - p.tab.cu_seq[s], B = p.tab.cu_bud[s + 1] - p.tab.cu_bud[s];
        const int64_t pieces = L > kPieceRows ? (L + kPieceRows - 1) / kPieceRows : 0, left = pieces * std::min<int64_t>(B, kPieceRows);
        if (pieces) (2 * left <= L ? pays : costs) = true;
        cand += left;
        wp->cu_piece[s + 1] = wp->cu_piece[s] + (int32_t)pieces;
        wp->cu_cand[s + 1] = (int32_t)std::min<int64_t>(cand, INT32_MAX);
        wp->most_rows = std::max(wp->most_rows, (int32_t)(pieces ? left : L));
    }
    if (!pays || costs || cand > INT32_MAX) {
        wp->most_rows = 0;
        for (int s = 0; s < p.n_seq; ++s) {
            wp->cu_piece[s + 1] = wp->cu_cand[s + 1] = 0;
            wp->most_rows = std::max(wp->most_rows, p.tab.cu_seq[s + 1] - p.tab.cu_seq[s]);
        }
    }
    const size_t heads = (size_t)p.n_layers * p.h_kv;
    wp->off_newest = up(heads * p.TB * sizeof(int32_t));  // (the kept rows' numbers in front, for callers that do not take them)
    wp->off_cand = wp->off_newest + up(heads * wp->cu_piece[p.n_seq] * sizeof(int32_t));
    wp->ws_bytes = wp->off_cand + up(heads * wp->cu_cand[p.n_seq] * 3 * sizeof(int32_t));
}

// Up to this many pieces each of them reads the others' positions too, instead of a launch that finds every piece's largest (us a call,
// 8 heads: four pieces 30.1, with the launch 32.0; eight 37.2 / 37.4, of four layers 51.9 / 51.6).
constexpr int kOwnNewest = 4;

template <int ROUNDS, bool HELD, int STAGE>
static hipError_t launch_select(const WeightArgs& a, dim3 grid, hipStream_t st) {
    constexpr int lds = kHistWords * 4;
    static std::atomic<uint64_t> done{0};
    const hipError_t e = allow_dynamic_lds((const void*)jq_weight_select_kernel<ROUNDS, HELD, STAGE>, lds, done);
    if (e != hipSuccess) return e;
    return launch_kernel(jq_weight_select_kernel<ROUNDS, HELD, STAGE>, grid, dim3(kWeightThreads), lds, st, nullptr, -1, a);
}

hipError_t launch_evict_weight(const Plan& p, const WeightPlan& wp, const int32_t* lens, const void* K, const void* V, const float* weights, const int32_t* pos,
                               void* K_out, void* V_out, float* weights_out, int32_t* pos_out, int32_t* idx, char* ws, hipStream_t st) {
    WeightArgs a{};
    a.K = (const char*)K; a.V = (const char*)V; a.K_out = (char*)K_out; a.V_out = (char*)V_out;
    a.weights = weights; a.weights_out = weights_out; a.pos = pos; a.pos_out = pos_out; a.lens = lens; a.idx = idx;
    a.layer_budgets = p.layer_budgets;
    a.n_layers = p.n_layers; a.h_kv = p.h_kv; a.keep_first = p.keep_first; a.keep_last = p.keep_last;
    a.T = p.T; a.TB = p.TB; a.pm = p.page_map(); a.tab = p.tab;
    a.n_pieces = wp.cu_piece[p.n_seq]; a.n_cand = wp.cu_cand[p.n_seq];
    for (int s = 0; s <= p.n_seq; ++s) { a.cu_piece[s] = wp.cu_piece[s]; a.cu_cand[s] = wp.cu_cand[s]; }
    a.newest = (int32_t*)(ws + wp.off_newest);
    a.cand_w = (float*)(ws + wp.off_cand);
    a.cand_pos = (int32_t*)(a.cand_w + (size_t)p.n_layers * p.h_kv * a.n_cand);
    a.cand_row = a.cand_pos + (size_t)p.n_layers * p.h_kv * a.n_cand;
    const dim3 whole((unsigned)(p.n_seq * p.h_kv), (unsigned)p.n_layers), pieces((unsigned)(a.n_pieces * p.h_kv), (unsigned)p.n_layers), block(kWeightThreads);
    hipError_t e = hipSuccess;
    if (a.n_pieces > 0) {
        int32_t most = 0;
        for (int s = 0; s < p.n_seq; ++s) most = std::max(most, wp.cu_piece[s + 1] - wp.cu_piece[s]);
        a.own_newest = most <= kOwnNewest;
        if (pos && p.keep_last > 0 && !a.own_newest) e = launch_kernel(jq_weight_newest_kernel, pieces, block, 0, st, nullptr, -1, a);
        if (e == hipSuccess) e = launch_select<4, true, kPieces>(a, pieces, st);
        if (e == hipSuccess) e = wp.most_rows <= kPieceRows ? launch_select<4, true, kRest>(a, whole, st) : launch_select<4, false, kRest>(a, whole, st);
    } else {
        e = wp.most_rows <= kPieceRows / 4 ? launch_select<1, true, kAllRows>(a, whole, st)
            : wp.most_rows <= kPieceRows   ? launch_select<4, true, kAllRows>(a, whole, st)
                                           : launch_select<4, false, kAllRows>(a, whole, st);
    }
    if (e != hipSuccess) return e;
    if (K_out == K)
        return launch_kernel(jq_weight_shift_kernel, dim3((unsigned)(8 * p.h_kv), (unsigned)p.n_seq, (unsigned)p.n_layers), dim3(kMoveThreads), 0, st, nullptr, -1, a);
    constexpr int64_t group = kMoveThreads / 16, most = (int64_t)(UINT32_MAX / kMoveThreads) * group;  // rows of a workgroup, of a launch
    const int64_t items = (int64_t)p.n_layers * p.TB * p.h_kv;
    for (; a.first_item < items; a.first_item += most) {
        const unsigned groups = (unsigned)((std::min(items - a.first_item, most) + group - 1) / group);
        e = launch_kernel(jq_weight_copy_kernel, dim3(groups), dim3(kMoveThreads), 0, st, nullptr, -1, a);
        if (e != hipSuccess) break;
    }
    return e;
}

hipError_t launch_replace(const Plan& p, const int32_t* lens, const void* k_new, const void* v_new, const int32_t* token, void* K, void* V, float* weights,
                          int32_t* pos, int32_t* slot, hipStream_t st) {
    ReplaceArgs a{};
    a.k_new = (const char*)k_new; a.v_new = (const char*)v_new; a.token = token; a.K = (char*)K; a.V = (char*)V;
    a.weights = weights; a.pos = pos; a.lens = lens; a.slot = slot;
    a.h_kv = p.h_kv; a.keep_first = p.keep_first; a.keep_last = p.keep_last;
    a.T = p.T; a.pm = p.page_map(); a.tab = p.tab;
    return launch_kernel(jq_replace_kernel, dim3((unsigned)p.h_kv, (unsigned)p.n_seq, (unsigned)p.n_layers), dim3(kReplaceThreads), 0, st, nullptr, -1, a);
}

}  // namespace jq
