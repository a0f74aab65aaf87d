// Eviction by accumulated attention weight (the accumulated-attention baseline that Section 5.1 compares with): every cached row
// carries the sum of the attention it has received (jq_attend adds to it) and the position of the token it came from.
//
//   jq_evict_weight        many rows at once: the B heaviest rows of a (layer, sequence, KV head) move to the front of the
//                          sequence's segment, in order, their weights and positions with them
//   jq_replace_lightest    one token: its row takes the slot of the lightest one
//
// Rows of the first keep_first positions and of the newest keep_last are never taken, whatever they weigh.
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
    const int32_t* layer_budgets;
    int32_t n_layers, h_kv, keep_first, keep_last;
    int64_t T, TB;
    PageMap pm;
    SeqTab tab;
};

__device__ __forceinline__ int live_of(const int32_t* lens, int n_seq, int layer, int s, int cap) {
    return lens ? min(max(lens[(int64_t)layer * n_seq + s], 0), cap) : cap;
}

// What a row is ranked by: its weight, and above every weight the rows that stay.
__device__ __forceinline__ uint32_t weight_key(float w, int pos, int keep_first, int64_t recent) {
    return pos < keep_first || pos > recent ? 0xFFFFFFFFu : sortable_key(w);
}

// One workgroup per (layer, sequence, KV head): exact radix select over the weights, four passes of eight bits, then the kept
// rows in ascending order with their weights and positions.  Every slot written is at or before the row it comes from, and later
// chunks read later rows only, so the weights and positions may be moved in place.
constexpr int kWeightThreads = 1024;
__global__ __launch_bounds__(kWeightThreads) void jq_weight_select_kernel(WeightArgs a) {
    __shared__ uint32_t hist[256];
    __shared__ uint32_t scan[kWeightThreads / 64];
    __shared__ uint32_t picked[2];
    const int g = blockIdx.x, s = blockIdx.y, layer = blockIdx.z, tid = threadIdx.x;
    const int cap = a.tab.cu_seq[s + 1] - a.tab.cu_seq[s];
    const int n = live_of(a.lens, a.tab.n_seq, layer, s, cap);
    const uint32_t B = budget_of(a.layer_budgets, a.tab, layer, s, a.keep_first + a.keep_last);
    const int64_t row0 = ((int64_t)layer * a.h_kv + g) * a.T + a.tab.cu_seq[s];
    const float* w = a.weights + row0;
    const int32_t* pos = a.pos ? a.pos + row0 : nullptr;
    int32_t* idx = a.idx + ((int64_t)layer * a.h_kv + g) * a.TB + a.tab.cu_bud[s];

    uint32_t tau = 0, ties = 0xFFFFFFFFu;  // every key above tau is kept, and the first `ties` rows of key tau
    int64_t recent = INT64_MAX;
    if ((uint32_t)n > B) {
        int newest = INT32_MIN;
        if (pos) {
            for (int j = tid; j < n; j += kWeightThreads) newest = max(newest, pos[j]);
            uint32_t top = wave_max((uint32_t)newest ^ 0x80000000u);
            if ((tid & 63) == 0) scan[tid >> 6] = top;
            __syncthreads();
            top = 0;
            for (int i = 0; i < kWeightThreads / 64; ++i) top = max(top, scan[i]);
            newest = (int)(top ^ 0x80000000u);
        } else {
            newest = n - 1;
        }
        recent = (int64_t)newest - a.keep_last;
        uint32_t left = B, prefix = 0, mask = 0;  // places left among the keys that agree with prefix under mask
        for (int shift = 24; shift >= 0; shift -= 8) {
            __syncthreads();
            if (tid < 256) hist[tid] = 0;
            __syncthreads();
            for (int j = tid; j < n; j += kWeightThreads) {
                const uint32_t k = weight_key(w[j], pos ? pos[j] : j, a.keep_first, recent);
                if ((k & mask) == prefix) atomicAdd(&hist[(k >> shift) & 255u], 1u);
            }
            __syncthreads();
            // bins from the largest down: the one in which the running count passes `left`
            const uint32_t c = tid < 256 ? hist[255 - tid] : 0u;
            uint32_t total;
            const uint32_t upto = block_scan_incl<kWeightThreads>(c, scan, &total);
            if (tid < 256 && upto >= left && upto - c < left) {
                picked[0] = 255 - tid;
                picked[1] = left - (upto - c);
            }
            __syncthreads();
            prefix |= picked[0] << shift;
            mask |= 255u << shift;
            left = picked[1];
        }
        tau = prefix;
        ties = left;
    }
    uint32_t kept = 0, equal = 0;  // before the present chunk
    for (int base = 0; base < n; base += kWeightThreads) {
        const int j = base + tid;
        const bool live = j < n;
        const float x = live ? w[j] : 0.0f;
        const int p = live ? (pos ? pos[j] : j) : 0;
        const uint32_t k = live ? weight_key(x, p, a.keep_first, recent) : 0u;
        const bool tie = live && k == tau;
        uint32_t n_tie, n_kept;
        const uint32_t tie_rank = equal + block_scan_incl<kWeightThreads>(tie ? 1u : 0u, scan, &n_tie);
        const bool keep = live && ((uint32_t)n <= B || k > tau || (tie && tie_rank <= ties));
        const uint32_t slot = kept + block_scan_incl<kWeightThreads>(keep ? 1u : 0u, scan, &n_kept) - 1;
        if (keep) {
            idx[slot] = j;
            a.weights_out[row0 + slot] = x;
            if (a.pos_out) a.pos_out[row0 + slot] = p;
        }
        kept += n_kept;
        equal += n_tie;
    }
}

// The kept rows of K and V, out of one cache into another: sixteen bytes a lane, sixteen lanes a row.
constexpr int kMoveThreads = 256;
__global__ __launch_bounds__(kMoveThreads) void jq_weight_copy_kernel(WeightArgs a) {
    const int64_t item = ((int64_t)blockIdx.x * kMoveThreads + threadIdx.x) / 16;  // (layer, kept row, head), heads fastest
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
// Columns have nothing to do with each other, so a (layer, sequence, head) is the work of eight workgroups.
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

// One workgroup per (layer, sequence, KV head): the row of least key (the lowest of equals) by a reduction, then the new row.
constexpr int kReplaceThreads = 256;
__global__ __launch_bounds__(kReplaceThreads) void jq_replace_kernel(ReplaceArgs a) {
    __shared__ uint64_t least[kReplaceThreads / 64];
    const int g = blockIdx.x, s = blockIdx.y, layer = blockIdx.z, tid = threadIdx.x;
    const int cap = a.tab.cu_seq[s + 1] - a.tab.cu_seq[s];
    const int n = live_of(a.lens, a.tab.n_seq, layer, s, cap);
    const int64_t row0 = ((int64_t)layer * a.h_kv + g) * a.T + a.tab.cu_seq[s];
    const int token = a.token[s];
    int slot = n;  // room left: the next row
    if (n == cap) {
        const int64_t recent = (int64_t)token - a.keep_last;  // the new token counts among the newest
        uint64_t best = UINT64_MAX;
        for (int j = tid; j < n; j += kReplaceThreads) {
            const uint64_t k = (uint64_t)weight_key(a.weights[row0 + j], a.pos[row0 + j], a.keep_first, recent) << 32 | (uint32_t)j;
            best = k < best ? k : best;
        }
        for (int d = 32; d; d >>= 1) {
            const uint64_t o = __shfl_xor((unsigned long long)best, d);
            best = o < best ? o : best;
        }
        if ((tid & 63) == 0) least[tid >> 6] = best;
        __syncthreads();
        for (int i = 0; i < kReplaceThreads / 64; ++i) best = least[i] < best ? least[i] : best;
        slot = (int)(uint32_t)best;
    }
    if (tid < 32) {  // sixteen lanes for the row of K, sixteen for V's
        const int part = tid & 15;
        const int64_t from = (((int64_t)layer * a.tab.n_seq + s) * a.h_kv + g) * (kHeadDim * 2) + part * 16;
        const int64_t to = (kv_row(a.pm, a.tab.cu_seq, a.T, layer, s, slot) * a.h_kv + g) * (kHeadDim * 2) + part * 16;
        *(wu32x4*)((tid < 16 ? a.K : a.V) + to) = *(const wu32x4*)((tid < 16 ? a.k_new : a.v_new) + from);
    }
    if (tid == 0) {
        a.weights[row0 + slot] = 0.0f;
        a.pos[row0 + slot] = token;
        if (a.slot) a.slot[((int64_t)layer * a.tab.n_seq + s) * a.h_kv + g] = slot;
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------------

hipError_t launch_evict_weight(const Plan& p, const int32_t* lens, const void* K, const void* V, const float* weights, const int32_t* pos,
                               void* K_out, void* V_out, float* weights_out, int32_t* pos_out, int32_t* idx, hipStream_t st) {
    WeightArgs a{};
    a.K = (const char*)K; a.V = (const char*)V; a.K_out = (char*)K_out; a.V_out = (char*)V_out;
    a.weights = weights; a.weights_out = weights_out; a.pos = pos; a.pos_out = pos_out; a.lens = lens; a.idx = idx;
    a.layer_budgets = p.layer_budgets;
    a.n_layers = p.n_layers; a.h_kv = p.h_kv; a.keep_first = p.keep_first; a.keep_last = p.keep_last;
    a.T = p.T; a.TB = p.TB; a.pm = p.page_map(); a.tab = p.tab;
    hipError_t e = launch_kernel(jq_weight_select_kernel, dim3((unsigned)p.h_kv, (unsigned)p.n_seq, (unsigned)p.n_layers), dim3(kWeightThreads), 0, st,
                                 nullptr, -1, a);
    if (e != hipSuccess) return e;
    if (K_out == K)
        return launch_kernel(jq_weight_shift_kernel, dim3((unsigned)(8 * p.h_kv), (unsigned)p.n_seq, (unsigned)p.n_layers), dim3(kMoveThreads), 0, st, nullptr, -1, a);
    const int64_t threads = (int64_t)p.n_layers * p.TB * p.h_kv * 16;
    return launch_kernel(jq_weight_copy_kernel, dim3((unsigned)((threads + kMoveThreads - 1) / kMoveThreads)), dim3(kMoveThreads), 0, st, nullptr, -1, a);
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
