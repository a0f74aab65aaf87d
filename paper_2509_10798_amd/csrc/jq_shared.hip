// Attention of sequences that continue shared prefixes: several answers to one (pruned) prompt, say.
//
//   out = sum_j p_j v[j] over the rows of a sequence's prefix and its own, p normalised over both
//
// A prefix is swept once for all the sequences that continue it: their query rows, which each would have brought alone, meet its keys
// together, as many query rows of one sequence do in jq_attend (jq_attend.h has both sweeps).  The sequences' own rows are swept in the
// same launch, by other workgroups or behind the prefixes, and a second launch joins the parts (m, z, unnormalised out) of both.
// Measured on one MI355X, whole calls, 8 KV heads of 4 query heads: 8 sequences of 40 rows behind 2048 rows 15.4 us (two launches, 11.9
// and 4), 32 of 700 behind 32768 58 (the sweeps 52, one behind the other; 17 MB of parts; the join 7.7), 16 of 500 behind 131072 119 (memory: 4.7
// TB/s over the sweeps).
#include <algorithm>

#include "jq_attend.h"

namespace jq {

constexpr int kSharedWaves = 8, kSharedThreads = 64 * kSharedWaves;

struct SharedArgs {
    PrefixArgs prefix;
    OwnArgs own;
    int32_t prefix_blocks, own_blocks;  // shares of either sweep; a workgroup may take one of each
};
static_assert(sizeof(SharedArgs) <= 4096, "a kernel's arguments");

// P: tiles of 16 query rows of a prefix that a workgroup takes, RT: of a sequence.
template <class Rows, int P, int RT>
__global__ __launch_bounds__(kSharedThreads, 2) void jq_attend_shared_kernel(SharedArgs) {
    const SharedArgs& a = kernel_args<SharedArgs>();
    const int bx = (int)blockIdx.x, grid = (int)gridDim.x;
    if (bx < a.prefix_blocks) {
        if constexpr (P <= 2) attend_few_rows<Rows, P, kSeeAll, false, kSharedWaves>(a.prefix, bx, (int)blockIdx.y);
        else attend_many_rows<Rows, P / 2, kSeeAll, false>(a.prefix, bx, (int)blockIdx.y);
    }
    // Shares of the sequences go to the workgroups that have none of a prefix, then around.
    for (int u = bx - a.prefix_blocks + (bx < a.prefix_blocks ? grid : 0); u < a.own_blocks; u += grid) {
        __syncthreads();  // (LDS: what the sums before lie in)
        attend_few_rows<Rows, RT, kSeeCausal, false, kSharedWaves>(a.own, u, (int)blockIdx.y);
    }
}

// A workgroup joins the parts of one (layer, sequence, KV head, query row): each of its waves every fourth, two at a time, all of them
// requested together ahead of the statistics (up to 64 parts; one wave a row, in turns of sixteen parts, took 2 us more).
constexpr int kJoinBatch = 8;
__global__ __launch_bounds__(kAttendThreads) void jq_attend_shared_join_kernel(SharedArgs) {
    __shared__ __align__(16) float sums[kAttendWaves][kHeadDim];
    const SharedArgs& a = kernel_args<SharedArgs>();
    const OwnArgs& own = a.own;
    const PrefixArgs& pre = a.prefix;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), layer = blockIdx.y;
    const int unit = (int)blockIdx.x / own.rows, row = (int)blockIdx.x - unit * own.rows, s = unit / own.h_kv, g = unit - s * own.h_kv;
    int p = 0;  // the sequence's prefix
    if (pre.n_seq > 1) {
        p = __popcll(__ballot(lane + 1 < pre.n_seq && pre.cu_member[min(lane + 1, pre.n_seq)] <= s));
        if (pre.n_seq > 64) p += __popcll(__ballot(lane + 65 < pre.n_seq && pre.cu_member[min(lane + 65, pre.n_seq)] <= s));
    }
    const int n_own = own.cu_split[s + 1] - own.cu_split[s], n = n_own + (pre.cu_part[p + 1] - pre.cu_part[p]) / query_rows(pre, p);
    const int64_t own_at = part_at(own, layer, s, own.cu_split[s], 0, g) + row, own_step = (int64_t)own.h_kv * own.rows;
    const int64_t pre_at = part_at(pre, layer, p, 0, 0, g) + (s - pre.cu_member[p]) * own.rows + row, pre_step = (int64_t)own.h_kv * query_rows(pre, p);
    auto stat = [&](int i) { return i < n_own ? own.stats[own_at + i * own_step] : pre.stats[pre_at + (i - n_own) * pre_step]; };
    const int d = (lane & 31) * 4;
    auto part = [&](int i) {
        const float* from = i < n_own ? own.part + (own_at + i * own_step) * kHeadDim : pre.part + (pre_at + (i - n_own) * pre_step) * kHeadDim;
        return *(const f32x4*)(from + d);
    };
    const int first = 2 * wave + (lane >> 5);  // the lane's parts: first, first + 8, ..
    constexpr int kStep = 2 * kAttendWaves;
    f32x4 x[kJoinBatch];
#pragma unroll
    for (int k = 0; k < kJoinBatch; ++k)
        if (kStep * k < n) x[k] = part(min(first + kStep * k, n - 1));
    const float2 mine = lane < n ? stat(lane) : make_float2(-__builtin_inff(), 0.0f);
    float m = mine.x;
    for (int i = lane + 64; i < n; i += 64) m = fmaxf(m, stat(i).x);
#pragma unroll
    for (int k = 32; k; k >>= 1) m = fmaxf(m, __shfl_xor(m, k));
    const float factor = rescale(mine.x, m);
    float z = mine.y * factor;
    for (int i = lane + 64; i < n; i += 64) {
        const float2 mz = stat(i);
        z += mz.y * rescale(mz.x, m);
    }
#pragma unroll
    for (int k = 32; k; k >>= 1) z += __shfl_xor(z, k);
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int i0 = 0; i0 < n; i0 += kStep * kJoinBatch) {
#pragma unroll
        for (int k = 0; k < kJoinBatch; ++k) {
            const int i = i0 + first + kStep * k;
            if (i0 + kStep * k >= n) break;
            if (i0) x[k] = part(min(i, n - 1));
            float f = __shfl(factor, i & 63);
            if (i >= 64) f = rescale(stat(min(i, n - 1)).x, m);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += i < n ? x[k][e] * f : 0.0f;  // (nothing times 0: a sum may be infinite)
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], 32);
    if (lane < 32) *(f32x4*)(sums[wave] + d) = o;
    __syncthreads();
    if (threadIdx.x >= 32) return;
    o = *(const f32x4*)(sums[0] + d);
#pragma unroll
    for (int w = 1; w < kAttendWaves; ++w) o += *(const f32x4*)(sums[w] + d);
    store_out(own, layer, s, g, row, d, o, m, z);
}

// ---- host ------------------------------------------------------------------------------------------------------------------

constexpr int kSharedChip = 256;  // workgroups that run at a time, one a CU

// How the work is shared out.  Prefixes and sequences are cut into shares, either side by side, on CUs of their own, or, where there is
// much of both, one behind the other on all of them: what a CU reads in a given time is limited, some 25 GB/s, however many of its
// waves ask, so a sweep that has few CUs takes long.  Fewer shares leave fewer parts to write and to join; fewer query rows a workgroup
// (and the prefix read twice, which meets in an XCD's L2) halve them too.  In nanoseconds, as measured on one MI355X.
constexpr int64_t kSharedStart = 6000, kSharedNext = 3000, kOwnRow = 22, kPartBytes = 4000;  // (the last: bytes a nanosecond, there and back)
static int64_t prefix_row_time(int tiles) { return tiles <= 8 ? 25 : 36; }
void plan_shared(const Plan& p, const Plan& pp, const int32_t* cu_members, SharedPlan* sp) {
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
    int64_t parts = 0, eighths = 0;
    for (int i = 0; i < pp.n_seq; ++i) {
        const int64_t ns = split(length[i], share);
        const int64_t groups = (rows[i] + sp->prefix_tiles * kTileRows - 1) / (sp->prefix_tiles * kTileRows);
        eighths += (ns * p.h_kv + 7) / 8 * groups;
        if (i == 0) { sp->first_groups = (int32_t)groups; sp->first_splits = (int32_t)ns; }
        sp->cu_split[i + 1] = (int32_t)eighths;
        parts += ns * rows[i];
        sp->cu_part[i + 1] = (int32_t)parts;
    }
    for (int s = 0; s < p.n_seq; ++s) sp->own_split[s + 1] = sp->own_split[s] + (int32_t)split(own_length[s], own_share);
    sp->fits = parts <= INT32_MAX && eighths <= INT32_MAX / 8;
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    const size_t pre = (size_t)heads * (size_t)parts, own = (size_t)heads * sp->own_split[p.n_seq] * p.rows;
    sp->off_prefix_stats = 0;
    sp->off_prefix_part = up(pre * sizeof(float2));
    sp->off_own_stats = sp->off_prefix_part + up(pre * kHeadDim * sizeof(float));
    sp->off_own_part = sp->off_own_stats + up(own * sizeof(float2));
    sp->ws_bytes = sp->off_own_part + up(own * kHeadDim * sizeof(float));
    const int64_t blocks = 8 * eighths + shared_blocks(sp->own_split[p.n_seq], p.h_kv, sp->own_groups);
    const int64_t joins = (int64_t)p.n_seq * p.h_kv * p.rows;
    sp->fits = sp->fits && blocks * kSharedThreads <= UINT32_MAX && joins * kAttendThreads <= UINT32_MAX;
}

static void common_args(const Plan& p, AttendArgs* a) {
    a->n_layers = p.n_layers; a->n_seq = p.n_seq; a->h_kv = p.h_kv;
    a->T = p.T;
    a->pm = p.page_map();
    for (int s = 0; s <= p.n_seq; ++s) a->cu_seq[s] = p.tab.cu_seq[s];
}

template <int P>
static hipError_t launch_shared_sweep(const SharedArgs& a, int own_tiles, dim3 grid, hipStream_t st) {
    constexpr int few1 = kSharedWaves * kTileRows * (kOutStride * 4 + 8), few2 = 2 * few1;
    constexpr int mine = P == 1 ? few1 : P == 2 ? few2 : Wide<P <= 2 ? 2 : P / 2>::kLds;
    auto go = [&](auto kernel, int lds, std::atomic<uint64_t>& done) {
        const hipError_t e = allow_dynamic_lds((const void*)kernel, lds, done);
        return e != hipSuccess ? e : launch_kernel(kernel, grid, dim3(kSharedThreads), lds, st, nullptr, -1, a);
    };
    static std::atomic<uint64_t> done1{0}, done2{0};
    if (own_tiles == 1) return go(jq_attend_shared_kernel<Rows16, P, 1>, std::max(mine, few1), done1);
    return go(jq_attend_shared_kernel<Rows16, P, 2>, std::max(mine, few2), done2);
}

hipError_t launch_attend_shared(const Plan& p, const Plan& pp, const SharedPlan& sp, const int32_t* cu_members, const int32_t* lens, const int32_t* prefix_lens,
                                const void* Q, const void* K_prefix, const void* V_prefix, const void* K, const void* V, void* out, float* lse, char* ws,
                                hipStream_t st) {
    SharedArgs a{};
    common_args(p, &a.own);
    common_args(pp, &a.prefix);
    AttendArgs* both[2] = {&a.prefix, &a.own};
    for (AttendArgs* x : both) {
        x->Q = (const char*)Q;
        x->n_q = p.n_q; x->h_q = p.h_q; x->group = p.group;
        x->scale2 = (float)(p.scale * 1.4426950408889634);
        x->out = (uint16_t*)out; x->lse = lse;
    }
    a.prefix.K = (const char*)K_prefix; a.prefix.V = (const char*)V_prefix; a.prefix.lens = prefix_lens;
    a.own.K = (const char*)K; a.own.V = (const char*)V; a.own.lens = lens;
    a.prefix.stats = (float2*)(ws + sp.off_prefix_stats); a.prefix.part = (float*)(ws + sp.off_prefix_part);
    a.own.stats = (float2*)(ws + sp.off_own_stats); a.own.part = (float*)(ws + sp.off_own_part);
    a.own.rows = p.rows;
    a.prefix.row_groups = sp.first_groups; a.prefix.n_splits = sp.first_splits;
    a.own.row_groups = sp.own_groups;
    a.own.n_splits = sp.own_split[p.n_seq];
    a.own.units = a.own.n_splits * p.h_kv;
    for (int i = 0; i <= pp.n_seq; ++i) { a.prefix.cu_split[i] = sp.cu_split[i]; a.prefix.cu_part[i] = sp.cu_part[i]; a.prefix.cu_member[i] = cu_members[i]; }
    for (int s = 0; s <= p.n_seq; ++s) a.own.cu_split[s] = sp.own_split[s];
    a.own.causal = p.window && p.n_q > 1;
    a.prefix_blocks = 8 * sp.cu_split[pp.n_seq];
    a.own_blocks = (int32_t)shared_blocks(a.own.n_splits, p.h_kv, sp.own_groups);
    // more than the CUs take at a time, with layers on top: all in one round of workgroups if the prefixes are
    const int64_t all = (int64_t)a.prefix_blocks + a.own_blocks, most = std::max<int64_t>(kSharedChip / p.n_layers, 1);
    const dim3 grid((unsigned)(all <= most || a.prefix_blocks > most ? all : most), (unsigned)p.n_layers);
    hipError_t e;
    switch (sp.prefix_tiles) {
        case 1: e = launch_shared_sweep<1>(a, sp.own_tiles, grid, st); break;
        case 2: e = launch_shared_sweep<2>(a, sp.own_tiles, grid, st); break;
        case 4: e = launch_shared_sweep<4>(a, sp.own_tiles, grid, st); break;
        case 8: e = launch_shared_sweep<8>(a, sp.own_tiles, grid, st); break;
        default: e = launch_shared_sweep<16>(a, sp.own_tiles, grid, st); break;
    }
    if (e != hipSuccess) return e;
    const int64_t joins = (int64_t)p.n_seq * p.h_kv * p.rows;
    return launch_kernel(jq_attend_shared_join_kernel, dim3((unsigned)joins, (unsigned)p.n_layers), dim3(kAttendThreads), 0, st, nullptr, -1, a);
}

}  // namespace jq
