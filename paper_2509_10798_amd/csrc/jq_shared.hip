// Attention of sequences that continue shared prefixes: several answers to one (pruned) prompt, say.
//
//   out = sum_j p_j v[j] over the rows of a sequence's prefix and its own, p normalised over both
//
// A prefix is swept once for all the sequences that continue it: their query rows, which each would have brought alone, meet its keys
// together, as many query rows of one sequence do in jq_attend (jq_attend.h has both sweeps).  The sequences' own rows are swept by
// other workgroups of the same launch, and a second launch joins the parts (m, z, unnormalised out) of both.
#include <algorithm>

#include "jq_attend.h"

namespace jq {

constexpr int kSharedWaves = 8, kSharedThreads = 64 * kSharedWaves;

struct SharedArgs {
    PrefixArgs prefix;
    OwnArgs own;
    int32_t prefix_blocks;
};

// P: tiles of 16 query rows of a prefix that a workgroup takes, RT: of a sequence.
template <class Rows, int P, int RT>
__global__ __launch_bounds__(kSharedThreads, 2) void jq_attend_shared_kernel(SharedArgs) {
    const SharedArgs& a = kernel_args<SharedArgs>();
    const int bx = (int)blockIdx.x;
    if (bx < a.prefix_blocks) {
        if constexpr (P <= 2) attend_few_rows<Rows, P, kSeeAll, false, kSharedWaves>(a.prefix, bx, (int)blockIdx.y);
        else attend_many_rows<Rows, P / 2, kSeeAll, false>(a.prefix, bx, (int)blockIdx.y);
    } else {
        attend_few_rows<Rows, RT, kSeeCausal, false, kSharedWaves>(a.own, bx - a.prefix_blocks, (int)blockIdx.y);
    }
}

// A wave joins the parts of one (layer, sequence, KV head, query row).
__global__ __launch_bounds__(kAttendThreads) void jq_attend_shared_join_kernel(SharedArgs) {
    const SharedArgs& a = kernel_args<SharedArgs>();
    const OwnArgs& own = a.own;
    const PrefixArgs& pre = a.prefix;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), layer = blockIdx.y;
    const int item = (int)blockIdx.x * kAttendWaves + wave;
    if (item >= own.n_seq * own.h_kv * own.rows) return;
    const int unit = item / own.rows, row = item - unit * own.rows, s = unit / own.h_kv, g = unit - s * own.h_kv;
    int p = 0;  // the sequence's prefix
    if (pre.n_seq > 1) {
        p = __popcll(__ballot(lane + 1 < pre.n_seq && pre.cu_member[min(lane + 1, pre.n_seq)] <= s));
        if (pre.n_seq > 64) p += __popcll(__ballot(lane + 65 < pre.n_seq && pre.cu_member[min(lane + 65, pre.n_seq)] <= s));
    }
    const int n_own = own.cu_split[s + 1] - own.cu_split[s], n = n_own + pre.cu_split[p + 1] - pre.cu_split[p];
    const int64_t own_at = part_at(own, layer, s, own.cu_split[s], 0, g) + row, own_step = (int64_t)own.h_kv * own.rows;
    const int64_t pre_at = part_at(pre, layer, p, 0, 0, g) + (s - pre.cu_member[p]) * own.rows + row, pre_step = (int64_t)own.h_kv * query_rows(pre, p);
    auto stat = [&](int i) { return i < n_own ? own.stats[own_at + i * own_step] : pre.stats[pre_at + (i - n_own) * pre_step]; };
    // two parts at a time, 16 bytes a lane; the first sixteen are requested ahead of the statistics
    const int half = lane >> 5, d = (lane & 31) * 4;
    auto part = [&](int i) {
        const float* from = i < n_own ? own.part + (own_at + i * own_step) * kHeadDim : pre.part + (pre_at + (i - n_own) * pre_step) * kHeadDim;
        return *(const f32x4*)(from + d);
    };
    constexpr int kBatch = 8;
    f32x4 x[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) x[k] = part(min(half + 2 * k, n - 1));
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
    for (int i0 = 0; i0 < n; i0 += 2 * kBatch) {
        if (i0)
#pragma unroll
            for (int k = 0; k < kBatch; ++k) x[k] = part(min(i0 + half + 2 * k, n - 1));
#pragma unroll
        for (int k = 0; k < kBatch; ++k) {
            const int i = i0 + half + 2 * k;
            float f = __shfl(factor, i & 63);
            if (i >= 64) f = rescale(stat(min(i, n - 1)).x, m);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += i < n ? x[k][e] * f : 0.0f;  // (nothing times 0: a sum may be infinite)
        }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], 32);
    if (lane < 32) store_out(own, layer, s, g, row, d, o, m, z);
}

// ---- host ------------------------------------------------------------------------------------------------------------------

constexpr int kSharedChip = 256;  // workgroups that run at a time, one a CU

// How the work is shared out: every prefix and every sequence in shares of at most so many rows, one size for all of them.
void plan_shared(const Plan& p, const Plan& pp, const int32_t* cu_members, SharedPlan* sp) {
    int32_t most_rows = 0;
    for (int i = 0; i < pp.n_seq; ++i) most_rows = std::max(most_rows, (cu_members[i + 1] - cu_members[i]) * p.rows);
    const int tiles = (most_rows + kTileRows - 1) / kTileRows;
    sp->prefix_tiles = tiles <= 1 ? 1 : tiles <= 2 ? 2 : tiles <= 4 ? 4 : tiles <= 8 ? 8 : 16;
    sp->prefix_groups = (tiles + sp->prefix_tiles - 1) / sp->prefix_tiles;
    const int own_tiles = (p.rows + kTileRows - 1) / kTileRows;
    sp->own_tiles = own_tiles <= 1 ? 1 : 2;
    sp->own_groups = (own_tiles + sp->own_tiles - 1) / sp->own_tiles;
    const int64_t heads = (int64_t)p.n_layers * p.h_kv, unit = 256, start = 512;
    auto length = [](const Plan& q, int s) { return (int64_t)q.tab.cu_seq[s + 1] - q.tab.cu_seq[s]; };
    auto groups = [&](int i) { return ((cu_members[i + 1] - cu_members[i]) * p.rows + sp->prefix_tiles * kTileRows - 1) / (sp->prefix_tiles * kTileRows); };
    int64_t total = 0;
    for (int i = 0; i < pp.n_seq; ++i) total += length(pp, i) * heads * groups(i);
    for (int s = 0; s < p.n_seq; ++s) total += length(p, s) * heads * sp->own_groups;
    // from four rounds of the chip to half of one
    int64_t best = INT64_MAX, share = 1;
    const int64_t even = total / (kSharedChip * unit);
    for (int64_t c = even / 4 + 1; c <= 2 * even + 2; c += 1 + c / 8) {
        const uint32_t size = (uint32_t)std::min(c * unit, (int64_t)INT32_MAX);
        int64_t n = 0, all = 0, largest = 0, last = 0;
        auto add = [&](int64_t rows, int64_t times) {
            const uint32_t k = ((uint32_t)rows + size - 1) / size;
            last = ((uint32_t)rows + k - 1) / k + start;
            n += k * times;
            all += k * times * last;
            largest = std::max(largest, last);
        };
        for (int i = 0; i < pp.n_seq; ++i) add(length(pp, i), heads * groups(i));
        for (int s = 0; s < p.n_seq; ++s) add(length(p, s), heads * sp->own_groups);
        const int64_t cost = n <= kSharedChip ? largest : std::max(largest, all / kSharedChip + last / 2);
        if (cost < best) { best = cost; share = c; }
    }
    const int64_t size = share * unit;
    sp->cu_split[0] = sp->cu_part[0] = sp->own_split[0] = 0;
    int64_t parts = 0;
    for (int i = 0; i < pp.n_seq; ++i) {
        const int64_t ns = (length(pp, i) + size - 1) / size;
        sp->cu_split[i + 1] = sp->cu_split[i] + (int32_t)ns;
        parts += ns * (cu_members[i + 1] - cu_members[i]) * p.rows;
        sp->cu_part[i + 1] = (int32_t)parts;
    }
    for (int s = 0; s < p.n_seq; ++s) sp->own_split[s + 1] = sp->own_split[s] + (int32_t)((length(p, s) + size - 1) / size);
    sp->fits = parts <= INT32_MAX;
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    const size_t pre = (size_t)heads * (size_t)parts, own = (size_t)heads * sp->own_split[p.n_seq] * p.rows;
    sp->off_prefix_stats = 0;
    sp->off_prefix_part = up(pre * sizeof(float2));
    sp->off_own_stats = sp->off_prefix_part + up(pre * kHeadDim * sizeof(float));
    sp->off_own_part = sp->off_own_stats + up(own * sizeof(float2));
    sp->ws_bytes = sp->off_own_part + up(own * kHeadDim * sizeof(float));
    const int64_t blocks = shared_blocks(sp->cu_split[pp.n_seq], p.h_kv, sp->prefix_groups) + shared_blocks(sp->own_split[p.n_seq], p.h_kv, sp->own_groups);
    const int64_t joins = ((int64_t)p.n_seq * p.h_kv * p.rows + kAttendWaves - 1) / kAttendWaves;
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
    a.prefix.row_groups = sp.prefix_groups; a.own.row_groups = sp.own_groups;
    a.prefix.n_splits = sp.cu_split[pp.n_seq]; a.own.n_splits = sp.own_split[p.n_seq];
    a.prefix.units = a.prefix.n_splits * p.h_kv; a.own.units = a.own.n_splits * p.h_kv;
    for (int i = 0; i <= pp.n_seq; ++i) { a.prefix.cu_split[i] = sp.cu_split[i]; a.prefix.cu_part[i] = sp.cu_part[i]; a.prefix.cu_member[i] = cu_members[i]; }
    for (int s = 0; s <= p.n_seq; ++s) a.own.cu_split[s] = sp.own_split[s];
    a.own.causal = p.window && p.n_q > 1;
    a.prefix_blocks = (int32_t)shared_blocks(a.prefix.n_splits, p.h_kv, sp.prefix_groups);
    const dim3 grid((unsigned)(a.prefix_blocks + shared_blocks(a.own.n_splits, p.h_kv, sp.own_groups)), (unsigned)p.n_layers);
    hipError_t e;
    switch (sp.prefix_tiles) {
        case 1: e = launch_shared_sweep<1>(a, sp.own_tiles, grid, st); break;
        case 2: e = launch_shared_sweep<2>(a, sp.own_tiles, grid, st); break;
        case 4: e = launch_shared_sweep<4>(a, sp.own_tiles, grid, st); break;
        case 8: e = launch_shared_sweep<8>(a, sp.own_tiles, grid, st); break;
        default: e = launch_shared_sweep<16>(a, sp.own_tiles, grid, st); break;
    }
    if (e != hipSuccess) return e;
    const int64_t joins = ((int64_t)p.n_seq * p.h_kv * p.rows + kAttendWaves - 1) / kAttendWaves;
    return launch_kernel(jq_attend_shared_join_kernel, dim3((unsigned)joins, (unsigned)p.n_layers), dim3(kAttendThreads), 0, st, nullptr, -1, a);
}

}  // namespace jq
