// Attention of sequences that continue shared prefixes: several answers to one (pruned) prompt, say.
//
//   out = sum_j p_j v[j] over the rows of a sequence's prefix and its own, p normalised over both
//
// A prefix is swept once for all the sequences that continue it: their query rows, which each would have brought alone, meet its keys
// together, as many query rows of one sequence do in jq_attend (jq_attend.h has both sweeps).  The sequences' own rows are swept in the
// same launch, by other workgroups or behind the prefixes, and a second launch joins the parts (m, z, unnormalised out) of both.
// Measured on one MI355X, whole calls, 8 KV heads of 4 query heads: 8 sequences of 40 rows behind 2048 rows 15.3 us (two launches, 12
// and 4), 32 of 700 behind 32768 62 (the sweeps 57, one behind the other; 17 MB of parts; the join 7.7), 16 of 500 behind 131072 119 (memory: 4.7
// TB/s over the sweeps).
#include <algorithm>

#include "jq_attend.h"

namespace jq {

struct SharedArgs {
    PrefixArgs prefix;
    OwnArgs own;
    int32_t prefix_blocks, own_blocks;  // shares of either sweep; a workgroup may take one of each
};
static_assert(sizeof(SharedArgs) <= 4096, "a kernel's arguments");
static_assert(kSharedJoinThreads == kAttendThreads, "what the plan counts");

// P: tiles of 16 query rows of a prefix that a workgroup takes, RT: of a sequence.
template <class Rows, int P, int RT>
__global__ __launch_bounds__(kSharedThreads, 2) void jq_attend_shared_kernel(SharedArgs) {
    const SharedArgs& a = kernel_args<SharedArgs>();
    const int bx = (int)blockIdx.x, grid = (int)gridDim.x;
    if (bx < a.prefix_blocks) {
        if constexpr (P <= 2) attend_few_rows<Rows, P, kSeeAll, false, kSharedWaves>(a.prefix, bx, (int)blockIdx.y);
        else attend_many_rows<Rows, P / 2, kSeeAll, false>(a.prefix, bx, (int)blockIdx.y);
    }
    for (int u = first_own(bx, a.prefix_blocks, grid); u < a.own_blocks; u += grid) {
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
    a.prefix_blocks = sp.prefix_blocks;
    a.own_blocks = sp.own_blocks;
    const dim3 grid((unsigned)sp.grid, (unsigned)p.n_layers);
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
