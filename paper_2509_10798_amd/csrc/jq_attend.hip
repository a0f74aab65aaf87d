// Attention over a cache: what joins the shares of a sequence, how the work is shared out, and the launches (jq_attend.h holds the
// sweeps).
#include "jq_codes.h"

namespace jq {

// (their kernels are compiled in files of their own)
extern template hipError_t launch_sweeps<RowsCoded<8, 8>>(const AttendArgs&, int, int, bool, dim3, hipStream_t);
extern template hipError_t launch_sweeps<RowsCoded<8, 4>>(const AttendArgs&, int, int, bool, dim3, hipStream_t);
extern template hipError_t launch_sweeps<RowsCoded<4, 4>>(const AttendArgs&, int, int, bool, dim3, hipStream_t);

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
    Weigher<kAttendThreads>(a, layer, s, g, b * kWeighKeys, min((b + 1) * kWeighKeys, n)).add(lse2, false);
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
// Over codes smaller shares are also looked for where whole sequences would do, for ragged ones (us, one round / up to four, 8 KV heads: 31
// sequences of 306 to 14833 rows, 8 bits, two causal tokens 100 / 63, of 313 to 15234 rows, 31 tokens 240 / 108; 4 bits, 344 to
// 10543 rows 59 / 38).
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
// `waves` of a workgroup that takes 32 or fewer query rows; shares of multiples of `step` rows of the cache.
static void plan_splits(const Plan& p, bool weights, bool coded, int waves, int64_t step, AttendPlan* ap) {
    const int row_tiles = (p.rows + kTileRows - 1) / kTileRows;
    ap->row_tiles = row_tiles <= 1 ? 1 : row_tiles <= 2 ? 2 : row_tiles <= 4 ? 4 : row_tiles <= 8 ? 8 : 16;
    ap->row_groups = (row_tiles + ap->row_tiles - 1) / ap->row_tiles;
    // Shares are counted in what a workgroup takes at a time; workgroups left over go to the sequences with the largest.
    const int64_t heads = (int64_t)p.n_layers * p.h_kv * ap->row_groups, unit = ap->row_tiles > 4 ? 64 : step;
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
    const int64_t start = ap->row_tiles > 2 ? kWideStart : (coded ? 2 : 1) * kStart;  // (rows of codes take half as long)
    for (int rounds = 1; rounds <= (p.n_seq * heads > kChip || (coded && p.n_seq > 1) ? kRounds : 1); ++rounds) {
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
        tiles = std::max(tiles, ((L + 31) / 32 + waves * ns[s] - 1) / (waves * ns[s]));  // of 32 keys, a wave
    }
    ap->waves = waves;
    ap->most_rows = (int32_t)std::min<int64_t>(share * unit, INT32_MAX);
    ap->hold_keys = weights && row_tiles <= 2 ? (int32_t)(tiles * 32 * waves) : 0;
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

static void plan_attend(const Plan& p, bool weights, bool coded, int waves, int64_t step, AttendPlan* ap) {
    plan_splits(p, weights, coded, waves, step, ap);
    const size_t parts = (size_t)p.n_layers * ap->cu_split[p.n_seq] * p.h_kv * p.rows;
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    ap->logit_T = 32 * (p.T / 32 + p.n_seq);
    ap->off_arrived = 0;
    ap->off_stats = up((size_t)p.n_layers * p.n_seq * p.h_kv * ap->row_groups * sizeof(uint64_t));
    ap->off_part = ap->off_stats + up(parts * sizeof(float2));
    ap->off_logits = ap->off_part + up(parts * kHeadDim * sizeof(float));
    ap->ws_bytes = ap->off_logits + (weights ? up((size_t)p.n_layers * p.h_kv * p.rows * ap->logit_T * sizeof(float)) : 0);
}

// Over codes a workgroup that takes 32 or fewer query rows has eight waves (RowsCoded::waves says why), but four where it takes 16 or fewer
// and its share is two tiles a wave of four or less: such a call is its start and its join, which take longer with eight.  Us of the kernel,
// four / eight waves, 8 KV heads of 4 query rows in 8 bits: one token over 1000 rows 9.7 / 11.2, 2000 10.4 / 11.4, 8 x 1024 11.7 / 12.4, 8192
// (shares of 256) 8.4 / 8.5, 12288 (384) 10.2 / 9.6, 16384 (512) 12.2 / 10.5; 1000 rows of 2 heads with weights 11.1 / 13.5.  (The wide sweeps
// have eight waves whatever the cache, over 128 or 64 keys together: Wide.)
constexpr int kShortShare = 256;
void plan_attend(const Plan& p, bool weights, bool coded, AttendPlan* ap) {
    plan_attend(p, weights, coded, kAttendWaves, 32 * kAttendWaves, ap);
    const int waves = coded && ap->row_tiles <= 2 ? RowsCoded<8, 8>::waves(ap->row_tiles, weights) : kAttendWaves;
    if (waves == kAttendWaves || (ap->row_tiles == 1 && ap->most_rows <= kShortShare)) return;
    plan_attend(p, weights, coded, waves, 32 * waves, ap);
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
    return sweep_groups(p, ap) * (ap.row_tiles > 2 ? 512 : 64 * ap.waves) <= UINT32_MAX && finish_groups(p, ap, weights).groups * kAttendThreads <= UINT32_MAX;
}

hipError_t launch_attend(const Plan& p, const AttendPlan& ap, const int32_t* lens, const uint32_t* seen, const void* Q, const void* K, const void* V,
                         void* out, float* lse, float* weights, char* ws, hipStream_t st, const Codes* codes) {
    AttendArgs a{};
    a.Q = (const char*)Q; a.K = (const char*)(codes ? codes->K : K); a.V = (const char*)(codes ? codes->V : V);
    if (codes) { a.K_scale = (const uint8_t*)codes->K_scale; a.V_scale = (const uint8_t*)codes->V_scale; }
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
    const dim3 grid((unsigned)sweep_groups(p, ap), (unsigned)p.n_layers);
    const bool causal = p.window && p.n_q > 1;
    const hipError_t e = !codes            ? launch_sweeps<Rows16>(a, ap.row_tiles, ap.waves, causal, grid, st)
                         : codes->k_bits == 4 ? launch_sweeps<RowsCoded<4, 4>>(a, ap.row_tiles, ap.waves, causal, grid, st)
                         : codes->v_bits == 4 ? launch_sweeps<RowsCoded<8, 4>>(a, ap.row_tiles, ap.waves, causal, grid, st)
                                              : launch_sweeps<RowsCoded<8, 8>>(a, ap.row_tiles, ap.waves, causal, grid, st);
    if (e != hipSuccess) return e;
    const Finish f = finish_groups(p, ap, weights != nullptr);
    if (f.groups == 0) return e;
    return launch_kernel(jq_attend_finish_kernel, dim3((unsigned)f.groups, (unsigned)p.n_layers), dim3(kAttendThreads), 0, st, nullptr, -1, a, (int)f.joins,
                         (int)f.blocks);
}

}  // namespace jq
