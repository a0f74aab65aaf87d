// Rows written into a cache of codes, and read back (jq_codes.h says what the codes are).
//
// Both kernels are bound by memory: 512 bytes of bf16 rows against 264 (K and V in 8 bits) or 136 (in 4) of codes and scales, a
// (row, KV head).  Sixteen lanes take a row, eight dimensions each, so that four of them hold a group and its largest value is found
// within a DPP quad.  A workgroup takes 64 rows of one head, of K and of V: what it writes of codes lies in one piece, and all its loads are
// under way together.  Nothing is read or written twice, so rows go past the caches in both directions, and codes on their way out;
// workgroups lie by head first.  Us of the two kernels for 32 layers of 2048 rows of 8 heads in 8 bits, 406 MB each: 71 and 73 (5.6 TB/s); through
// the caches 91 and 69; the heads of a row side by side 76 and 77.  12 ragged sequences of 48605 rows in pages of 64 rows, V in 4 bits, 277 MB:
// 60 and 62 (4.5 TB/s; four bytes a lane of V's codes).
#include "jq_codes.h"

namespace jq {

constexpr int kCodeThreads = 256, kCodeRows = 64, kCodePasses = kCodeRows / (kCodeThreads / 16);

struct CodeArgs {
    const char* K_in; const char* V_in;  // written from, or
    char* K_out; char* V_out;            // read back into: bf16 [n_layers][TB][h_kv][128]
    char* K; char* V;                    // codes
    uint8_t* K_scale; uint8_t* V_scale;
    const int32_t* first;                // DEVICE [n_layers][n_seq] row of the cache that a sequence's first row is, or null: 0
    const int32_t* layer_budgets;
    int32_t h_kv, blocks;                // blocks of kCodeRows rows
    int64_t T, TB;
    PageMap pm;
    SeqTab tab;
};

// Which rows a workgroup's thread takes: row number among all (`slot`) and the row of the cache, -1 for none.
struct CodeRows {
    int64_t slot[kCodePasses], at[kCodePasses];
    int g, layer;
    __device__ __forceinline__ CodeRows(const CodeArgs& a, int32_t* ends) {
        const int block = (int)blockIdx.x % a.blocks, sub = (int)threadIdx.x >> 4;
        g = (int)blockIdx.x / a.blocks;
        layer = blockIdx.y;
        const int n = a.tab.n_seq;
        if (n > 1) {
            if ((int)threadIdx.x < n) ends[threadIdx.x] = a.tab.cu_bud[threadIdx.x + 1];
            __syncthreads();
        }
#pragma unroll
        for (int i = 0; i < kCodePasses; ++i) {
            slot[i] = (int64_t)block * kCodeRows + 16 * i + sub;
            at[i] = -1;
            if (slot[i] >= a.TB) continue;
            int s = 0;
            if (n > 1)  // the number of sequences that end at or before the row
                for (int step = 64; step; step >>= 1)
                    if (s + step <= n && ends[s + step - 1] <= (int32_t)slot[i]) s += step;
            const int b = (int)(slot[i] - a.tab.cu_bud[s]);
            if (a.layer_budgets && b >= a.layer_budgets[(int64_t)layer * n + s]) continue;
            const int64_t pos = (int64_t)(a.first ? a.first[(int64_t)layer * n + s] : 0) + b;
            if (pos < 0 || pos >= a.tab.cu_seq[s + 1] - a.tab.cu_seq[s]) continue;  // no room: neither written nor read
            if (!a.pm.block_table) {
                at[i] = ((int64_t)layer * a.h_kv + g) * a.T + a.tab.cu_seq[s] + pos;
            } else {
                const int32_t e = a.pm.block_table[(int64_t)s * a.pm.max_pages + (pos >> a.pm.page_shift)];
                if ((uint32_t)e >= (uint32_t)a.pm.n_pages) continue;  // no page: clamped, the row would go over somebody's
                const int64_t page = (int64_t)layer * a.pm.n_pages + e;
                at[i] = ((page * a.h_kv + g) << a.pm.page_shift) + (pos & ((1 << a.pm.page_shift) - 1));
            }
        }
    }
};

template <int BITS>
__device__ __forceinline__ void store_eight(char* p, const uint32_t* codes) {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    if constexpr (BITS == 8) __builtin_nontemporal_store(u32x2{codes[0], codes[1]}, (u32x2*)p);
    else __builtin_nontemporal_store(codes[0], (uint32_t*)p);
}

// The codes of a lane's eight dimensions and its group's scale byte, out of bf16 patterns.
template <int BITS>
__device__ __forceinline__ uint32_t encode(au32x4 x, uint32_t* codes) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 most = {0, 0};
#pragma unroll
    for (int w = 0; w < 4; ++w) most = __builtin_elementwise_max(most, __builtin_bit_cast(u16x2, x[w] & 0x7FFF7FFFu));
    uint32_t a = max(most[0], most[1]);  // magnitudes are in the order of their patterns, what is not finite above all others
    a = max(a, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0xB1, 0xF, 0xF, false));  // the lane's neighbour
    a = max(a, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)a, 0x4E, 0xF, 0xF, false));  // the other two
    // 1.m * 2^E <= 448 * 2^x = 1.75 * 2^(x + 8), or 6 * 2^x = 1.5 * 2^(x + 2).  Not below -100, where a code's last place is 2^-109, and
    // not where the largest code would be no finite bf16: values beyond it become it.
    constexpr uint32_t kPart = BITS == 8 ? 0x60 : 0x40, kPower = BITS == 8 ? 8 : 2, kTop = BITS == 8 ? 246 : 252;
    const int byte = (int)(a >> 7) - (int)kPower + ((a & 0x7F) > kPart ? 1 : 0);
    const uint32_t scale = (uint32_t)min(max(byte, 27), (int)kTop);
    if (__any(a > (0x7F00u | kPart))) {  // (rare: 2^127 and more, and what is not finite)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            u16x2 size = __builtin_elementwise_min(__builtin_bit_cast(u16x2, x[w] & 0x7FFF7FFFu), u16x2{(uint16_t)(0x7F00u | kPart), (uint16_t)(0x7F00u | kPart)});
            x[w] = a >= 0x7F80u ? 0u : (x[w] & 0x80008000u) | __builtin_bit_cast(uint32_t, size);
        }
    }
    const float f = scale_of(scale);
    bf16x2 two[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const uint32_t word = x[w];  // (a bit cast of the vector's element itself takes its first one, ROCm 7.2)
        two[w] = __builtin_bit_cast(bf16x2, word);
    }
    if constexpr (BITS == 8) {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            s16x2 c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(s16x2{0, 0}, two[2 * w], f, false);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, two[2 * w + 1], f, true);
            codes[w] = __builtin_bit_cast(uint32_t, c);
        }
    } else {
        uint32_t c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(0u, two[0], f, 0);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, two[1], f, 1);
        c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, two[2], f, 2);
        codes[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, two[3], f, 3);
    }
    return a >= 0x7F80u ? 255u : scale;
}

template <int BITS>
__device__ __forceinline__ void write_row(char* codes_to, uint8_t* scales, int64_t at, au32x4 x) {
    const int part = threadIdx.x & 15;
    uint32_t codes[2];
    uint32_t word = encode<BITS>(x, codes) << 8 * (part >> 2);  // the row's four scale bytes, in its first lane
    word |= (uint32_t)__shfl_xor((int)word, 4);
    word |= (uint32_t)__shfl_xor((int)word, 8);
    if (at < 0) return;
    store_eight<BITS>(codes_to + at * (kHeadDim * BITS / 8) + part * BITS, codes);
    if (part == 0) *(uint32_t*)(scales + at * kGroups) = word;
}

template <int KB, int VB>
__global__ __launch_bounds__(kCodeThreads) void jq_quantize_kernel(CodeArgs a) {
    __shared__ int32_t ends[JQ_MAX_SEQ];
    const CodeRows rows(a, ends);
    const int part = threadIdx.x & 15;
    au32x4 k[kCodePasses], v[kCodePasses];
#pragma unroll
    for (int i = 0; i < kCodePasses; ++i) {  // (rows that are not written are read from the last one there is)
        const int64_t slot = min(rows.slot[i], a.TB - 1);
        const int64_t from = (((int64_t)rows.layer * a.TB + slot) * a.h_kv + rows.g) * (kHeadDim * 2) + part * 16;
        k[i] = __builtin_nontemporal_load((const au32x4*)(a.K_in + from));
        v[i] = __builtin_nontemporal_load((const au32x4*)(a.V_in + from));
    }
#pragma unroll
    for (int i = 0; i < kCodePasses; ++i) {
        write_row<KB>(a.K, a.K_scale, rows.at[i], k[i]);
        write_row<VB>(a.V, a.V_scale, rows.at[i], v[i]);
    }
}

template <int KB, int VB>
__global__ __launch_bounds__(kCodeThreads) void jq_dequantize_kernel(CodeArgs a) {
    __shared__ int32_t ends[JQ_MAX_SEQ];
    const CodeRows rows(a, ends);
    const int part = threadIdx.x & 15;
    uint32_t k[kCodePasses][2], v[kCodePasses][2], ks[kCodePasses], vs[kCodePasses];
#pragma unroll
    for (int i = 0; i < kCodePasses; ++i) {
        const int64_t at = max(rows.at[i], (int64_t)0);
        load_eight<KB>(k[i], a.K + at * (kHeadDim * KB / 8) + part * KB);
        load_eight<VB>(v[i], a.V + at * (kHeadDim * VB / 8) + part * VB);
        ks[i] = a.K_scale[at * kGroups + (part >> 2)];
        vs[i] = a.V_scale[at * kGroups + (part >> 2)];
    }
#pragma unroll
    for (int i = 0; i < kCodePasses; ++i) {
        if (rows.at[i] < 0) continue;
        const int64_t to = (((int64_t)rows.layer * a.TB + rows.slot[i]) * a.h_kv + rows.g) * (kHeadDim * 2) + part * 16;
        __builtin_nontemporal_store(eight_values<KB>(k[i], scale_of(ks[i])), (au32x4*)(a.K_out + to));
        __builtin_nontemporal_store(eight_values<VB>(v[i], scale_of(vs[i])), (au32x4*)(a.V_out + to));
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------------

static int64_t code_groups(const Plan& p) { return (p.TB + kCodeRows - 1) / kCodeRows * p.h_kv; }
bool codes_fit(const Plan& p) { return code_groups(p) * kCodeThreads <= UINT32_MAX; }

static CodeArgs code_args(const Plan& p, const Codes& c, const int32_t* first) {
    CodeArgs a{};
    a.K = (char*)c.K; a.V = (char*)c.V; a.K_scale = (uint8_t*)c.K_scale; a.V_scale = (uint8_t*)c.V_scale;
    a.first = first; a.layer_budgets = p.layer_budgets;
    a.h_kv = p.h_kv; a.blocks = (int32_t)((p.TB + kCodeRows - 1) / kCodeRows);
    a.T = p.T; a.TB = p.TB;
    a.pm = p.page_map(); a.tab = p.tab;
    return a;
}

hipError_t launch_quantize(const Plan& p, const Codes& c, const int32_t* first, const void* K, const void* V, hipStream_t st) {
    CodeArgs a = code_args(p, c, first);
    a.K_in = (const char*)K; a.V_in = (const char*)V;
    const dim3 grid((unsigned)code_groups(p), (unsigned)p.n_layers), block(kCodeThreads);
    if (c.k_bits == 4) return launch_kernel(jq_quantize_kernel<4, 4>, grid, block, 0, st, nullptr, -1, a);
    if (c.v_bits == 4) return launch_kernel(jq_quantize_kernel<8, 4>, grid, block, 0, st, nullptr, -1, a);
    return launch_kernel(jq_quantize_kernel<8, 8>, grid, block, 0, st, nullptr, -1, a);
}

hipError_t launch_dequantize(const Plan& p, const Codes& c, const int32_t* first, void* K, void* V, hipStream_t st) {
    CodeArgs a = code_args(p, c, first);
    a.K_out = (char*)K; a.V_out = (char*)V;
    const dim3 grid((unsigned)code_groups(p), (unsigned)p.n_layers), block(kCodeThreads);
    if (c.k_bits == 4) return launch_kernel(jq_dequantize_kernel<4, 4>, grid, block, 0, st, nullptr, -1, a);
    if (c.v_bits == 4) return launch_kernel(jq_dequantize_kernel<8, 4>, grid, block, 0, st, nullptr, -1, a);
    return launch_kernel(jq_dequantize_kernel<8, 8>, grid, block, 0, st, nullptr, -1, a);
}

}  // namespace jq
