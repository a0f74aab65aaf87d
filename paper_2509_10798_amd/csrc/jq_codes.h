// A cache held in codes: every 32 neighbouring dimensions of a row (a group) share a scale 2^x, and each value is a code of 8 bits
// (e4m3: sign, 4 bits of exponent, 3 of mantissa, largest 448) or 4 (e2m1, largest 6) times it.  The scale is a byte, x + 127; 255 says
// that the group held a value that is not finite, and makes NaN of all its codes.
//
// These are the formats that the conversions v_cvt_scalef32_* take, two values an instruction, with the scale as the exponent of a
// float.  A code has at most four significant bits, so its value is exact in bf16: attention over codes is attention over the bf16
// rows that they stand for, and differs from it in nothing but how the rows come into registers.  The matrix instruction that takes codes
// and scales as they lie (16x16x128, f8f6f4) was measured and left: its sums of 128 products are off by 2^-13 of the sum of their sizes.
//
// Layout: [layers][KV heads][rows][bytes], in pages [layers][pages][KV heads][rows of a page][bytes], the four scales of a row apart in
// the same order.  Heads lie outside the rows, other than in a bf16 cache, because a workgroup reads one head's: rows of 64 or 128 bytes
// are then read in one piece, and four bytes of scales do not bring the 28 of seven other heads with them.
#pragma once
#include "jq_attend.h"

namespace jq {

constexpr int kGroupDims = 32;
constexpr int kGroups = kHeadDim / kGroupDims;

typedef short s16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// Word `w` (two values) of the bf16 values of eight codes: two registers of 8-bit ones, one of 4-bit ones.
template <int BITS, int W>
__device__ __forceinline__ uint32_t two_values(const uint32_t* codes, float scale) {
    if constexpr (BITS == 8) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes[W / 2], scale, W % 2 != 0));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes[0], scale, W));
}
template <int BITS>
__device__ __forceinline__ au32x4 eight_values(const uint32_t* codes, float scale) {
    return au32x4{two_values<BITS, 0>(codes, scale), two_values<BITS, 1>(codes, scale), two_values<BITS, 2>(codes, scale), two_values<BITS, 3>(codes, scale)};
}
// The codes of eight dimensions of a row.
template <int BITS>
__device__ __forceinline__ void load_eight(uint32_t* codes, const char* p) {
    if constexpr (BITS == 8) {
        const uint2 x = *(const uint2*)p;
        codes[0] = x.x;
        codes[1] = x.y;
    } else {
        codes[0] = *(const uint32_t*)p;
    }
}

// One head's rows of one sequence.
template <int KB, int VB>
struct RowsCoded {
    static constexpr bool kCoded = true;
    // Two waves a SIMD: one issues a vector instruction every five cycles, two of them every other.  Twice the tiles of a bf16 cache
    // go through a CU in the time that memory takes, and with four waves a workgroup that bounded the call (us with four / eight:
    // one token over 131072 rows in 4 bits 46.7 / 37, 32 sequences of 2048 rows in 8 bits with weights 34.6 / 29.2).  Tiles requested two and
    // four ahead took 1.5 and 7 us more: a call this short is over before the longer start has paid.  (17 to 32 query rows with weights: the
    // sums of eight waves and the logits held do not fit LDS together.)
    static constexpr int waves(int row_tiles, bool weights) { return row_tiles == 1 || !weights ? 8 : kAttendWaves; }
    static constexpr int least_waves(int) { return 2; }
    static constexpr int kKRow = kHeadDim * KB / 8, kVRow = kHeadDim * VB / 8;
    // The scale that lane `E` of the lane's four holds.
    template <int E>
    static __device__ __forceinline__ float scale_in_four(uint32_t byte) {
        return scale_of((uint32_t)__builtin_amdgcn_mov_dpp((int)byte, E * 0x55, 0xF, 0xF, true));
    }
    // 32 keys: of key 16 i + l % 16 the group l / 16 of K, whose 32 terms of a sum are then the lane's; of V eight dimensions of key
    // 16 i + 4 (l / 16) + e as in a KvTile, whose group is (l % 16) / 4, and of the four lanes that share this group one scale each.
    struct Tile {
        uint32_t k[2][KB], v[2][4][VB / 4], k_scale[2], v_scale[2];
        __device__ __forceinline__ au32x4 key_piece(int i, int c) const { return eight_values<KB>(k[i] + c * (KB / 4), scale_of(k_scale[i])); }
        template <int W>
        __device__ __forceinline__ void value_words(uint32_t (&x)[2][4]) const {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                x[i][0] = two_values<VB, W>(v[i][0], scale_in_four<0>(v_scale[i]));
                x[i][1] = two_values<VB, W>(v[i][1], scale_in_four<1>(v_scale[i]));
                x[i][2] = two_values<VB, W>(v[i][2], scale_in_four<2>(v_scale[i]));
                x[i][3] = two_values<VB, W>(v[i][3], scale_in_four<3>(v_scale[i]));
            }
        }
    };
    struct Piece {
        uint32_t codes[2], scale;
    };
    const char* K; const char* V;
    const uint8_t* K_scale; const uint8_t* V_scale;
    const_i32_ptr table;
    int shift, n_pages, h_kv, g;
    bool paged;

    __device__ __forceinline__ RowsCoded(const AttendArgs& a, int layer, int s, int g_) : shift(a.pm.page_shift), n_pages(a.pm.n_pages), h_kv(a.h_kv), g(g_) {
        paged = a.pm.block_table != nullptr;
        const int64_t first_row = paged ? ((int64_t)layer * n_pages * h_kv) << shift : ((int64_t)layer * h_kv + g) * a.T + a.cu_seq[s];
        K = a.K + first_row * kKRow;
        V = a.V + first_row * kVRow;
        K_scale = a.K_scale + first_row * kGroups;
        V_scale = a.V_scale + first_row * kGroups;
        table = (const_i32_ptr)(paged ? a.pm.block_table + (int64_t)s * a.pm.max_pages : nullptr);
    }
    __device__ __forceinline__ uint32_t row(int key) const {
        if (!paged) return (uint32_t)key;
        return (((uint32_t)clamp_page(table[key >> shift], n_pages) * (uint32_t)h_kv + (uint32_t)g) << shift) + (uint32_t)(key & ((1 << shift) - 1));
    }
    static __device__ __forceinline__ int q_at(int c, int lane) { return 64 * (lane >> 4) + 16 * c; }
    __device__ __forceinline__ void load(Tile& t, uint32_t row0, int last, int lane) const {
        const uint32_t quarter = (uint32_t)(lane >> 4);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t at = row0 + (uint32_t)min(16 * i + (lane & 15), last);
            t.k_scale[i] = K_scale[at * kGroups + quarter];
#pragma unroll
            for (int h = 0; h < KB / 4; ++h) {
                const au32x4 x = *(const au32x4*)(K + (at * kKRow + quarter * (kKRow / 4) + 16u * h));
#pragma unroll
                for (int w = 0; w < 4; ++w) t.k[i][4 * h + w] = x[w];
            }
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint32_t mine = row0 + (uint32_t)min(16 * i + 4 * (lane >> 4) + (lane & 3), last);
            t.v_scale[i] = V_scale[mine * kGroups + (uint32_t)((lane & 15) >> 2)];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t at = row0 + (uint32_t)min(16 * i + 4 * (lane >> 4) + e, last);
                load_eight<VB>(t.v[i][e], V + (at * kVRow + (uint32_t)(lane & 15) * VB));
            }
        }
    }
    // The same of a tile that is all there: a uniform address, the lane's offset from it, the rest in the instruction.
    __device__ __forceinline__ void load_whole(Tile& t, uint32_t row0, int lane) const {
        const uint32_t quarter = (uint32_t)(lane >> 4), part = (uint32_t)(lane & 15);
        const char* k = K + row0 * kKRow;
        const char* v = V + row0 * kVRow;
        const uint8_t* ks = K_scale + row0 * kGroups;
        const uint8_t* vs = V_scale + row0 * kGroups;
        const uint32_t k_at = part * kKRow + quarter * (kKRow / 4), v_at = quarter * (4 * kVRow) + part * VB;
        const uint32_t ks_at = part * kGroups + quarter, vs_at = (4 * quarter + (part & 3)) * kGroups + (part >> 2);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            t.k_scale[i] = (ks + ks_at)[16 * i * kGroups];
            t.v_scale[i] = (vs + vs_at)[16 * i * kGroups];
#pragma unroll
            for (int h = 0; h < KB / 4; ++h) {
                const au32x4 x = *(const au32x4*)((k + k_at) + (16 * i * kKRow + 16 * h));
#pragma unroll
                for (int w = 0; w < 4; ++w) t.k[i][4 * h + w] = x[w];
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) load_eight<VB>(t.v[i][e], (v + v_at) + (16 * i + e) * kVRow);
        }
    }
    static __device__ __forceinline__ void unpack(KvTile& to, const Tile& t, int) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float scale = scale_of(t.k_scale[i]);
#pragma unroll
            for (int c = 0; c < 4; ++c) to.k[i][c] = eight_values<KB>(t.k[i] + c * (KB / 4), scale);
            to.v[i][0] = eight_values<VB>(t.v[i][0], scale_in_four<0>(t.v_scale[i]));
            to.v[i][1] = eight_values<VB>(t.v[i][1], scale_in_four<1>(t.v_scale[i]));
            to.v[i][2] = eight_values<VB>(t.v[i][2], scale_in_four<2>(t.v_scale[i]));
            to.v[i][3] = eight_values<VB>(t.v[i][3], scale_in_four<3>(t.v_scale[i]));
        }
    }
    struct Source {
        const char* base;
        const uint8_t* scales;
        bool is_v;
        __device__ __forceinline__ Source(const RowsCoded& rows, bool is_v_, int lane)
            : base(is_v_ ? rows.V + (lane & 15) * VB : rows.K + (lane & 15) * KB), scales((is_v_ ? rows.V_scale : rows.K_scale) + ((lane & 15) >> 2)), is_v(is_v_) {}
        __device__ __forceinline__ Piece request(uint32_t at) const {
            Piece x;
            x.scale = scales[at * kGroups];
            if (KB == VB || !is_v) load_eight<KB>(x.codes, base + at * kKRow);
            else load_eight<VB>(x.codes, base + at * kVRow);
            return x;
        }
        __device__ __forceinline__ au32x4 values(const Piece& x) const {
            if (KB == VB || !is_v) return eight_values<KB>(x.codes, scale_of(x.scale));
            return eight_values<VB>(x.codes, scale_of(x.scale));
        }
    };
    __device__ __forceinline__ uint32_t v_at(uint32_t at) const { return at; }
    __device__ __forceinline__ au32x4 v_piece(uint32_t at, int lane) const {
        uint32_t codes[2];
        load_eight<VB>(codes, V + (at * kVRow + (uint32_t)(lane & 15) * VB));
        return eight_values<VB>(codes, scale_of(V_scale[at * kGroups + (uint32_t)((lane & 15) >> 2)]));
    }
    __device__ __forceinline__ uint32_t v_value(uint32_t at, int d) const {
        uint32_t codes[2];
        load_eight<VB>(codes, V + (at * kVRow + (uint32_t)(d >> 3) * VB));
        const au32x4 x = eight_values<VB>(codes, scale_of(V_scale[at * kGroups + (uint32_t)(d / kGroupDims)]));
        const uint32_t two = d & 4 ? (d & 2 ? x[3] : x[2]) : (d & 2 ? x[1] : x[0]);
        return (d & 1 ? two >> 16 : two) & 0xFFFFu;
    }
};

}  // namespace jq
