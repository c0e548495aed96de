// The paged KV cache: device view, element order, launchers of its operations.
#pragma once

#include "common.h"

namespace bz {

constexpr float kE4m3Max = 448.f;

// Device-side view of a paged cache of one layer.  The elements of a (page, kv head) are blocks of 32 positions, each in the
// order in which a 32x32x16 MFMA reads its row operand: of activation elements as in KvView; of e4m3, sixteen elements to the
// 16 bytes a lane loads, which are two k-steps of the product:
//   K: [d/16][position][16], a lane half h reading piece 2i + h holds dims 32i + 16h + 0..15 of its position;
//   V: [h][j][16], the positions {4h + 0..3, 8 + 4h + 0..3} and the same 16 further on, of head dim j.
struct PagedView {
    void* k;
    void* v;
    const int32_t* table;      // [rows][per_row]
    int n_pages, per_row, page_shift;
    int Hkv, d;
    float k_scale, v_scale;    // what 1 in the cache stands for
    float k_inv, v_inv;        // their reciprocals
};

struct PagedRope {
    const float* tab;          // [positions][d/2] pairs of cos, sin; null: no rotation
    int positions;
};

// Offset inside a block of 32 positions.
template <bool E4M3>
__host__ __device__ inline int k_block_offset(int p, int j) {
    return E4M3 ? ((j >> 4) * 32 + p) * 16 + (j & 15) : ((j >> 3) * 32 + p) * 8 + (j & 7);
}
template <bool E4M3>
__host__ __device__ inline int v_block_offset(int p, int j, int d) {
    const int t = p >> 4, a = (p >> 3) & 1, h = (p >> 2) & 1, b = p & 3;
    return E4M3 ? (h * d + j) * 16 + 8 * t + 4 * a + b : ((2 * t + h) * d + j) * 8 + 4 * a + b;
}

// Page that holds `pos` of table row `row`; -1 if it is not there.  Whatever the table holds, the result is in range.
__device__ __forceinline__ int page_of(const PagedView& kv, int row, int pos) {
    const int i = pos >> kv.page_shift;
    if (i >= kv.per_row) return -1;
    // through the constant address space: a scalar load where the position is uniform, also behind stores and barriers
    typedef const __attribute__((address_space(4))) int32_t* entry_t;
    const int id = *(entry_t)(uintptr_t)(kv.table + (size_t)row * kv.per_row + i);
    return id >= 0 && id < kv.n_pages ? id : -1;
}
// First element of the block of 32 positions that holds `pos`, in page `id`, of kv head `head`.
__device__ __forceinline__ size_t block_base(const PagedView& kv, int id, int head, int pos) {
    const int in_page = pos & ((1 << kv.page_shift) - 1) & ~31;
    return ((((size_t)id * kv.Hkv + head) << kv.page_shift) + in_page) * kv.d;
}
// A position's row of the rotary table.  The host has checked the lengths; the bound holds for a captured graph that is
// replayed on longer ones.
__device__ __forceinline__ const float* rope_row(const PagedRope& rope, int pos, int d) {
    return rope.tab + (size_t)(pos < rope.positions ? pos : rope.positions - 1) * d;
}

// x / scale, given the scale's reciprocal, rounded to the odd one of the two floats around it: rounding that to e4m3 is rounding the
// quotient itself.  The product with the reciprocal can be off by a step, which makes a tie between two e4m3 numbers none (87.5 / 7 is
// 12.5, times 1/7 more); with what is left over, exact in the multiply-add, times the reciprocal it is the nearest float, and the sign of
// what is left then says on which side the quotient lies.  Beyond the largest e4m3 number, and for zeros with their sign, the product
// will do.
__device__ __forceinline__ float quotient(float x, float scale, float inv) {
    const float y = x * inv, q = fmaf(fmaf(-y, scale, x), inv, y), left = fmaf(-q, scale, x);
    const int bits = __float_as_int(q), step = (bits & 1) || left == 0.f ? 0 : (__float_as_int(left) ^ bits) < 0 ? -1 : 1;
    return y != 0.f && fabsf(y) < 2.f * kE4m3Max ? __int_as_float(bits + step) : y;
}
// Saturates to the largest e4m3 number; NaN stays.
__device__ __forceinline__ float e4m3_range(float x) {
    const float c = fminf(fmaxf(x, -kE4m3Max), kE4m3Max);
    return x != x ? x : c;
}
__device__ __forceinline__ uint8_t to_e4m3(float x) {
    return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(e4m3_range(x), 0.f, 0, false) & 0xff);
}
__device__ __forceinline__ float from_e4m3(uint8_t b) { return __builtin_amdgcn_cvt_f32_fp8((int)b, 0); }

// One element of a cache, as the number it holds (scale not applied).
template <bool E4M3>
__device__ __forceinline__ float cache_get(const void* base, size_t at) {
    if (E4M3) return from_e4m3(static_cast<const uint8_t*>(base)[at]);
    return to_f32(static_cast<const act_t*>(base)[at]);
}
template <bool E4M3>
__device__ __forceinline__ void cache_put(void* base, size_t at, float x) {
    if (E4M3) static_cast<uint8_t*>(base)[at] = to_e4m3(x);
    else from_f32(static_cast<act_t*>(base)[at], x);
}

// Whether a launch can have as many workgroups as an operation takes: the runtime counts a grid's threads in 32 bits.
constexpr int64_t kMaxWorkgroups = 0xffffffffLL / 256;      // of 256 threads
bool paged_append_fits(bool e4m3, const BatchView& bv, const PagedView& kv);
bool paged_read_fits(bool e4m3, const PagedView& kv, int pos0, int n);
void launch_paged_append(const act_t* k, size_t k_stride, const act_t* v, size_t v_stride, const PagedRope& rope, bool e4m3,
                         const BatchView& bv, const PagedView& kv, hipStream_t st);
void launch_paged_read(bool e4m3, const PagedView& kv, int row, int pos0, int n, act_t* k, act_t* v, hipStream_t st);

struct PagedQuery {
    const act_t* q;
    act_t* out;
    size_t q_stride, out_stride;
    PagedRope rope;
    int Hq, window;
    float scale_log2;          // score scale times log2 e, and times what 1 in the K cache stands for
};
// Division of 0 <= n < 2^31 by a number the host knows: with c = ceil(log2 d), mul = ceil(2^(31+c) / d) fits 32 bits,
// and n * mul / 2^(31+c) exceeds n / d by less than n / 2^(31+c) < 2^-c <= 1 / d: both have the same floor.
struct Divisor {
    uint32_t mul;              // 0: division by one
    int shift, d;
    __host__ __device__ int divide(int n) const {
#ifdef __HIP_DEVICE_COMPILE__
        return mul ? (int)(__umulhi((uint32_t)n, mul) >> shift) : n;
#else
        return mul ? (int)(((uint64_t)(uint32_t)n * mul) >> 32 >> shift) : n;
#endif
    }
};
inline Divisor divisor(int d) {
    int c = 0;
    while (((int64_t)1 << c) < d) ++c;
    if (c == 0) return Divisor{0, 0, 1};
    return Divisor{(uint32_t)((((uint64_t)1 << (31 + c)) + d - 1) / d), c - 1, d};
}

// How the attention of a batch is cut, from the host's copy of its lengths.  A sequence's new tokens times the query heads of a
// kv head are its rows there.  Narrow: single new tokens, and sequences of few rows; a workgroup takes up to kNarrowRows of them
// over one chunk of kDecodeChunk positions.  Wide: a workgroup takes kWideRows rows over the keys they see, or over one of
// `splits` ranges of them.
constexpr int kNarrowRows = 32, kWideRows = 128;
struct PagedWork {
    int n_short, short_tokens; // sequences of several tokens that are narrow (the first of BatchView::short_seqs), their most tokens
    int list;                  // workgroups of single tokens that the batch's work list names (no window), for one kv head
    int first;                 // sequences of decode_seqs and short_seqs from here on have `chunks` workgroups each per kv head
    int chunks;
    int max_chunks;            // of any narrow sequence
    int col_tiles;             // tiles of kNarrowRows rows of a narrow sequence
    int narrow_rows;           // most rows of one
    int narrow_limit;          // most rows of a sequence of several tokens that is narrow
    int wide_units;            // workgroups of wide rows that have work, times kv heads and ranges
    int splits;
    Divisor by_heads, by_chunks, by_tiles, by_group;   // n_kv_heads * col_tiles, chunks, col_tiles, G
};
bool paged_attention_fits(const PagedWork& w, const BatchView& bv, int Hq, int Hkv);
size_t paged_attention_bytes(const PagedWork& w, const BatchView& bv, int Hq, int Hkv, int d);
void launch_paged_attention(const PagedQuery& q, const PagedWork& w, bool e4m3, const BatchView& bv, const PagedView& kv,
                            float* ws, hipStream_t st);

}  // namespace bz
