// Attention of a batch's new tokens over a paged KV cache.
//
// A kv head's query heads and a sequence's new tokens are rows of one problem: row r of (sequence, kv head) is token r / G and
// query head kvh * G + r % G, G = Hq / Hkv, so every K and V that a workgroup reads serves all rows it holds.  Per row, with
// scores s_j in base 2 (scale times log2 e), m = max s_j, l = sum 2^(s_j - m), o = sum 2^(s_j - m) V_j / l, taken over the keys
// in pieces: (m, l, o) of two pieces join as m' = max, l' = l 2^(m - m') + ..., o' likewise.  A piece in which a row sees nothing
// has m = -inf, l = 0.
//
// Masked positions get weight 0, and 0 times a NaN is a NaN: values at positions that none of the workgroup's rows may see
// (behind the sequence, before the first row's window, on a page that is not there) are cleared before the product.  One that some of
// them see and that is not finite reaches the others as well: to tell them apart would cost every tile that a mask crosses.
#include "paged.h"

#include <algorithm>
#include <cfloat>

namespace bz {

#ifndef BZ_FP32_DEBUG
namespace {

typedef __attribute__((address_space(3))) void* lptr_t;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

// weights below the normal range flush to zero: the largest of a row's is 1
__device__ __forceinline__ float exp2_flush(float x) { return __builtin_amdgcn_exp2f(x); }

// reference of a running maximum that may not have seen a key yet
__device__ __forceinline__ float finite_or_0(float m) { return m > -INFINITY ? m : 0.f; }

// eight e4m3 numbers to bf16, which holds each of them exactly
__device__ __forceinline__ bf16x8 e4m3_to_bf16(uint32_t a, uint32_t b) {
    const bf16x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false), p1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true);
    const bf16x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false), p3 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true);
    return bf16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}

// eight e4m3 numbers to fp16, which holds each of them exactly as well
__device__ __forceinline__ f16x8 e4m3_to_f16(uint32_t a, uint32_t b) {
    const f16x2 p0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, false), p1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, true);
    const f16x2 p2 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, false), p3 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, true);
    return f16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
}

__device__ __forceinline__ f32x16 product(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 product(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
// c plus the sum of a pair of weights
__device__ __forceinline__ float add_pair(bf16x2 p, float c) { return __builtin_amdgcn_fdot2_f32_bf16(p, bf16x2{(bf16)1.f, (bf16)1.f}, c, false); }
__device__ __forceinline__ float add_pair(f16x2 p, float c) { return __builtin_amdgcn_fdot2(p, f16x2{(_Float16)1.f, (_Float16)1.f}, c, false); }

// 8 pairs (j0 + e, j0 + e + d/2) of a query: as they are, or rotated and scaled, as the sum of two bf16
template <bool ROTATE, int QP>
__device__ __forceinline__ void query8(const bf16* q, const float* cs, float scale, int half, bf16x8 (&lower)[QP], bf16x8 (&upper)[QP]) {
    lower[0] = *reinterpret_cast<const bf16x8*>(q);
    upper[0] = *reinterpret_cast<const bf16x8*>(q + half);
    if (!ROTATE) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float2 v = *reinterpret_cast<const float2*>(cs + 2 * e);
        const float y = (float)lower[0][e], z = (float)upper[0][e];
        const float a = (y * v.x - z * v.y) * scale, b = (z * v.x + y * v.y) * scale;
        lower[0][e] = (bf16)a;
        upper[0][e] = (bf16)b;
        lower[QP - 1][e] = (bf16)(a - (float)lower[0][e]);
        upper[QP - 1][e] = (bf16)(b - (float)upper[0][e]);
    }
}

// the same in fp16, times `factor`, which keeps the row within range
template <bool ROTATE>
__device__ __forceinline__ void query8(bf16x8 y8, bf16x8 z8, const float* cs, float factor, f16x8& lower, f16x8& upper) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float2 v = ROTATE ? *reinterpret_cast<const float2*>(cs + 2 * e) : make_float2(1.f, 0.f);
        const float y = (float)y8[e] * factor, z = (float)z8[e] * factor;
        lower[e] = (_Float16)(ROTATE ? y * v.x - z * v.y : y);
        upper[e] = (_Float16)(ROTATE ? z * v.x + y * v.y : z);
    }
}
// largest exponent of eight numbers, as bf16 holds it
__device__ __forceinline__ int top_exponent(bf16x8 v, int top) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const bf16 x = v[e];
        const int m = (__builtin_bit_cast(uint16_t, x) >> 7) & 255;
        top = m > top ? m : top;
    }
    return top;
}

// the larger, or the sum, of a lane's value and that of its partner 32 lanes on: a vector instruction, no trip through LDS
__device__ __forceinline__ float2 pair_of(float x) {
    const uint32_t b = __float_as_uint(x);
    const auto r = __builtin_amdgcn_permlane32_swap(b, b, false, false);
    const uint32_t lower = r[0], upper = r[1];
    return make_float2(__uint_as_float(lower), __uint_as_float(upper));
}
__device__ __forceinline__ float pair_max(float x) {
    const float2 v = pair_of(x);
    return fmaxf(v.x, v.y);
}
__device__ __forceinline__ float pair_sum(float x) {
    const float2 v = pair_of(x);
    return v.x + v.y;
}

// The softmax of a tile of 64 keys for rows that lane pairs own, against a reference that only has to be within 2^kLag of the
// largest score so far: then most tiles leave the accumulators alone.  The row's largest weight is 2^TOP when the reference is set,
// and weights are at most 2^(TOP + kLag): everything is relative to it and no bits are lost.  With TOP = 6 fp16, which ends at 2^-24,
// holds weights down to 2^-30 of the largest.
constexpr float kLag = 8.f;
template <int DB, bool SCALED, typename P2, typename P8, int TOP>
struct RowSoftmax {
    float ref = 0.f, l = 0.f;            // l over this lane's half of the keys
    bool seen = false;                   // the reference is one
    f32x16 start;                        // SCALED: -ref sixteen times, what the score products start from

    __device__ __forceinline__ void init() {
#pragma unroll
        for (int x = 0; x < 16; ++x) start[x] = 0.f;
    }
    // scores (SCALED: in base 2, the reference taken off by the product; else raw) to weights
    __device__ __forceinline__ void weigh(f32x16 (&s)[2], float scale, f32x16 (&o)[DB], P8 (&pf)[4]) {
        float mx = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int x = 0; x < 16; ++x) mx = fmaxf(mx, s[kb][x]);
        mx = SCALED ? pair_max(mx) : fmaf(pair_max(mx), scale, -ref);      // above the reference
        const bool move = mx > (seen ? TOP + kLag : -INFINITY);
        if (__builtin_amdgcn_ballot_w64(move) != 0) {
            const float up = move ? mx - TOP : 0.f, alpha = move && !seen ? 0.f : exp2_flush(-up);
            seen |= move;
            ref += up;
            l *= alpha;
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
                for (int x = 0; x < 16; ++x) o[b][x] *= alpha;
            if (SCALED) {
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int x = 0; x < 16; ++x) s[kb][x] -= up;
#pragma unroll
                for (int x = 0; x < 16; ++x) start[x] = -ref;
            }
        }
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const float a = s[t >> 1][8 * (t & 1) + e], b = s[t >> 1][8 * (t & 1) + e + 1];
                P2 p;
                p[0] = exp2_flush(SCALED ? a : fmaf(a, scale, -ref));
                p[1] = exp2_flush(SCALED ? b : fmaf(b, scale, -ref));
                l = add_pair(p, l);                          // the sum of the weights as the product will use them
                pf[t][e] = p[0];
                pf[t][e + 1] = p[1];
            }
    }
};

// the part of a number that `mask`, 16 bits or none, leaves of it
__device__ __forceinline__ float above(float x, uint32_t mask) { return __uint_as_float(__float_as_uint(x) & mask); }
// two numbers as bf16, cut off: what is cut is `x - above(x, 0xffff0000)`, exactly
__device__ __forceinline__ bf16x2 upper_halves(float x, float y) {
    return __builtin_bit_cast(bf16x2, __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u));
}

// x of the lane plus x of the lane eight further in its row of sixteen
__device__ __forceinline__ float add_eighth(float x) {
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), 0x128, 0xf, 0xf, true));
}

__device__ __forceinline__ int first_seen(int pos, int window) { return window && pos + 1 > window ? pos + 1 - window : 0; }

// Partial results of narrow sequences: per (token, query head) and chunk D floats of the output, and behind all of those maximum and
// sum.  Single tokens come first, then `short_tokens` per sequence.
__device__ __forceinline__ size_t partial_at(const PagedWork& w, int n_decode, int i, int token, int Hq, int head, int chunk) {
    const int t = i < n_decode ? i : n_decode + (i - n_decode) * w.short_tokens + token;
    return ((size_t)t * Hq + head) * w.max_chunks + chunk;
}
__device__ __forceinline__ float2* partial_sums(float* partial, const PagedWork& w, int n_decode, int Hq, int D) {
    return reinterpret_cast<float2*>(partial + (size_t)(n_decode + w.n_short * w.short_tokens) * Hq * w.max_chunks * D);
}

}  // namespace

// ---------------------------------------------------------------------------------------------
// Narrow: a workgroup reads one chunk of 256 positions of one kv head once, for up to RT rows.  Each of its four waves takes 64
// positions, with all their loads in flight at once, and computes S = K Q^T and O = V^T P^T with 32x32x16 products whose
// row operand is the cache as it lies in memory; rows of the problem are the 32 columns.  The four waves' results are merged through
// LDS in wave order.  Bound by the cache's bytes (64 sequences of up to 4096 positions on 8 kv heads with four query heads each, bf16:
// 95.5 us, 5.8 TB/s; a streaming read has 7.1 at best), in few workgroups by one's 6.6 us from launch to end.
//
// Queries are kept as the sum of two bf16, rounded after the rotation to 16 bits and not to 8, and so are weights, cut off behind 15 or 16:
// what the matrix pipe does beside the stream costs little.  With up to eight rows the second parts are columns 8..15, which the first
// parts leave free, and two columns' scores, outputs and sums are added across lanes (of weights: 32 sequences on e4m3 80.4 -> 80.8 us a
// call, 64 on bf16 99.8 both).  With more they are products of their own (of weights: 24 drafts 47.8 -> 48.2); over e4m3, where that costs
// 6 %, weights are fp16 instead, 11 bits down to 2^-28 of the largest.  The
// output's distance from a computation in 64 bits is 1.7e-3 (rms), which is its own rounding to bf16; with weights of one bf16 it was 2.1e-3,
// with queries of one, too, 2.7e-3.
//
// A chunk's partial results are written and read once more, RT * (d + 2) floats for 512 * d cache elements: a sixteenth of the bytes
// for eight rows of e4m3.  Chunks of twice the length halve that and gain nothing (32 sequences of up to 12000 positions on 8 kv heads
// with eight query heads each, kernel and join, weights of one bf16: 81.3 us with one step of 64 positions per wave and four waves per SIMD, 83.8 with two
// steps and the three waves that these leave room for).
template <int D, bool E4M3, int RT, int WAVES>
__global__ __attribute__((amdgpu_waves_per_eu(WAVES, WAVES))) __launch_bounds__(256) void paged_narrow_kernel(
    PagedQuery a, PagedWork w, BatchView bv, PagedView kv, float* __restrict__ partial) {
    constexpr int CH = kDecodeChunk, KS = D / 16, DB = D / 32, LD = D + 8;
    constexpr int NF = E4M3 ? D / 32 : D / 16;               // 16-byte loads per lane and block, of K and again of V
    __shared__ float wmx[4][RT], wsum[4][RT];
    constexpr int PARTS = RT > 8 ? 2 : 1, DP = D / PARTS;    // of the head dim that are merged at a time: LDS for one workgroup more
    __shared__ __attribute__((aligned(16))) float osh[4][RT][DP + 4];        // rows 16 bytes out of step: lanes write rows
    __shared__ __attribute__((aligned(16))) bf16 qs[2][RT][LD];

    const int G = w.by_group.d;
    // kv heads next to each other, then chunks, then sequences: the order in which pages lie in memory
    int e = w.by_heads.divide(blockIdx.x);
    const int hc = blockIdx.x - e * w.by_heads.d, kvh = w.by_tiles.divide(hc), ct = hc - kvh * w.by_tiles.d;
    int i, s, row, chunk;
    if (e < w.list) {
        const int4 item = bv.decode_work[2 * e];
        s = item.x;
        row = item.y;
        i = item.z;
        chunk = e - bv.decode_work[2 * e + 1].x;
    } else {
        e -= w.list;
        i = w.by_chunks.divide(e);
        chunk = e - i * w.by_chunks.d;
        i += w.first;
        s = bv.decode_seqs[i];
        row = bv.seq_slot[s];
    }
    const int q0 = bv.q_start[s], n = bv.q_start[s + 1] - q0, before = bv.kv_before[s];
    const int hi = before + n, lo = first_seen(before, a.window);
    const int c0 = (lo & ~63) + chunk * CH;
    const int r0 = ct * kNarrowRows, R = n * G;
    if (c0 >= hi || r0 >= R || chunk >= w.max_chunks) return;
    const int rows = R - r0 < RT ? R - r0 : RT;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lq = lane & 31, lh = lane >> 5;
    const int w0 = c0 + wave * 64;
    const bool live = w0 < hi;                               // wave-uniform
    int id[2];                                               // pages, -1 for one that is not there
#pragma unroll
    for (int b = 0; b < 2; ++b) id[b] = w0 + 32 * b < hi ? page_of(kv, row, w0 + 32 * b) : -1;

    // queries: unit = 8 pairs of a row, requested before the stream
    constexpr int UPR = D / 16;
    const int units = rows * UPR;
    const int u = tid < units ? tid : units - 1;
    const int ur = u / UPR, uj = (u - ur * UPR) * 8;
    const int ut = w.by_group.divide(r0 + ur), uh = kvh * G + (r0 + ur) - ut * G;
    const bf16* qp = a.q + (size_t)(q0 + ut) * a.q_stride + uh * D + uj;
    bf16x8 qlo = *reinterpret_cast<const bf16x8*>(qp), qhi = *reinterpret_cast<const bf16x8*>(qp + D / 2);
    f32x4 cs[4] = {};
    if (a.rope.tab) {
        const float* c = rope_row(a.rope, before + ut, D) + 2 * uj;
#pragma unroll
        for (int x = 0; x < 4; ++x) cs[x] = *reinterpret_cast<const f32x4*>(c + 4 * x);
    }
    __builtin_amdgcn_sched_barrier(0);

    // non-temporal: nobody reads them again.  A base in scalar registers, one vector register for all addresses of K, one for V.
    constexpr int EL = E4M3 ? 1 : 2;
    auto block = [&](void* cache, int b) {
        const int page = id[b] < 0 ? 0 : id[b];              // read in bounds, masked below
        return __builtin_amdgcn_make_buffer_rsrc(static_cast<uint8_t*>(cache) + block_base(kv, page, kvh, w0 + 32 * b) * EL, 0, 32 * D * EL,
                                                 0x00020000);
    };
    auto load = [&](__amdgpu_buffer_rsrc_t r, int lane_at, int at) {
        return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, lane_at, at, 2));
    };
    // pieces of K: [piece][position]; a step takes two, one per lane half.  Pieces of V: [2t + h][j], or [h][j] with both t.
    const int lane_k = (lh * 32 + lq) * 16, lane_v = (lh * D + lq) * 16;
    u32x4 kf[2][NF], vf[2][NF];
    auto load_k = [&]() {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const __amdgpu_buffer_rsrc_t r = block(kv.k, b);
#pragma unroll
            for (int x = 0; x < NF; ++x) kf[b][x] = load(r, lane_k, x * 1024);
        }
    };
    auto load_v = [&]() {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const __amdgpu_buffer_rsrc_t r = block(kv.v, b);
#pragma unroll
            for (int x = 0; x < NF; ++x) vf[b][x] = load(r, lane_v, E4M3 ? x * 512 : (x / DB) * (2 * D * 16) + (x % DB) * 512);
        }
    };
    if (live) {
        load_k();
        if (RT == 8) load_v();
    }
    __builtin_amdgcn_sched_barrier(0);
    bf16x8 rlo = {}, rhi = {};                               // the second parts
    if (a.rope.tab) {
#pragma unroll
        for (int x = 0; x < 8; ++x) {
            const float c = cs[x >> 1][2 * (x & 1)], sn = cs[x >> 1][2 * (x & 1) + 1];
            const float y = (float)qlo[x], z = (float)qhi[x], p = y * c - z * sn, q = z * c + y * sn;
            qlo[x] = (bf16)p;
            qhi[x] = (bf16)q;
            rlo[x] = (bf16)(p - (float)qlo[x]);
            rhi[x] = (bf16)(q - (float)qhi[x]);
        }
    }
    if (tid < units) {
        *reinterpret_cast<bf16x8*>(&qs[0][ur][uj]) = qlo;
        *reinterpret_cast<bf16x8*>(&qs[0][ur][D / 2 + uj]) = qhi;
        *reinterpret_cast<bf16x8*>(&qs[1][ur][uj]) = rlo;
        *reinterpret_cast<bf16x8*>(&qs[1][ur][D / 2 + uj]) = rhi;
    }
    // with more queries to keep on the way, V's requests would leave them no registers
    if (RT > 8 && live) load_v();
    // hand-over through LDS; a full barrier would drain the stream
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");

    float m = -INFINITY, l = 0.f;                            // of the lane's column
    f32x16 oacc[DB];
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[db][r] = 0.f;
    // columns past the rows repeat the first and are dropped
    constexpr bool BESIDE = RT == 8;                         // second parts in columns of their own
    // weights: two bf16; over e4m3 without room beside, fp16, from 2^14 down, which is exact in that as well
    constexpr bool HALF = E4M3 && !BESIDE;
    using P2 = typename std::conditional<HALF, f16x2, bf16x2>::type;
    using P8 = typename std::conditional<HALF, f16x8, bf16x8>::type;
    const int col = BESIDE ? lq & 7 : lq, qr = col < rows ? col : 0;
    const bf16* qcol = &qs[BESIDE ? (lq >> 3) & 1 : 0][qr][0];
    if (live) {
        const int qpos = before + w.by_group.divide(r0 + qr);
        const int p_min = before + w.by_group.divide(r0), p_max = before + w.by_group.divide(r0 + rows - 1);
        const bool whole = id[0] >= 0 && id[1] >= 0;
        f32x16 sacc[2];
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) sacc[b][r] = 0.f;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            // e4m3: product 2x + y takes bytes 8y.. of piece pair x, dims 32x + 16h + 8y ..
            const int j = E4M3 ? (ks >> 1) * 32 + lh * 16 + (ks & 1) * 8 : ks * 16 + lh * 8;
            const bf16x8 qf = *reinterpret_cast<const bf16x8*>(qcol + j);
            bf16x8 ql;
            if (!BESIDE) ql = *reinterpret_cast<const bf16x8*>(&qs[1][qr][j]);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                bf16x8 kk;
                if (E4M3) kk = e4m3_to_bf16(kf[b][ks >> 1][2 * (ks & 1)], kf[b][ks >> 1][2 * (ks & 1) + 1]);
                else kk = *reinterpret_cast<const bf16x8*>(&kf[b][ks]);
                sacc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kk, qf, sacc[b], 0, 0, 0);
                if (!BESIDE) sacc[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kk, ql, sacc[b], 0, 0, 0);
            }
        }
        if (BESIDE)
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) sacc[b][r] = add_eighth(sacc[b][r]);
        // lane (column lq, half lh) holds positions w0 + 32 b + 8 (r / 4) + 4 lh + r % 4
        if (w0 + 63 > p_min || (a.window && w0 <= p_max - a.window) || !whole) {
            const int from = first_seen(qpos, a.window);
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int pos = w0 + b * 32 + 8 * (r >> 2) + 4 * lh + (r & 3);
                    const uint32_t reach = id[b] >= 0 ? qpos - from + 1 : 0;
                    sacc[b][r] = (uint32_t)(pos - from) < reach ? sacc[b][r] : -INFINITY;
                    __builtin_amdgcn_sched_barrier(0);   // one at a time: 32 lane masks do not fit the scalar registers
                }
            if (w0 + 64 > hi || w0 < lo || !whole) {
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const uint32_t length = id[b] >= 0 ? hi - lo : 0;
                    auto keep = [&](int off) { return (uint32_t)(w0 + 32 * b + 4 * lh + off - lo) < length; };   // inside the block
#pragma unroll
                    for (int t = 0; t < 2; ++t)
#pragma unroll
                        for (int g = 0; g < 2; ++g) {
                            __builtin_amdgcn_sched_barrier(0);
                            const int off = 16 * t + 8 * g;      // positions 16 t + 8 g + 4 lh + 0..3
                            if (E4M3) {
                                const uint32_t k4 = (keep(off) ? 0xffu : 0) | (keep(off + 1) ? 0xff00u : 0) |
                                                    (keep(off + 2) ? 0xff0000u : 0) | (keep(off + 3) ? 0xff000000u : 0);
#pragma unroll
                                for (int x = 0; x < NF; ++x) vf[b][x][2 * t + g] &= k4;
                            } else {
                                const uint32_t m0 = (keep(off) ? 0xffffu : 0) | (keep(off + 1) ? 0xffff0000u : 0);
                                const uint32_t m1 = (keep(off + 2) ? 0xffffu : 0) | (keep(off + 3) ? 0xffff0000u : 0);
#pragma unroll
                                for (int db = 0; db < DB; ++db) {
                                    vf[b][t * DB + db][2 * g] &= m0;
                                    vf[b][t * DB + db][2 * g + 1] &= m1;
                                }
                            }
                        }
                }
            }
        }
        float mx = -INFINITY;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sacc[b][r]);
        m = pair_max(mx) * a.scale_log2 - (HALF ? 14.f : 0.f);      // scale > 0
        const float ref = finite_or_0(m);
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) sacc[b][r] = exp2_flush(fmaf(sacc[b][r], a.scale_log2, -ref));
        // columns 8..15 take the second parts of the weights, as they did of the queries
        const uint32_t second = lq & 8 ? 0xffff0000u : 0;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                P8 pf, pl;
#pragma unroll
                for (int x = 0; x < 8; x += 2) {
                    const float y = sacc[b][8 * t + x], z = sacc[b][8 * t + x + 1];
                    P2 p;                                    // l: of the weights as the product will use them
                    if constexpr (HALF) p = P2{(_Float16)y, (_Float16)z};
                    else p = BESIDE ? upper_halves(y - above(y, second), z - above(z, second)) : upper_halves(y, z);
                    l = add_pair(p, l);
                    pf[x] = p[0];
                    pf[x + 1] = p[1];
                    if constexpr (!HALF && !BESIDE) {
                        const P2 r = upper_halves(y - above(y, 0xffff0000u), z - above(z, 0xffff0000u));
                        l = add_pair(r, l);
                        pl[x] = r[0];
                        pl[x + 1] = r[1];
                    }
                }
#pragma unroll
                for (int db = 0; db < DB; ++db) {
                    P8 vv;
                    if constexpr (HALF) vv = e4m3_to_f16(vf[b][db][2 * t], vf[b][db][2 * t + 1]);
                    else if constexpr (E4M3) vv = e4m3_to_bf16(vf[b][db][2 * t], vf[b][db][2 * t + 1]);
                    else vv = *reinterpret_cast<const bf16x8*>(&vf[b][t * DB + db]);
                    oacc[db] = product(vv, pf, oacc[db]);
                    if constexpr (!HALF && !BESIDE) oacc[db] = product(vv, pl, oacc[db]);
                }
            }
        if (BESIDE) {
            l = add_eighth(l);
#pragma unroll
            for (int db = 0; db < DB; ++db)
#pragma unroll
                for (int r = 0; r < 16; ++r) oacc[db][r] = add_eighth(oacc[db][r]);
        }
        l = pair_sum(l);
    }
    // a wave that had nothing leaves m = -inf, l = 0, o = 0
    if (lq < rows && lh == 0) {
        wmx[wave][lq] = m;
        wsum[wave][lq] = l;
    }
    const bool alone = hi - (lo & ~63) <= CH;                // the only chunk: the output itself
#pragma unroll
    for (int part = 0; part < PARTS; ++part) {
        if (part) __syncthreads();
        if (lq < rows) {
#pragma unroll
            for (int db = 0; db < DB / PARTS; ++db)
#pragma unroll
                for (int r4 = 0; r4 < 4; ++r4) {
                    const f32x16& v = oacc[part * (DB / PARTS) + db];
                    *reinterpret_cast<float4*>(&osh[wave][lq][db * 32 + 8 * r4 + 4 * lh]) =
                        make_float4(v[4 * r4], v[4 * r4 + 1], v[4 * r4 + 2], v[4 * r4 + 3]);
                }
        }
        __syncthreads();
        for (int x = tid * 4; x < rows * DP; x += 1024) {
            const int g = x / DP, dd = x - g * DP;
            const float M = fmaxf(fmaxf(wmx[0][g], wmx[1][g]), fmaxf(wmx[2][g], wmx[3][g]));
            const float ref = finite_or_0(M);
            float L = 0.f;
            f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float f = exp2_flush(wmx[v][g] - ref);
                const f32x4 y = *reinterpret_cast<const f32x4*>(&osh[v][g][dd]);
#pragma unroll
                for (int z = 0; z < 4; ++z) acc[z] = fmaf(y[z], f, acc[z]);
                L = fmaf(wsum[v][g], f, L);
            }
            const int t = w.by_group.divide(r0 + g), head = kvh * G + (r0 + g) - t * G, j = part * DP + dd;
            if (alone) {
                const float inv = L > 0.f ? kv.v_scale / L : 0.f;
                const bf16x4 y = {(bf16)(acc[0] * inv), (bf16)(acc[1] * inv), (bf16)(acc[2] * inv), (bf16)(acc[3] * inv)};
                *reinterpret_cast<bf16x4*>(a.out + (size_t)(q0 + t) * a.out_stride + head * D + j) = y;
            } else {
                const size_t at = partial_at(w, bv.n_decode, i, t, a.Hq, head, chunk);
                *reinterpret_cast<f32x4*>(partial + at * D + j) = acc;
                if (j == 0) partial_sums(partial, w, bv.n_decode, a.Hq, D)[at] = make_float2(M, L);
            }
        }
    }
}

// ---------------------------------------------------------------------------------------------
// Wide: 128 rows per workgroup, 32 per wave, keys in tiles of 64 through LDS.  S^T = K Q^T, so that a lane pair (lane, lane + 32)
// owns a row: its maximum and sum need one exchange, the rescale of O^T is a per-lane factor, and P^T goes from the score
// accumulators into O^T = V^T P^T without leaving registers, since V's pieces hold the positions in the accumulators' order.
// Activation caches move global -> LDS by DMA, the next tile's loads between the score products; e4m3 goes through registers, one tile
// ahead, where it becomes fp16.
//
// What is rounded: a bf16 cache is multiplied by queries that are, after the rotation, the sum of two bf16, and by weights in bf16;
// an e4m3 cache, which fp16 holds exactly, by queries and weights in fp16, a query's row brought to fp16's range by a power of two
// that its scores give back.  Distance of the output from a computation in 64 bits, rms: 2.0e-3 to 2.3e-3 over bf16 and 1.7e-3, the
// output's own rounding, over e4m3.  With rotated queries in one bf16 it is 2.5e-3 to 2.9e-3, and the 48 products per tile and wave are
// 32 (four prompts of 2048 tokens on 8 kv heads with eight query heads each: 299 us, with two 375).
//
// Bound by the matrix pipe: those 48 products of random numbers take 1.2 us at the clock that the chip's power allows (25 ns each and
// SIMD, registers only), a tile 1.4 per CU.  The softmax between them is the other wave's time on the SIMD: 32 exponentials, 16 of each of
// maximum, conversion and sum.  Its pieces that pay: a reference that lags the maximum (above), taken off by the product
// itself, which starts from it; the tile's sum as a product with ones.
// ---------------------------------------------------------------------------------------------
struct WideUnit {
    int item, sub, split, kvh;
};
// XCD-aware: workgroups go to the eight XCDs in turn; with a multiple of eight kv heads each XCD takes whole kv heads and walks
// one after the other, longest key ranges first, so that what runs on it at a time shares the K and V in its L2.  A grid that fits the
// chip in one go, two workgroups per CU, lasts as long as its busiest CU, which holds an XCD's workgroups c and 32 + c: the second half
// is walked backwards, long with short (one prompt of 2048 tokens on 32 kv heads: 77 -> 61 us).
__device__ __forceinline__ WideUnit wide_unit(int b, int n_items, int subs, int Hkv, int splits) {
    const int per_head = n_items * subs * splits;
    WideUnit u;
    int rest;
    if ((Hkv & 7) == 0) {
        const int n_x = per_head * (Hkv >> 3);
        int seq = b >> 3;
        if (n_x <= 64 && seq >= 32) seq = 32 + (n_x - 1 - seq);
        const int k = seq / per_head;
        u.kvh = (b & 7) * (Hkv >> 3) + k;
        rest = seq - k * per_head;
    } else {
        u.kvh = b / per_head;
        rest = b - u.kvh * per_head;
    }
    u.item = rest / (subs * splits);
    rest -= u.item * (subs * splits);
    u.sub = subs - 1 - rest / splits;
    u.split = rest % splits;
    return u;
}

// the tiles of 64 keys that kWideRows rows from r0 on see, or the range of them that `split` names
struct WideKeys {
    int t0, t1, splits;
};
__device__ __forceinline__ WideKeys wide_keys(int before, int r0, int R, int G, int window, int split, int splits) {
    const int first = before + r0 / G, last = before + (r0 + kWideRows < R ? r0 + kWideRows - 1 : R - 1) / G;
    WideKeys k;
    k.t0 = first_seen(first, window) >> 6;
    k.t1 = (last >> 6) + 1;
    const int per = (k.t1 - k.t0 + splits - 1) / splits;
    k.splits = (k.t1 - k.t0 + per - 1) / per;
    k.t0 += split * per;
    if (k.t0 + per < k.t1) k.t1 = k.t0 + per;
    return k;
}

// Where the two blocks of a tile of 64 keys lie, counted in blocks of 32 positions from the start of the cache, -1 for one that is
// behind the sequence or on a page that is not there.  A wave keeps 64 tiles' in its lanes: the table is read once per 4096
// positions, and a tile's entry costs a lane read, where a scalar load behind LDS reads would wait for all of them.
struct TileMap {
    int base, x, y;
    __device__ __forceinline__ void load(const PagedView& kv, int row, int kvh, int hi, int from) {
        base = from;
        const int pos = (int)(((uint32_t)from + (threadIdx.x & 63)) * 64), per_page = kv.page_shift - 5;
        auto block = [&](int p) {
            const int id = p < hi && p >= 0 ? page_of(kv, row, p) : -1;
            return id < 0 ? -1 : ((id * kv.Hkv + kvh) << per_page) + ((p >> 5) & ((1 << per_page) - 1));
        };
        x = block(pos);
        y = block(pos + 32);
    }
    __device__ __forceinline__ int2 operator()(const PagedView& kv, int row, int kvh, int hi, int tile) {
        if (tile >= base + 64) load(kv, row, kvh, hi, tile);
        return make_int2(__builtin_amdgcn_readlane(x, tile - base), __builtin_amdgcn_readlane(y, tile - base));
    }
};
// first element of a block; the cache's first block in place of none: read in bounds, masked
template <int D>
__device__ __forceinline__ size_t block_start(int block) { return (size_t)(uint32_t)(block < 0 ? 0 : block) * (32 * D); }

// Partial results of key ranges: [kv head][range][dims by fours][row of the batch, token * G + query head of the group][4], and behind
// those maximum and sum, [kv head][range][row][2].
__device__ __forceinline__ float2* wide_sums(float* partial, size_t rows, int Hkv, int splits, int D) {
    return reinterpret_cast<float2*>(partial + rows * Hkv * splits * D);
}

template <int D, bool E4M3, bool ROTATE, bool SPLIT>
__global__ __launch_bounds__(256, 2) void paged_wide_kernel(PagedQuery a, PagedWork w, BatchView bv, PagedView kv,
                                                            float* __restrict__ partial) {
    constexpr int DB = D / 32, KS = D / 16, BLK = 32 * D;
    constexpr int NL = D / 32;           // 1 KiB DMA loads per wave and tile, of K and again of V
    constexpr int NC = D / 64;           // e4m3: 16-byte loads per thread and tile, of K and again of V
    constexpr int STAGE = 4 * BLK;       // K tile (two blocks), V tile (two blocks)
    // two bytes each: the cache's bf16, or e4m3 as fp16
    using T2 = typename std::conditional<E4M3, f16x2, bf16x2>::type;
    using T8 = typename std::conditional<E4M3, f16x8, bf16x8>::type;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem_raw[];
    bf16* smem = reinterpret_cast<bf16*>(smem_raw);

    const int Hkv = kv.Hkv, G = a.Hq / Hkv;
    const WideUnit unit = wide_unit(blockIdx.x, bv.n_prefill_items, G, Hkv, w.splits);
    const int s = bv.prefill_items[2 * unit.item], qt = bv.prefill_items[2 * unit.item + 1];
    const int q0 = bv.q_start[s], n = bv.q_start[s + 1] - q0, before = bv.kv_before[s], row = bv.seq_slot[s];
    const int R = n * G, r0 = (qt * G + unit.sub) * kWideRows;
    if (r0 >= R || R <= w.narrow_limit) return;
    const WideKeys keys = wide_keys(before, r0, R, G, a.window, unit.split, w.splits);
    if (SPLIT && keys.t0 >= keys.t1) return;
    const int hi = before + n, lo = first_seen(before + r0 / G, a.window);
    const int kvh = unit.kvh;

    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int lq = lane & 31, lh = lane >> 5;
    const int r = r0 + wave * 32 + lq;
    const bool valid = r < R;
    const int rc = valid ? r : R - 1, token = w.by_group.divide(rc), head = kvh * G + rc - token * G, qpos = before + token;
    const int wr = r0 + wave * 32 < R - 1 ? r0 + wave * 32 : R - 1, wl = r0 + wave * 32 + 31 < R - 1 ? r0 + wave * 32 + 31 : R - 1;
    const int wave_min_pos = before + wr / G, wave_max_pos = before + wl / G;

    TileMap map;
    map.load(kv, row, kvh, hi, keys.t0);
    auto look_up = [&](int tile) { return map(kv, row, kvh, hi, tile); };
    // this wave's block of a tile: waves 0 and 1 move the first, 2 and 3 the second
    const int wblk = wave >> 1;
    // DMA loads through buffer resources of the wave's half of a K and of a V block: a base in scalar registers, one vector register
    // for all addresses
    auto source = [&](int2 t) { return block_start<D>(wblk ? t.y : t.x) + (wave & 1) * (BLK / 2); };
    const int lane16 = lane * 16;
    auto issue_one = [&](size_t src, int stage, int q) {
        const int j = q % NL;                                // of the wave's 1 KiB pieces
        bf16* to = smem + stage * STAGE + (q < NL ? 0 : 2 * BLK) + wave * (BLK / 2) + j * 512;
        const __amdgpu_buffer_rsrc_t r =
            __builtin_amdgcn_make_buffer_rsrc(static_cast<bf16*>(q < NL ? kv.k : kv.v) + src, 0, BLK, 0x00020000);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (lptr_t)to, 16, lane16, j * 1024, 0, 0);
    };
    u32x4 kreg[NC], vreg[NC];
    auto fetch = [&](int2 t) {                               // e4m3
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = tid + 256 * i, blk = NC == 2 ? i : wblk, in = c - blk * (2 * D);
            const size_t at = block_start<D>(blk ? t.y : t.x) + in * 16;
            kreg[i] = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(kv.k) + at);
            vreg[i] = *reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(kv.v) + at);
        }
    };
    auto unpack = [&](int stage) {
        bf16* ks = smem + stage * STAGE;
        bf16* vs = ks + 2 * BLK;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = tid + 256 * i, blk = NC == 2 ? i : wblk, in = c - blk * (2 * D);
            const int piece = in >> 5, p = in & 31, h = in / D, j = in - h * D;
            *reinterpret_cast<f16x8*>(ks + blk * BLK + ((2 * piece) * 32 + p) * 8) = e4m3_to_f16(kreg[i][0], kreg[i][1]);
            *reinterpret_cast<f16x8*>(ks + blk * BLK + ((2 * piece + 1) * 32 + p) * 8) = e4m3_to_f16(kreg[i][2], kreg[i][3]);
            *reinterpret_cast<f16x8*>(vs + blk * BLK + (h * D + j) * 8) = e4m3_to_f16(vreg[i][0], vreg[i][1]);
            *reinterpret_cast<f16x8*>(vs + blk * BLK + ((2 + h) * D + j) * 8) = e4m3_to_f16(vreg[i][2], vreg[i][3]);
        }
    };

    int2 now = look_up(keys.t0);
    if (E4M3) {
        fetch(now);
        unpack(0);
    } else {
        const size_t src = source(now);
#pragma unroll
        for (int q = 0; q < 2 * NL; ++q) issue_one(src, 0, q);
    }

    constexpr int QP = !E4M3 && ROTATE ? 2 : 1;              // parts of a query: a rotated one does not fit one bf16
    T8 qf[KS][QP];
    float row_scale = a.scale_log2;      // of this lane's row, for raw scores
    {
        const bf16* qp = a.q + (size_t)(q0 + token) * a.q_stride + head * D + lh * 8;
        const float* cs = ROTATE ? rope_row(a.rope, qpos, D) + 2 * (lh * 8) : nullptr;
        if constexpr (E4M3) {
            bf16x8 raw[KS];
            int top = 0;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                raw[ks] = *reinterpret_cast<const bf16x8*>(qp + ks * 16);
                top = top_exponent(raw[ks], top);
            }
            // to below 2^14 and, after the rotation, 2^15
            top = (int)pair_max((float)top);
            const int up = 140 - (top > 20 ? top : 20);
            const float factor = ldexpf(1.f, up);
            row_scale = fminf(fmaxf(ldexpf(a.scale_log2, -up), FLT_MIN), FLT_MAX);     // 0 times -inf, a masked score, is a NaN
#pragma unroll
            for (int ks = 0; ks < KS / 2; ++ks) query8<ROTATE>(raw[ks], raw[ks + KS / 2], cs + 32 * ks, factor, qf[ks][0], qf[ks + KS / 2][0]);
        } else {
#pragma unroll
            for (int ks = 0; ks < KS / 2; ++ks) query8<ROTATE>(qp + ks * 16, cs + 32 * ks, a.scale_log2, D / 2, qf[ks], qf[ks + KS / 2]);
        }
    }
    f32x16 o[DB];
#pragma unroll
    for (int b = 0; b < DB; ++b)
#pragma unroll
        for (int x = 0; x < 16; ++x) o[b][x] = 0.f;
    // rotated queries that are the sum of two bf16 are scaled as well; fp16 has few exponents, its weights reach up to 2^(6 + kLag)
    constexpr bool SCALED = QP == 2;
    RowSoftmax<DB, SCALED, T2, T8, E4M3 ? 6 : 0> rows;
    rows.init();

    for (int tile = keys.t0; tile < keys.t1; ++tile) {
        const int stage = (tile - keys.t0) & 1, kbase = tile * 64;
        __builtin_amdgcn_s_waitcnt(0x0070);                  // own pieces of this tile landed, own LDS accesses done
        __syncthreads();                                     // everyone's; the other stage is free
        const bf16* Ks = smem + stage * STAGE;
        const bf16* Vs = Ks + 2 * BLK;
        const int2 cur = now;
        const bool whole = cur.x >= 0 && cur.y >= 0;
        // after the last tile it is requested once more into the idle stage: no branch between the products
        if (tile + 1 < keys.t1) now = look_up(tile + 1);
        const size_t src = source(now);
        if (E4M3) fetch(now);
        if (kbase + 64 > hi || kbase < lo || !whole) {     // workgroup-uniform
            // values that nobody may see: one thread per 8 positions of a head dim
            bf16* vw = smem + stage * STAGE + 2 * BLK;
            int c = tid;
            asm volatile("" : "+v"(c));                      // rare: nothing of this is worth a register over the whole loop
            for (; c < 8 * D; c += 256) {
                const int blk = c / (4 * D), piece = (c / D) & 3;
                const int p = kbase + 32 * blk + 16 * (piece >> 1) + 4 * (piece & 1);
                bf16x8 v = *reinterpret_cast<bf16x8*>(vw + c * 8);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int pos = p + (e & 3) + 8 * (e >> 2);
                    if ((blk ? cur.y : cur.x) < 0 || pos < lo || pos >= hi) v[e] = (bf16)0.f;
                }
                *reinterpret_cast<bf16x8*>(vw + c * 8) = v;
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
            __builtin_amdgcn_s_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
        }
        // a wave whose rows see nothing of this tile computes it like the others: as a branch it cost a copy of the accumulators
        f32x16 sacc[2];
        // operand fetch runs ahead of the products by hand: each K fragment of the first key block is replaced by the second
        // block's when its product has gone, and under the second block's the first V fragments are requested
        constexpr int EVERY = (2 * KS) / (2 * NL);
        auto k_frag = [&](int kb, int ks) { return *reinterpret_cast<const T8*>(&Ks[kb * BLK + ((ks * 2 + lh) * 32 + lq) * 8]); };
        auto v_frag = [&](int t, int b) {
            return *reinterpret_cast<const T8*>(&Vs[(t >> 1) * BLK + ((2 * (t & 1) + lh) * D + b * 32 + lq) * 8]);
        };
        T8 ka[KS], vfr[2][DB];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) ka[ks] = k_frag(0, ks);
        if (!SCALED) rows.init();
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                sacc[kb] = product(ka[ks], qf[ks][0], ks ? sacc[kb] : rows.start);
                if (QP == 2) sacc[kb] = product(ka[ks], qf[ks][QP - 1], sacc[kb]);
                if (kb == 0) ka[ks] = k_frag(1, ks);
                else if (ks < 2 * DB) vfr[ks / DB][ks % DB] = v_frag(ks / DB, ks % DB);
                const int step = kb * KS + ks;
                if (!E4M3 && step % EVERY == EVERY - 1) issue_one(src, stage ^ 1, step / EVERY);
                __builtin_amdgcn_sched_barrier(0);
            }
        if (kbase + 63 > wave_min_pos || (a.window && kbase <= wave_max_pos - a.window) || !whole) {
            const int from = first_seen(qpos, a.window);
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int x = 0; x < 16; ++x) {
                    const int pos = kbase + kb * 32 + 8 * (x >> 2) + 4 * lh + (x & 3);
                    const uint32_t reach = (kb ? cur.y : cur.x) >= 0 ? qpos - from + 1 : 0;
                    sacc[kb][x] = (uint32_t)(pos - from) < reach ? sacc[kb][x] : -INFINITY;
                }
        }
        T8 pf[4];
        rows.weigh(sacc, row_scale, o, pf);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
#pragma unroll
            for (int b = 0; b < DB; ++b) {
                o[b] = product(vfr[t & 1][b], pf[t], o[b]);
                if (t + 2 < 4) vfr[t & 1][b] = v_frag(t + 2, b);
            }
        }
        if (E4M3) unpack(stage ^ 1);
    }

    const float l = pair_sum(rows.l);
    __builtin_amdgcn_s_waitcnt(0x0070);                      // no LDS write may be in flight when the workgroup ends
    if (SPLIT) {
        if (valid) {
            const size_t total = (size_t)bv.T * G, part = ((size_t)kvh * w.splits + unit.split) * total, at = (size_t)q0 * G + r;
            float* op = partial + (part * (D / 4) + at) * 4;
#pragma unroll
            for (int b = 0; b < DB; ++b)
#pragma unroll
                for (int r4 = 0; r4 < 4; ++r4)
                    *reinterpret_cast<float4*>(op + ((b * 4 + r4) * 2 + lh) * total * 4) =
                        make_float4(o[b][4 * r4], o[b][4 * r4 + 1], o[b][4 * r4 + 2], o[b][4 * r4 + 3]);
            if (lh == 0)
                wide_sums(partial, total, Hkv, w.splits, D)[part + at] = make_float2(rows.seen ? rows.ref : -INFINITY, l);
        }
    } else if (valid) {
        const float inv = l > 0.f ? kv.v_scale / l : 0.f;
        int at = rc;
        asm volatile("" : "+v"(at));                         // found again rather than kept over the loop
        const int tok = w.by_group.divide(at), hd = kvh * G + at - tok * G;
        bf16* op = a.out + (size_t)(q0 + tok) * a.out_stride + hd * D;
#pragma unroll
        for (int b = 0; b < DB; ++b)
#pragma unroll
            for (int r4 = 0; r4 < 4; ++r4) {
                bf16x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = (bf16)(o[b][r4 * 4 + e] * inv);
                *reinterpret_cast<bf16x4*>(op + b * 32 + 8 * r4 + 4 * lh) = v;
            }
    }
}

// ---------------------------------------------------------------------------------------------
// Joins the pieces: one launch for the chunks of narrow sequences and the key ranges of wide rows, where a batch has both (512 new tokens
// on 3001 beside 40 single ones: 113.8 us, with a launch each 118).  Bound by the launch and two trips to memory, with many wide rows by the
// bytes of their partial results.
// ---------------------------------------------------------------------------------------------
// Chunks of the narrow sequences that have several, in increasing order: D / 4 threads per (token, query head), eight chunks' loads in
// flight at once.
template <int D, int THREADS>
__device__ __forceinline__ void join_narrow(const PagedQuery& a, const PagedWork& w, const BatchView& bv, const PagedView& kv,
                                            float* partial, int i) {
    constexpr int NB = 8, TPR = D / 4;
    int token = 0;
    if (i >= bv.n_decode) {
        const int x = i - bv.n_decode;
        i = bv.n_decode + x / w.short_tokens;
        token = x % w.short_tokens;
    }
    const int h = blockIdx.y * (THREADS / TPR) + threadIdx.x / TPR, j = (threadIdx.x % TPR) * 4;
    const int s = bv.decode_seqs[i];
    const int q0 = bv.q_start[s], n = bv.q_start[s + 1] - q0, before = bv.kv_before[s];
    if (token >= n || h >= a.Hq) return;
    int nch = (before + n - (first_seen(before, a.window) & ~63) + kDecodeChunk - 1) / kDecodeChunk;
    if (nch == 1) return;                                    // the output is there
    if (nch > w.max_chunks) nch = w.max_chunks;
    const size_t at = partial_at(w, bv.n_decode, i, token, a.Hq, h, 0);
    const float* o = partial + at * D + j;
    const float2* ml = partial_sums(partial, w, bv.n_decode, a.Hq, D) + at;
    float M = -INFINITY, den = 0.f;
    f32x4 num = {0.f, 0.f, 0.f, 0.f};
    for (int c0 = 0; c0 < nch; c0 += NB) {
        float2 mv[NB];
        f32x4 ov[NB];
#pragma unroll
        for (int u = 0; u < NB; ++u) {
            const int c = c0 + u < nch ? c0 + u : nch - 1;
            mv[u] = ml[c];
            ov[u] = *reinterpret_cast<const f32x4*>(o + (size_t)c * D);
        }
        float Mb = M;
#pragma unroll
        for (int u = 0; u < NB; ++u) Mb = fmaxf(Mb, mv[u].x);
        const float ref = finite_or_0(Mb), keep = exp2_flush(M - ref);
        num *= keep;
        den *= keep;
        M = Mb;
        // no branches: behind one every load would be waited for by itself.  A chunk past the end gets weight zero.
#pragma unroll
        for (int u = 0; u < NB; ++u) {
            const float f = c0 + u < nch ? exp2_flush(mv[u].x - ref) : 0.f;
#pragma unroll
            for (int z = 0; z < 4; ++z) num[z] = fmaf(ov[u][z], f, num[z]);
            den = fmaf(mv[u].y, f, den);
        }
    }
    const float inv = den > 0.f ? kv.v_scale / den : 0.f;
    const bf16x4 y = {(bf16)(num[0] * inv), (bf16)(num[1] * inv), (bf16)(num[2] * inv), (bf16)(num[3] * inv)};
    *reinterpret_cast<bf16x4*>(a.out + (size_t)(q0 + token) * a.out_stride + h * D + j) = y;
}

// Key ranges of wide rows, in increasing order: 32 rows of a kv head.
template <int D>
__device__ __forceinline__ void join_wide(const PagedQuery& a, const PagedWork& w, const BatchView& bv, const PagedView& kv,
                                          float* partial, int rows32) {
    const int Hkv = kv.Hkv, G = w.by_group.d, kvh = blockIdx.y;
    const int64_t total = (int64_t)bv.T * G, at = (int64_t)rows32 * 32 + (threadIdx.x & 31);
    if (at >= total || kvh >= Hkv) return;
    const int t = w.by_group.divide((int)at), s = bv.token_seq[t], q0 = bv.q_start[s], n = bv.q_start[s + 1] - q0;
    const int R = n * G, r = (int)at - q0 * G;
    if (n < 2 || R <= w.narrow_limit) return;
    const WideKeys keys = wide_keys(bv.kv_before[s], r & ~(kWideRows - 1), R, G, a.window, 0, w.splits);
    const float2* ml = wide_sums(partial, total, Hkv, w.splits, D) + (size_t)kvh * w.splits * total + at;
    const float* o = partial + ((size_t)kvh * w.splits * total * (D / 4) + at) * 4;
    float M = -INFINITY;
    for (int k = 0; k < keys.splits; ++k) M = fmaxf(M, ml[k * total].x);
    const float ref = finite_or_0(M);
    constexpr int NQ = D / 32;
    f32x4 acc[NQ] = {};
    float L = 0.f;
    for (int k = 0; k < keys.splits; ++k) {
        const float2 x = ml[k * total];
        const float f = exp2_flush(x.x - ref);
        L = fmaf(x.y, f, L);
        const float* ok = o + (size_t)k * total * D;
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            const f32x4 v = *reinterpret_cast<const f32x4*>(ok + (size_t)(i * 8 + (threadIdx.x >> 5)) * total * 4);
#pragma unroll
            for (int z = 0; z < 4; ++z) acc[i][z] = fmaf(v[z], f, acc[i][z]);
        }
    }
    const float inv = L > 0.f ? kv.v_scale / L : 0.f;
    bf16* op = a.out + (size_t)t * a.out_stride + (kvh * G + (int)at - t * G) * D + (threadIdx.x >> 5) * 4;
#pragma unroll
    for (int i = 0; i < NQ; ++i) {
        const bf16x4 v = {(bf16)(acc[i][0] * inv), (bf16)(acc[i][1] * inv), (bf16)(acc[i][2] * inv), (bf16)(acc[i][3] * inv)};
        *reinterpret_cast<bf16x4*>(op + i * 32) = v;
    }
}

template <int D, bool CHUNKS, bool RANGES>
__global__ __launch_bounds__(RANGES ? 256 : 128) void paged_join_kernel(PagedQuery a, PagedWork w, BatchView bv, PagedView kv,
                                                                        float* __restrict__ narrow, float* __restrict__ wide,
                                                                        int tokens) {
    if (CHUNKS && (!RANGES || (int)blockIdx.x < tokens)) join_narrow<D, RANGES ? 256 : 128>(a, w, bv, kv, narrow, blockIdx.x);
    else if (RANGES) join_wide<D>(a, w, bv, kv, wide, blockIdx.x - tokens);
}

// ---------------------------------------------------------------------------------------------
static size_t narrow_bytes(const PagedWork& w, const BatchView& bv, int Hq, int d) {
    if (w.max_chunks <= 1) return 0;
    const size_t tokens = (size_t)bv.n_decode + (size_t)w.n_short * w.short_tokens;
    return (tokens * Hq * w.max_chunks * (d + 2) * sizeof(float) + 255) / 256 * 256;
}

size_t paged_attention_bytes(const PagedWork& w, const BatchView& bv, int Hq, int, int d) {
    const size_t wide = w.splits > 1 ? (size_t)bv.T * Hq * w.splits * (d + 2) * sizeof(float) : 0;
    return narrow_bytes(w, bv, Hq, d) + wide;
}

static int64_t narrow_grid(const PagedWork& w, const BatchView& bv, int Hkv) {
    return (w.list + ((int64_t)bv.n_decode + w.n_short - w.first) * w.chunks) * Hkv * w.col_tiles;
}
static int64_t wide_grid(const PagedWork& w, const BatchView& bv, int Hq) {
    return w.wide_units > 0 ? (int64_t)bv.n_prefill_items * Hq * w.splits : 0;
}
// tokens whose chunks are joined, and groups of 32 rows whose key ranges are
static int64_t join_tokens(const PagedWork& w, const BatchView& bv) {
    return w.max_chunks > 1 ? bv.n_decode + (int64_t)w.n_short * w.short_tokens : 0;
}
static int64_t join_rows(const PagedWork& w, const BatchView& bv) {
    return w.wide_units > 0 && w.splits > 1 ? ((int64_t)bv.T * w.by_group.d + 31) / 32 : 0;
}
bool paged_attention_fits(const PagedWork& w, const BatchView& bv, int Hq, int Hkv) {
    return narrow_grid(w, bv, Hkv) <= kMaxWorkgroups && wide_grid(w, bv, Hq) <= kMaxWorkgroups &&
           join_tokens(w, bv) + join_rows(w, bv) <= kMaxWorkgroups && (int64_t)bv.T * w.by_group.d < 0x7fffff00LL;     // rows are ints
}

template <int D, bool E4M3, bool ROTATE, bool SPLIT>
static void launch_wide(const PagedQuery& q, const PagedWork& w, const BatchView& bv, const PagedView& kv, float* ws, hipStream_t st) {
    constexpr int kLds = 2 * 4 * 32 * D * (int)sizeof(bf16);             // two stages of a K and a V tile
    static LdsLimit limit;
    (void)limit.raise(reinterpret_cast<const void*>(paged_wide_kernel<D, E4M3, ROTATE, SPLIT>), kLds);
    hipLaunchKernelGGL((paged_wide_kernel<D, E4M3, ROTATE, SPLIT>), dim3((unsigned)wide_grid(w, bv, q.Hq)), dim3(256), kLds, st, q, w, bv,
                       kv, ws);
}

template <int D, bool E4M3>
static void launch_all(const PagedQuery& q, const PagedWork& w, const BatchView& bv, const PagedView& kv, float* ws, hipStream_t st) {
    const int n_narrow = bv.n_decode + w.n_short;
    if (n_narrow > 0) {
        // waves per SIMD: what the registers, and with 32 rows the LDS, leave room for; two for bf16 of d = 128, where a third
        // keeps the memory streams in shorter runs
        constexpr int FEW = E4M3 || D == 64 ? 4 : 2;
        // one form for the whole launch, by its widest sequence: single tokens beside a draft of more than eight rows take the 32-row form,
        // too (64 on 256 to 4096 positions of 8 kv heads, four query heads each, with one draft of 8 rows 99.4 us, of 16 rows 102.3)
        const unsigned grid = (unsigned)narrow_grid(w, bv, kv.Hkv);
        auto kern = w.narrow_rows <= 8 ? paged_narrow_kernel<D, E4M3, 8, FEW> : paged_narrow_kernel<D, E4M3, kNarrowRows, 3>;
        hipLaunchKernelGGL(kern, dim3(grid), dim3(256), 0, st, q, w, bv, kv, ws);
    }
    float* wide = ws ? ws + narrow_bytes(w, bv, q.Hq, D) / sizeof(float) : nullptr;
    if (w.wide_units > 0) {
        auto rows = q.rope.tab ? (w.splits > 1 ? launch_wide<D, E4M3, true, true> : launch_wide<D, E4M3, true, false>)
                               : (w.splits > 1 ? launch_wide<D, E4M3, false, true> : launch_wide<D, E4M3, false, false>);
        rows(q, w, bv, kv, wide, st);
    }
    const int tokens = (int)join_tokens(w, bv), rows32 = (int)join_rows(w, bv);
    const bool chunks = tokens > 0, ranges = rows32 > 0;
    if (!chunks && !ranges) return;
    const int threads = ranges ? 256 : 128, heads = threads / (D / 4);       // of one workgroup
    const unsigned across = std::max(chunks ? (q.Hq + heads - 1) / heads : 0, ranges ? kv.Hkv : 0);
    auto join = chunks ? (ranges ? paged_join_kernel<D, true, true> : paged_join_kernel<D, true, false>) : paged_join_kernel<D, false, true>;
    hipLaunchKernelGGL(join, dim3(tokens + rows32, across), dim3(threads), 0, st, q, w, bv, kv, ws, wide, tokens);
}

void launch_paged_attention(const PagedQuery& q, const PagedWork& w, bool e4m3, const BatchView& bv, const PagedView& kv, float* ws,
                            hipStream_t st) {
    auto go = kv.d == 128 ? (e4m3 ? launch_all<128, true> : launch_all<128, false>) : (e4m3 ? launch_all<64, true> : launch_all<64, false>);
    go(q, w, bv, kv, ws, st);
}

#else  // BZ_FP32_DEBUG
// ---------------------------------------------------------------------------------------------
// fp32 debug build: one wave per (token, query head), 64 positions at a time with a running maximum and sum; a lane scores one
// position and owns d / 64 dims of the output.
// ---------------------------------------------------------------------------------------------
template <bool E4M3, int D>
__global__ __launch_bounds__(64) void paged_attn_plain_kernel(PagedQuery a, BatchView bv, PagedView kv) {
    __shared__ float qs[D];
    const int t = blockIdx.x, h = blockIdx.y, lane = threadIdx.x;
    const int s = bv.token_seq[t], row = bv.seq_slot[s];
    const int pos = bv.kv_before[s] + (t - bv.q_start[s]);
    const int kvh = h / (a.Hq / kv.Hkv);
    const act_t* q = a.q + (size_t)t * a.q_stride + h * D;
    for (int j = lane; j < D / 2; j += 64) {
        const float lo = to_f32(q[j]), hi = to_f32(q[D / 2 + j]);
        float o_lo = lo, o_hi = hi;
        if (a.rope.tab) {
            const float* cs = rope_row(a.rope, pos, D);
            o_lo = lo * cs[2 * j] - hi * cs[2 * j + 1];
            o_hi = hi * cs[2 * j] + lo * cs[2 * j + 1];
        }
        act_t r;
        from_f32(r, o_lo);
        qs[j] = to_f32(r);
        from_f32(r, o_hi);
        qs[D / 2 + j] = to_f32(r);
    }
    __syncthreads();
    const int first = a.window && pos + 1 > a.window ? pos + 1 - a.window : 0;
    float m = -INFINITY, l = 0.f, o[D / 64] = {};
    for (int c0 = first & ~63; c0 <= pos; c0 += 64) {
        const int kp = c0 + lane;
        const int id = kp <= pos && kp >= first ? page_of(kv, row, kp) : -1;
        float sc = -INFINITY;
        if (id >= 0) {
            const size_t at = block_base(kv, id, kvh, kp);
            float x = 0.f;
            for (int j = 0; j < D; ++j) x = fmaf(qs[j], cache_get<E4M3>(kv.k, at + k_block_offset<E4M3>(kp & 31, j)), x);
            sc = x * a.scale_log2;
        }
        const float mx = fmaxf(m, wave_max(sc));
        if (mx == -INFINITY) continue;                       // nothing seen yet; wave-uniform
        const float alpha = exp2f(m - mx), w = exp2f(sc - mx);
        m = mx;
        l = l * alpha + wave_sum(w);
        for (int i = 0; i < D / 64; ++i) o[i] *= alpha;
        const int n = pos + 1 - c0 < 64 ? pos + 1 - c0 : 64;
        for (int u = 0; u < n; ++u) {
            const int uid = __shfl(id, u, 64);
            if (uid < 0) continue;
            const float wu = __shfl(w, u, 64);
            const size_t at = block_base(kv, uid, kvh, c0 + u);
            for (int i = 0; i < D / 64; ++i)
                o[i] = fmaf(wu, cache_get<E4M3>(kv.v, at + v_block_offset<E4M3>((c0 + u) & 31, lane + 64 * i, D)), o[i]);
        }
    }
    for (int i = 0; i < D / 64; ++i)
        from_f32(a.out[(size_t)t * a.out_stride + h * D + lane + 64 * i], l > 0.f ? o[i] / l * kv.v_scale : 0.f);
}

bool paged_attention_fits(const PagedWork&, const BatchView&, int, int) { return true; }      // 64 threads per token

size_t paged_attention_bytes(const PagedWork&, const BatchView&, int, int, int) { return 0; }

void launch_paged_attention(const PagedQuery& a, const PagedWork&, bool e4m3, const BatchView& bv, const PagedView& kv, float*,
                            hipStream_t st) {
    auto kern = kv.d == 128 ? (e4m3 ? paged_attn_plain_kernel<true, 128> : paged_attn_plain_kernel<false, 128>)
                            : (e4m3 ? paged_attn_plain_kernel<true, 64> : paged_attn_plain_kernel<false, 64>);
    hipLaunchKernelGGL(kern, dim3(bv.T, a.Hq), dim3(64), 0, st, a, bv, kv);
}
#endif

}  // namespace bz
