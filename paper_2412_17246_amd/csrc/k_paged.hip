// Operations on the paged KV cache that move it: the append of a batch's new tokens with the rotation on the way, and the way
// back out.
#include "paged.h"

namespace bz {

#ifndef BZ_FP32_DEBUG
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Both operations go by blocks of 32 positions of a head, which 256 threads take one (bf16, d = 128), two or four at a time.
//   K: a thread has 8 (e4m3: 16) pairs (j, j + d/2) of one position, which are a piece of the lower and one of the upper half;
//      consecutive threads have consecutive pieces, so rows are read or written by whole 128-byte lines, and eight of them
//      consecutive positions, 128 bytes in the cache.
//   V: a thread has two consecutive head dims of the 8 (e4m3: 16) positions of a piece: 256 bytes of a row per wave, and 32
//      consecutive bytes per thread in the cache.
template <int D, bool E4M3>
struct Blocks {
    static constexpr int VEC = E4M3 ? 16 : 8;                // elements of a 16-byte piece
    static constexpr int THREADS = 32 * D / 2 / VEC;         // of one head
    static constexpr int PAR = 256 / THREADS;                // heads side by side
    static constexpr int UNITS = D / 2 / VEC;                // pieces of half a head

    // position within the block of element e of V piece w
    __device__ static int v_pos(int w, int e) {
        return E4M3 ? 16 * (e >> 3) + 4 * w + 8 * ((e >> 2) & 1) + (e & 3) : 16 * (w >> 1) + 4 * (w & 1) + 8 * (e >> 2) + (e & 3);
    }
};

// four numbers from x[i] on over the scale, as e4m3
template <int VEC>
__device__ __forceinline__ uint32_t pack4(const float (&x)[VEC], int i, float scale, float inv) {
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = e4m3_range(quotient(x[i + e], scale, inv));
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
}
// VEC numbers as the cache holds them
template <bool E4M3, int VEC>
__device__ __forceinline__ u32x4 pack(const float (&x)[VEC], float scale, float inv) {
    if constexpr (E4M3) {
        u32x4 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = pack4(x, 4 * i, scale, inv);
        return r;
    } else {
        bf16x8 r;
#pragma unroll
        for (int i = 0; i < 8; ++i) r[i] = (bf16)x[i];
        return __builtin_bit_cast(u32x4, r);
    }
}
template <bool E4M3, int VEC>
__device__ __forceinline__ void unpack(u32x4 r, float scale, float (&x)[VEC]) {
    if constexpr (E4M3) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)r[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)r[i], true);
            x[4 * i] = lo[0] * scale;
            x[4 * i + 1] = lo[1] * scale;
            x[4 * i + 2] = hi[0] * scale;
            x[4 * i + 3] = hi[1] * scale;
        }
    } else {
        const bf16x8 v = __builtin_bit_cast(bf16x8, r);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
    }
}
template <int VEC>
__device__ __forceinline__ void load_row(const bf16* p, float (&x)[VEC]) {
#pragma unroll
    for (int i = 0; i < VEC; i += 8) {
        const bf16x8 v = *reinterpret_cast<const bf16x8*>(p + i);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i + e] = (float)v[e];
    }
}
template <int VEC>
__device__ __forceinline__ void rotate(float (&lo)[VEC], float (&hi)[VEC], const float* cs) {
#pragma unroll
    for (int e = 0; e < VEC; e += 2) {
        const float4 c = *reinterpret_cast<const float4*>(cs + 2 * e);
        const float l0 = lo[e], h0 = hi[e], l1 = lo[e + 1], h1 = hi[e + 1];
        lo[e] = l0 * c.x - h0 * c.y;
        hi[e] = h0 * c.x + l0 * c.y;
        lo[e + 1] = l1 * c.z - h1 * c.w;
        hi[e + 1] = h1 * c.z + l1 * c.w;
    }
}

}  // namespace

// ---------------------------------------------------------------------------------------------
// Append.  Sequences with several new tokens: one workgroup per block of 32 positions and `heads_per_wg` heads.  Single new tokens:
// workgroups from `block_wgs` on, `row_wgs` per token, a thread per 8 rotation pairs or 8 values.  Bound by bytes, each moved once
// (9378 tokens on 40 kv heads, bf16: 96 us, 4.1 TB/s, where a large copy has 4.7); a single token by the launch (2.1 us), many by the
// lines that they touch: a value is one element of each of d pieces of 16 bytes (161 tokens on 32 heads, e4m3: 6.6 us for 10.5 MB of lines
// in which 0.66 MB change; with eight neighbouring head dims to a thread, every store 64 lines, 8.9).
// ---------------------------------------------------------------------------------------------
constexpr int kAppendBlocks = kPrefillTileQ / 32 + 1;        // blocks that 128 tokens may touch

template <int D, bool E4M3>
__global__ __launch_bounds__(256) void paged_append_kernel(const bf16* __restrict__ k, size_t k_stride, const bf16* __restrict__ v,
                                                           size_t v_stride, PagedRope rope, BatchView bv, PagedView kv,
                                                           int heads_per_wg, int hgroups, int block_wgs, int row_wgs) {
    typedef Blocks<D, E4M3> B;
    const int Hkv = kv.Hkv, tid = threadIdx.x;
    constexpr int EL = E4M3 ? 1 : 2;
    uint8_t* kc = static_cast<uint8_t*>(kv.k);
    uint8_t* vc = static_cast<uint8_t*>(kv.v);
    if ((int)blockIdx.x >= block_wgs) {
        const int b = blockIdx.x - block_wgs, i = b / row_wgs, s = bv.decode_seqs[i];
        int unit = (b - i * row_wgs) * 256 + tid;
        const int t = bv.q_start[s], pos = bv.kv_before[s], p = pos & 31;
        const int id = page_of(kv, bv.seq_slot[s], pos);
        if (id < 0) return;
        constexpr int KU = D / 16, VU = D / 8;               // units of a head
        if (unit < Hkv * KU) {
            const int head = unit / KU, j = (unit - head * KU) * 8;
            const bf16* src = k + (size_t)t * k_stride + head * D + j;
            float lo[8], hi[8];
            load_row(src, lo);
            load_row(src + D / 2, hi);
            if (rope.tab) rotate(lo, hi, rope_row(rope, pos, D) + 2 * j);
            const size_t at = block_base(kv, id, head, pos);
            if constexpr (E4M3) {
                uint2 a, c;
                a.x = pack4(lo, 0, kv.k_scale, kv.k_inv);
                a.y = pack4(lo, 4, kv.k_scale, kv.k_inv);
                c.x = pack4(hi, 0, kv.k_scale, kv.k_inv);
                c.y = pack4(hi, 4, kv.k_scale, kv.k_inv);
                *reinterpret_cast<uint2*>(kc + at + k_block_offset<true>(p, j)) = a;
                *reinterpret_cast<uint2*>(kc + at + k_block_offset<true>(p, D / 2 + j)) = c;
            } else {
                *reinterpret_cast<u32x4*>(kc + (at + k_block_offset<false>(p, j)) * 2) = pack<false>(lo, 1.f, 1.f);
                *reinterpret_cast<u32x4*>(kc + (at + k_block_offset<false>(p, D / 2 + j)) * 2) = pack<false>(hi, 1.f, 1.f);
            }
        } else if ((unit -= Hkv * KU) < Hkv * VU) {
            // neighbouring threads have neighbouring head dims: a wave's store touches few lines
            const int head = unit / VU, j = unit - head * VU;
            const bf16* src = v + (size_t)t * v_stride + head * D + j;
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (float)src[e * VU];
            const size_t at = block_base(kv, id, head, pos);
#pragma unroll
            for (int e = 0; e < 8; ++e) cache_put<E4M3>(kv.v, at + v_block_offset<E4M3>(p, j + e * VU, D), E4M3 ? quotient(x[e], kv.v_scale, kv.v_inv) : x[e]);
        }
        return;
    }
    const int item = blockIdx.x / (kAppendBlocks * hgroups);
    const int rest = blockIdx.x - item * (kAppendBlocks * hgroups);
    const int sub = rest / hgroups, hg = rest - sub * hgroups;
    const int s = bv.prefill_items[2 * item], qt = bv.prefill_items[2 * item + 1];
    const int q0 = bv.q_start[s], qlen = bv.q_start[s + 1] - q0;
    // the item's last block is the next one's first
    if (sub == kAppendBlocks - 1 && (qt + 1) * kPrefillTileQ < qlen) return;
    const int before = bv.kv_before[s], end = before + qlen;
    const int first = ((before >> 5) + qt * (kPrefillTileQ / 32) + sub) * 32;      // of the block
    const int p_lo = first > before ? first : before, p_hi = first + 32 < end ? first + 32 : end;
    if (p_lo >= p_hi) return;
    const int id = page_of(kv, bv.seq_slot[s], first);
    if (id < 0) return;
    const int hsub = tid / B::THREADS, ht = tid - hsub * B::THREADS;
    const int h0 = hg * heads_per_wg + hsub;
    const int h1 = (hg + 1) * heads_per_wg < Hkv ? (hg + 1) * heads_per_wg : Hkv;
    const size_t head_bytes = ((size_t)D << kv.page_shift) * EL, base = block_base(kv, id, 0, first) * EL;

    const int kp = ht / B::UNITS, unit = ht - kp * B::UNITS;
    const bool k_in = first + kp >= p_lo && first + kp < p_hi;
    const int kpos = k_in ? first + kp : p_lo;               // read in bounds, not stored
    const float* cs = rope.tab ? rope_row(rope, kpos, D) + unit * (2 * B::VEC) : nullptr;
    const bf16* krow = k + (size_t)(q0 + kpos - before) * k_stride + unit * B::VEC;
    const int w = ht / (D / 2), j = (ht - w * (D / 2)) * 2;
    for (int h = h0; h < h1; h += B::PAR) {
        float lo[B::VEC], hi[B::VEC];
        load_row(krow + h * D, lo);
        load_row(krow + h * D + D / 2, hi);
        bf16x2 r[B::VEC];
#pragma unroll
        for (int e = 0; e < B::VEC; ++e) {
            int pe = first + B::v_pos(w, e);
            pe = pe < p_lo ? p_lo : pe > p_hi - 1 ? p_hi - 1 : pe;
            r[e] = *reinterpret_cast<const bf16x2*>(v + (size_t)(q0 + pe - before) * v_stride + h * D + j);
        }
        if (cs) rotate(lo, hi, cs);
        uint8_t* kd = kc + base + h * head_bytes + kp * 16;
        if (k_in) {
            *reinterpret_cast<u32x4*>(kd + unit * 512) = pack<E4M3>(lo, kv.k_scale, kv.k_inv);
            *reinterpret_cast<u32x4*>(kd + (unit + B::UNITS) * 512) = pack<E4M3>(hi, kv.k_scale, kv.k_inv);
        }
        float x[B::VEC], y[B::VEC];
        bool all = true;
#pragma unroll
        for (int e = 0; e < B::VEC; ++e) {
            x[e] = (float)r[e][0];
            y[e] = (float)r[e][1];
            const int pe = first + B::v_pos(w, e);
            all &= pe >= p_lo && pe < p_hi;
        }
        const u32x4 px = pack<E4M3>(x, kv.v_scale, kv.v_inv), py = pack<E4M3>(y, kv.v_scale, kv.v_inv);
        uint8_t* vd = vc + base + h * head_bytes + (w * D + j) * 16;
        if (all) {
            *reinterpret_cast<u32x4*>(vd) = px;
            *reinterpret_cast<u32x4*>(vd + 16) = py;
        } else {
#pragma unroll
            for (int e = 0; e < B::VEC; ++e) {
                const int pe = first + B::v_pos(w, e);
                if (pe < p_lo || pe >= p_hi) continue;
                if constexpr (E4M3) {
                    vd[e] = (uint8_t)(px[e >> 2] >> (8 * (e & 3)));
                    vd[16 + e] = (uint8_t)(py[e >> 2] >> (8 * (e & 3)));
                } else {
                    reinterpret_cast<bf16*>(vd)[e] = r[e][0];
                    reinterpret_cast<bf16*>(vd)[8 + e] = r[e][1];
                }
            }
        }
    }
}

// heads of one workgroup: as many as leave some thousand workgroups, up to `most`
static int heads_together(int64_t blocks, int Hkv, int par, int most) {
    const int64_t n = blocks * Hkv / 4096;
    const int h = n < par ? par : n > most ? most : (int)n;
    return (h + par - 1) / par * par;
}

struct AppendGrid {
    int heads_per_wg, hgroups, row_wgs;
    int64_t block_wgs, all;
};
template <int D, bool E4M3>
static AppendGrid append_grid(const BatchView& bv, const PagedView& kv) {
    AppendGrid g;
    const int64_t blocks = (int64_t)bv.n_prefill_items * kAppendBlocks;
    g.heads_per_wg = heads_together(blocks, kv.Hkv, Blocks<D, E4M3>::PAR, 8);
    g.hgroups = (kv.Hkv + g.heads_per_wg - 1) / g.heads_per_wg;
    g.row_wgs = (kv.Hkv * (D / 16 + D / 8) + 255) / 256;
    g.block_wgs = blocks * g.hgroups;
    g.all = g.block_wgs + (int64_t)bv.n_decode * g.row_wgs;
    return g;
}
static AppendGrid append_grid(bool e4m3, const BatchView& bv, const PagedView& kv) {
    auto grid = kv.d == 128 ? (e4m3 ? append_grid<128, true> : append_grid<128, false>) : (e4m3 ? append_grid<64, true> : append_grid<64, false>);
    return grid(bv, kv);
}
bool paged_append_fits(bool e4m3, const BatchView& bv, const PagedView& kv) { return append_grid(e4m3, bv, kv).all <= kMaxWorkgroups; }

template <int D, bool E4M3>
static void launch_append(const act_t* k, size_t k_stride, const act_t* v, size_t v_stride, const PagedRope& rope, const BatchView& bv,
                          const PagedView& kv, hipStream_t st) {
    const AppendGrid g = append_grid<D, E4M3>(bv, kv);
    if (g.all > 0)
        hipLaunchKernelGGL((paged_append_kernel<D, E4M3>), dim3((unsigned)g.all), dim3(256), 0, st, k, k_stride, v, v_stride, rope, bv, kv,
                           g.heads_per_wg, g.hgroups, (int)g.block_wgs, g.row_wgs);
}

void launch_paged_append(const act_t* k, size_t k_stride, const act_t* v, size_t v_stride, const PagedRope& rope, bool e4m3,
                         const BatchView& bv, const PagedView& kv, hipStream_t st) {
    auto go = kv.d == 128 ? (e4m3 ? launch_append<128, true> : launch_append<128, false>) : (e4m3 ? launch_append<64, true> : launch_append<64, false>);
    go(k, k_stride, v, v_stride, rope, bv, kv, st);
}

// ---------------------------------------------------------------------------------------------
// Read: one workgroup per block of 32 positions and `heads_per_wg` heads.  Bound by bytes (16000
// positions on 40 heads, e4m3 to bf16: 103 us, 4.8 TB/s, what a large copy has).
// ---------------------------------------------------------------------------------------------
template <int D, bool E4M3>
__global__ __launch_bounds__(256) void paged_read_kernel(PagedView kv, int row, int pos0, int n, bf16* __restrict__ k, bf16* __restrict__ v,
                                                         int heads_per_wg, int hgroups) {
    typedef Blocks<D, E4M3> B;
    constexpr int EL = E4M3 ? 1 : 2;
    const int Hkv = kv.Hkv, tid = threadIdx.x;
    const int blk = blockIdx.x / hgroups, hg = blockIdx.x - blk * hgroups;
    const int first = ((pos0 >> 5) + blk) * 32;
    const int p_lo = first > pos0 ? first : pos0, p_hi = first + 32 < pos0 + n ? first + 32 : pos0 + n;
    const int id = page_of(kv, row, first);                  // block-uniform
    const int hsub = tid / B::THREADS, ht = tid - hsub * B::THREADS;
    const int h0 = hg * heads_per_wg + hsub;
    const int h1 = (hg + 1) * heads_per_wg < Hkv ? (hg + 1) * heads_per_wg : Hkv;
    const size_t head_bytes = ((size_t)D << kv.page_shift) * EL, base = block_base(kv, id < 0 ? 0 : id, 0, first) * EL;
    const size_t pitch = (size_t)Hkv * D;

    const int kp = ht / B::UNITS, unit = ht - kp * B::UNITS, w = ht / (D / 2), j = (ht - w * (D / 2)) * 2;
    const bool k_in = first + kp >= p_lo && first + kp < p_hi;
    bf16* kd = k + (size_t)(k_in ? first + kp - pos0 : 0) * pitch + unit * B::VEC;
    for (int h = h0; h < h1; h += B::PAR) {
        const uint8_t* ks = static_cast<const uint8_t*>(kv.k) + base + h * head_bytes + kp * 16;
        const uint8_t* vs = static_cast<const uint8_t*>(kv.v) + base + h * head_bytes + (w * D + j) * 16;
        u32x4 a = {}, b = {}, c = {}, d = {};
        if (id >= 0) {
            a = *reinterpret_cast<const u32x4*>(ks + unit * 512);
            b = *reinterpret_cast<const u32x4*>(ks + (unit + B::UNITS) * 512);
            c = *reinterpret_cast<const u32x4*>(vs);
            d = *reinterpret_cast<const u32x4*>(vs + 16);
        }
        float x[B::VEC], y[B::VEC];
        unpack<E4M3>(a, kv.k_scale, x);
        unpack<E4M3>(b, kv.k_scale, y);
        if (k_in) {
#pragma unroll
            for (int i = 0; i < B::VEC; i += 8) {
                bf16x8 lo, hi;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    lo[e] = (bf16)x[i + e];
                    hi[e] = (bf16)y[i + e];
                }
                *reinterpret_cast<bf16x8*>(kd + h * D + i) = lo;
                *reinterpret_cast<bf16x8*>(kd + h * D + D / 2 + i) = hi;
            }
        }
        unpack<E4M3>(c, kv.v_scale, x);
        unpack<E4M3>(d, kv.v_scale, y);
#pragma unroll
        for (int e = 0; e < B::VEC; ++e) {
            const int pe = first + B::v_pos(w, e);
            const bf16x2 r = {(bf16)x[e], (bf16)y[e]};
            if (pe >= p_lo && pe < p_hi) *reinterpret_cast<bf16x2*>(v + (size_t)(pe - pos0) * pitch + h * D + j) = r;
        }
    }
}

static int read_blocks(int pos0, int n) { return ((pos0 + n - 1) >> 5) - (pos0 >> 5) + 1; }

template <int D, bool E4M3>
static void launch_read(const PagedView& kv, int row, int pos0, int n, act_t* k, act_t* v, hipStream_t st) {
    const int blocks = read_blocks(pos0, n);
    const int hpw = heads_together(blocks, kv.Hkv, Blocks<D, E4M3>::PAR, 8), hgroups = (kv.Hkv + hpw - 1) / hpw;
    hipLaunchKernelGGL((paged_read_kernel<D, E4M3>), dim3(blocks * hgroups), dim3(256), 0, st, kv, row, pos0, n, k, v, hpw, hgroups);
}

bool paged_read_fits(bool e4m3, const PagedView& kv, int pos0, int n) {
    const int64_t blocks = read_blocks(pos0, n);
    const int par = kv.d == 128 ? (e4m3 ? Blocks<128, true>::PAR : Blocks<128, false>::PAR) : (e4m3 ? Blocks<64, true>::PAR : Blocks<64, false>::PAR);
    const int hpw = heads_together(blocks, kv.Hkv, par, 8);
    return blocks * ((kv.Hkv + hpw - 1) / hpw) <= kMaxWorkgroups;
}

void launch_paged_read(bool e4m3, const PagedView& kv, int row, int pos0, int n, act_t* k, act_t* v, hipStream_t st) {
    auto go = kv.d == 128 ? (e4m3 ? launch_read<128, true> : launch_read<128, false>) : (e4m3 ? launch_read<64, true> : launch_read<64, false>);
    go(kv, row, pos0, n, k, v, st);
}

#else  // BZ_FP32_DEBUG: one workgroup per token, or position

template <bool E4M3>
__global__ __launch_bounds__(256) void paged_append_kernel(const act_t* __restrict__ k, size_t k_stride, const act_t* __restrict__ v,
                                                           size_t v_stride, PagedRope rope, BatchView bv, PagedView kv) {
    const int t = blockIdx.x, s = bv.token_seq[t];
    const int pos = bv.kv_before[s] + (t - bv.q_start[s]), p = pos & 31;
    const int id = page_of(kv, bv.seq_slot[s], pos);
    if (id < 0) return;
    const int d = kv.d, half = d >> 1;
    const act_t* kr = k + (size_t)t * k_stride;
    const act_t* vr = v + (size_t)t * v_stride;
    const float* cs = rope.tab ? rope_row(rope, pos, d) : nullptr;
    for (int u = threadIdx.x; u < kv.Hkv * half; u += 256) {
        const int head = u / half, j = u - head * half;
        const size_t at = block_base(kv, id, head, pos);
        const float lo = to_f32(kr[head * d + j]), hi = to_f32(kr[head * d + half + j]);
        const float c = cs ? cs[2 * j] : 1.f, sn = cs ? cs[2 * j + 1] : 0.f;
        const float o_lo = cs ? lo * c - hi * sn : lo, o_hi = cs ? hi * c + lo * sn : hi;
        cache_put<E4M3>(kv.k, at + k_block_offset<E4M3>(p, j), E4M3 ? quotient(o_lo, kv.k_scale, kv.k_inv) : o_lo);
        cache_put<E4M3>(kv.k, at + k_block_offset<E4M3>(p, half + j), E4M3 ? quotient(o_hi, kv.k_scale, kv.k_inv) : o_hi);
    }
    for (int u = threadIdx.x; u < kv.Hkv * d; u += 256) {
        const int head = u / d, j = u - head * d;
        const float x = to_f32(vr[u]);
        cache_put<E4M3>(kv.v, block_base(kv, id, head, pos) + v_block_offset<E4M3>(p, j, d), E4M3 ? quotient(x, kv.v_scale, kv.v_inv) : x);
    }
}

bool paged_append_fits(bool, const BatchView& bv, const PagedView&) { return bv.T <= kMaxWorkgroups; }

void launch_paged_append(const act_t* k, size_t k_stride, const act_t* v, size_t v_stride, const PagedRope& rope, bool e4m3,
                         const BatchView& bv, const PagedView& kv, hipStream_t st) {
    auto kern = e4m3 ? paged_append_kernel<true> : paged_append_kernel<false>;
    hipLaunchKernelGGL(kern, dim3(bv.T), dim3(256), 0, st, k, k_stride, v, v_stride, rope, bv, kv);
}

template <bool E4M3>
__global__ __launch_bounds__(256) void paged_read_kernel(PagedView kv, int row, int pos0, act_t* __restrict__ k, act_t* __restrict__ v) {
    const int i = blockIdx.x, pos = pos0 + i, p = pos & 31, d = kv.d;
    const int id = page_of(kv, row, pos);
    for (int u = threadIdx.x; u < kv.Hkv * d; u += 256) {
        const int head = u / d, j = u - head * d;
        const size_t at = id < 0 ? 0 : block_base(kv, id, head, pos);
        const float kx = id < 0 ? 0.f : cache_get<E4M3>(kv.k, at + k_block_offset<E4M3>(p, j)) * kv.k_scale;
        const float vx = id < 0 ? 0.f : cache_get<E4M3>(kv.v, at + v_block_offset<E4M3>(p, j, d)) * kv.v_scale;
        from_f32(k[(size_t)i * kv.Hkv * d + u], kx);
        from_f32(v[(size_t)i * kv.Hkv * d + u], vx);
    }
}

bool paged_read_fits(bool, const PagedView&, int, int n) { return n <= kMaxWorkgroups; }

void launch_paged_read(bool e4m3, const PagedView& kv, int row, int pos0, int n, act_t* k, act_t* v, hipStream_t st) {
    auto kern = e4m3 ? paged_read_kernel<true> : paged_read_kernel<false>;
    hipLaunchKernelGGL(kern, dim3(n), dim3(256), 0, st, kv, row, pos0, k, v);
}
#endif

}  // namespace bz
