// Operations on the paged KV cache that move it: the append of a batch's new tokens with the rotation on the way, and the way
// back out.  Plain attention over the pages, one wave per (token, query head).
#include "paged.h"

namespace bz {

// ---------------------------------------------------------------------------------------------
// Append: one workgroup per new token, a thread per rotation pair and per value.
// ---------------------------------------------------------------------------------------------
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
        cache_put<E4M3>(kv.k, at + k_block_offset<E4M3>(p, j), E4M3 ? o_lo * kv.k_inv : o_lo);
        cache_put<E4M3>(kv.k, at + k_block_offset<E4M3>(p, half + j), E4M3 ? o_hi * kv.k_inv : o_hi);
    }
    for (int u = threadIdx.x; u < kv.Hkv * d; u += 256) {
        const int head = u / d, j = u - head * d;
        const float x = to_f32(vr[u]);
        cache_put<E4M3>(kv.v, block_base(kv, id, head, pos) + v_block_offset<E4M3>(p, j, d), E4M3 ? x * kv.v_inv : x);
    }
}

void launch_paged_append(const act_t* k, size_t k_stride, const act_t* v, size_t v_stride, const PagedRope& rope, bool e4m3,
                         const BatchView& bv, const PagedView& kv, hipStream_t st) {
    auto kern = e4m3 ? paged_append_kernel<true> : paged_append_kernel<false>;
    hipLaunchKernelGGL(kern, dim3(bv.T), dim3(256), 0, st, k, k_stride, v, v_stride, rope, bv, kv);
}

// ---------------------------------------------------------------------------------------------
// Read: one workgroup per position.
// ---------------------------------------------------------------------------------------------
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

void launch_paged_read(bool e4m3, const PagedView& kv, int row, int pos0, int n, act_t* k, act_t* v, hipStream_t st) {
    auto kern = e4m3 ? paged_read_kernel<true> : paged_read_kernel<false>;
    hipLaunchKernelGGL(kern, dim3(n), dim3(256), 0, st, kv, row, pos0, k, v);
}

// ---------------------------------------------------------------------------------------------
// Attention, plain: one wave per (token, query head), 64 positions at a time with a running maximum and sum; a lane scores one
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

size_t paged_attention_bytes(const PagedWork&, const BatchView&, int, int, int) { return 0; }

void launch_paged_attention(const PagedQuery& a, const PagedWork&, bool e4m3, const BatchView& bv, const PagedView& kv, float*,
                            hipStream_t st) {
    auto kern = kv.d == 128 ? (e4m3 ? paged_attn_plain_kernel<true, 128> : paged_attn_plain_kernel<false, 128>)
                            : (e4m3 ? paged_attn_plain_kernel<true, 64> : paged_attn_plain_kernel<false, 64>);
    hipLaunchKernelGGL(kern, dim3(bv.T, a.Hq), dim3(64), 0, st, a, bv, kv);
}

}  // namespace bz
