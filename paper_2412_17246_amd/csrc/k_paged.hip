// Operations on the paged KV cache that move it: the append of a batch's new tokens with the rotation on the way, and the way
// back out.
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

}  // namespace bz
