// Host side of the paged KV cache's operations: argument checks and launches.
#include <math.h>

#include <algorithm>
#include <cmath>
#include <vector>

#include "instance.h"
#include "paged.h"

using namespace bz;

namespace {

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

bool shape_ok(const bz_paged_kv* kv) {
    if (!kv || kv->n_pages < 1 || kv->n_rows < 1 || kv->pages_per_row < 1 || kv->n_kv_heads < 1 || kv->n_kv_heads > 1024) return false;
    if (kv->page_size < 32 || kv->page_size > 1024 || (kv->page_size & (kv->page_size - 1))) return false;
    if ((int64_t)kv->pages_per_row * kv->page_size > 1 << 30) return false;     // positions, and a few thousand more, are 32-bit numbers
    if ((int64_t)kv->n_pages * kv->n_kv_heads * (kv->page_size / 32) > 0x7fffffffLL) return false;    // blocks have 32-bit numbers
    if (kv->head_dim != 64 && kv->head_dim != 128) return false;
    if (kv->dtype == BZ_KV_E4M3) return kv->k_scale > 0.f && kv->v_scale > 0.f && std::isfinite(kv->k_scale) && std::isfinite(kv->v_scale) &&
                                        std::isfinite(1.f / kv->k_scale) && std::isfinite(1.f / kv->v_scale);
    return kv->dtype == BZ_KV_ACT && kv->k_scale == 1.f && kv->v_scale == 1.f;
}

bool cache_ok(const bz_paged_kv* kv) {
    return shape_ok(kv) && kv->k && kv->v && aligned16(kv->k) && aligned16(kv->v) && kv->page_table && !((uintptr_t)kv->page_table & 3);
}

bool rows_ok(const void* p, int64_t stride, int64_t width) {
    return p && aligned16(p) && stride >= width && stride % 8 == 0;
}

bool rope_ok(const float* rope, int positions) { return !rope || (aligned16(rope) && positions >= 1); }

PagedView view_of(const bz_paged_kv* kv) {
    PagedView v;
    v.k = kv->k;
    v.v = kv->v;
    v.table = kv->page_table;
    v.n_pages = kv->n_pages;
    v.per_row = kv->pages_per_row;
    v.page_shift = __builtin_ctz((unsigned)kv->page_size);
    v.Hkv = kv->n_kv_heads;
    v.d = kv->head_dim;
    v.k_scale = kv->k_scale;
    v.v_scale = kv->v_scale;
    v.k_inv = 1.f / kv->k_scale;
    v.v_inv = 1.f / kv->v_scale;
    return v;
}

// every sequence with new tokens has a row of the table, and the row and the rotary table reach as far as it does
int lengths_ok(const bz_batch* b, const bz_paged_kv* kv, const float* rope, int rope_positions) {
    const int64_t room = (int64_t)kv->pages_per_row * kv->page_size;
    for (int s = 0; s < b->B; ++s) {
        const int n = b->q_start[s + 1] - b->q_start[s];
        if (n == 0) continue;
        if (b->seq_slot[s] >= kv->n_rows) return BZ_EINVAL;
        const int64_t end = (int64_t)b->kv_before[s] + n;
        if (end > room || (rope && end > rope_positions)) return BZ_ECAPACITY;
    }
    return BZ_OK;
}

int chunks_of(int64_t keys) { return (int)((keys + kDecodeChunk - 1) / kDecodeChunk); }

// keys that the tokens of a sequence see between them, from a multiple of 64 on
int64_t keys_of(int64_t before, int64_t n, int window) {
    const int64_t lo = window && before + 1 > window ? (before + 1 - window) & ~(int64_t)63 : 0;
    return before + n - lo;
}

PagedWork work_of(const bz_batch* b, const BatchView& bv, int Hq, int Hkv, int window) {
    PagedWork w{};
    const int G = Hq / Hkv;
    int64_t most = 0;
    w.narrow_limit = b->short_qlen.empty() ? 0 : kNarrowRows;       // a batch in tight storage has no list of them
    while (w.n_short < (int)b->short_qlen.size() && b->short_qlen[w.n_short] * G <= kNarrowRows) ++w.n_short;
    w.short_tokens = w.n_short ? b->short_qlen[w.n_short - 1] : 0;
    for (int i = 0; i < w.n_short; ++i) most = std::max(most, keys_of(b->kv_before[b->short_seqs[i]], b->short_qlen[i], window));
    if (window)
        for (int s : b->decode_seqs) most = std::max(most, keys_of(b->kv_before[s], 1, window));
    w.col_tiles = (std::max(G, 1) + kNarrowRows - 1) / kNarrowRows;
    w.narrow_rows = std::max(std::min(G, kNarrowRows), w.short_tokens * G);
    w.list = window ? 0 : bv.n_decode_work;
    w.first = window ? 0 : bv.n_decode;
    w.chunks = chunks_of(most);
    w.max_chunks = std::max(w.chunks, window ? 0 : bv.decode_chunks);
    int64_t units = 0, keys = 0;
    for (int s = 0; s < b->B; ++s) {
        const int n = b->q_start[s + 1] - b->q_start[s];
        if (n < 2 || (int64_t)n * G <= w.narrow_limit) continue;
        const int64_t rows = (int64_t)n * G;
        units += (rows + kWideRows - 1) / kWideRows * Hkv;
        keys = std::max(keys, keys_of((int64_t)b->kv_before[s] + n - std::min<int64_t>(n, kWideRows / G + 1), std::min<int64_t>(n, kWideRows / G + 1), window));
    }
    // Ranges of the keys: one workgroup per CU, or two where a range keeps twelve tiles of 64 keys.  Two on a CU hide each other's waits,
    // but every range costs its rows' partial results twice; and one range, which needs none, has a launch less, too.
    // (us with 256 / 512 workgroups: 128 rows on 8000 keys 38 / 44, 512 on 3001 53 / 53, 16 drafts of 10 to 16 tokens 79 / 57,
    // 1000 rows on 2000 keys, 250 workgroups in one range, 67 / 70.)
    const int64_t tiles = (keys + 63) / 64;
    const auto ranges = [&](int64_t n) { return units ? std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(n / units, 16), tiles / 4)) : 1; };
    w.splits = (int)ranges(256);
    if (tiles >= 12 * ranges(512) && (w.splits > 1 || tiles >= 64)) w.splits = (int)ranges(512);
    w.wide_units = (int)std::min<int64_t>(units, 0x7fffffff);
    w.by_heads = divisor(Hkv * w.col_tiles);
    w.by_chunks = divisor(std::max(w.chunks, 1));
    w.by_tiles = divisor(w.col_tiles);
    w.by_group = divisor(G);
    return w;
}

int launched(const bz_batch* b, hipStream_t st) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return hip_fail(e, "launch");
    return batch_after_run(b, st, false);
}

}  // namespace

extern "C" {

size_t bz_paged_kv_bytes(const bz_paged_kv* kv) {
    if (!shape_ok(kv)) return 0;
    return (size_t)kv->n_pages * kv->n_kv_heads * kv->page_size * kv->head_dim * (kv->dtype == BZ_KV_E4M3 ? 1 : sizeof(act_t));
}

int bz_rope_table(int positions, int head_dim, float base, float* out) try {
    if (positions < 1 || head_dim < 2 || head_dim % 2 || !(base > 1.f) || !std::isfinite(base) || !out) return BZ_EINVAL;
    const int half = head_dim / 2;
    std::vector<double> theta(half);
    for (int j = 0; j < half; ++j) theta[j] = pow((double)base, -2.0 * j / head_dim);
    for (int p = 0; p < positions; ++p)
        for (int j = 0; j < half; ++j) {
            const double a = (double)p * theta[j];
            out[((size_t)p * half + j) * 2] = (float)cos(a);
            out[((size_t)p * half + j) * 2 + 1] = (float)sin(a);
        }
    return BZ_OK;
} catch (...) {
    return BZ_ENOMEM;
}

int bz_op_paged_append(const bz_batch* batch, const bz_paged_kv* kv, const void* k, int64_t k_stride, const void* v,
                       int64_t v_stride, const float* rope, int rope_positions, void* stream) try {
    if (!batch || !cache_ok(kv) || !rope_ok(rope, rope_positions)) return BZ_EINVAL;
    const int64_t width = (int64_t)kv->n_kv_heads * kv->head_dim;
    if (!rows_ok(k, k_stride, width) || !rows_ok(v, v_stride, width)) return BZ_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    int rc = lengths_ok(batch, kv, rope, rope_positions);
    if (rc) return rc;
    const BatchView bv = batch_view(batch);
    const PagedView view = view_of(kv);
    const bool e4m3 = kv->dtype == BZ_KV_E4M3;
    if (!paged_append_fits(e4m3, bv, view)) return BZ_ECAPACITY;
    rc = batch_before_run(batch, st);
    if (rc) return rc;
    launch_paged_append((const act_t*)k, (size_t)k_stride, (const act_t*)v, (size_t)v_stride, PagedRope{rope, rope_positions},
                        e4m3, bv, view, st);
    return launched(batch, st);
} catch (...) {
    return BZ_ENOMEM;
}

size_t bz_op_paged_attention_workspace_bytes(const bz_batch* batch, const bz_paged_kv* kv, int n_q_heads, int window) {
    if (!batch || !shape_ok(kv) || n_q_heads < 1 || n_q_heads % kv->n_kv_heads || n_q_heads > 1024 || window < 0) return 0;
    const BatchView bv = batch_view(batch);
    return paged_attention_bytes(work_of(batch, bv, n_q_heads, kv->n_kv_heads, window), bv, n_q_heads, kv->n_kv_heads, kv->head_dim);
}

int bz_op_paged_attention(const bz_batch* batch, const bz_paged_kv* kv, const void* q, int64_t q_stride, void* out,
                          int64_t out_stride, int n_q_heads, float scale, int window, const float* rope, int rope_positions,
                          void* workspace, size_t workspace_bytes, void* stream) try {
    if (!batch || !cache_ok(kv) || !rope_ok(rope, rope_positions)) return BZ_EINVAL;
    if (n_q_heads < 1 || n_q_heads % kv->n_kv_heads || n_q_heads > 1024 || window < 0) return BZ_EINVAL;
    if (!(scale >= 0.f)) return BZ_EINVAL;
    // of scores in base 2; a product that vanished would make a NaN of a masked score
    const float scale_log2 = (scale > 0.f ? scale : 1.f / sqrtf((float)kv->head_dim)) * 1.4426950408889634f * kv->k_scale;
    if (!std::isnormal(scale_log2)) return BZ_EINVAL;
    const int64_t width = (int64_t)n_q_heads * kv->head_dim;
    if (!rows_ok(q, q_stride, width) || !rows_ok(out, out_stride, width)) return BZ_EINVAL;
    if (q == out && q_stride != out_stride && batch->T > 1) return BZ_EINVAL;      // a row would overwrite another's query
    if (workspace && !aligned16(workspace)) return BZ_EINVAL;
    hipStream_t st = (hipStream_t)stream;
    int rc = lengths_ok(batch, kv, rope, rope_positions);
    if (rc) return rc;
    const BatchView bv = batch_view(batch);
    const PagedWork work = work_of(batch, bv, n_q_heads, kv->n_kv_heads, window);
    if (!paged_attention_fits(work, bv, n_q_heads, kv->n_kv_heads)) return BZ_ECAPACITY;
    const size_t need = paged_attention_bytes(work, bv, n_q_heads, kv->n_kv_heads, kv->head_dim);
    if (need && (!workspace || workspace_bytes < need)) return BZ_ENOMEM;
    rc = batch_before_run(batch, st);
    if (rc) return rc;
    PagedQuery a;
    a.q = (const act_t*)q;
    a.out = (act_t*)out;
    a.q_stride = (size_t)q_stride;
    a.out_stride = (size_t)out_stride;
    a.rope = PagedRope{rope, rope_positions};
    a.Hq = n_q_heads;
    a.window = window;
    a.scale_log2 = scale_log2;
    launch_paged_attention(a, work, kv->dtype == BZ_KV_E4M3, bv, view_of(kv), (float*)workspace, st);
    return launched(batch, st);
} catch (...) {
    return BZ_ENOMEM;
}

int bz_op_paged_read(const bz_paged_kv* kv, int row, int pos0, int n, void* k, void* v, void* stream) {
    if (!cache_ok(kv) || row < 0 || row >= kv->n_rows || pos0 < 0 || n < 0) return BZ_EINVAL;
    if ((int64_t)pos0 + n > (int64_t)kv->pages_per_row * kv->page_size) return BZ_ECAPACITY;
    if (n == 0) return BZ_OK;
    if (!k || !v || !aligned16(k) || !aligned16(v)) return BZ_EINVAL;
    if (!paged_read_fits(kv->dtype == BZ_KV_E4M3, view_of(kv), pos0, n)) return BZ_ECAPACITY;
    launch_paged_read(kv->dtype == BZ_KV_E4M3, view_of(kv), row, pos0, n, (act_t*)k, (act_t*)v, (hipStream_t)stream);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? BZ_OK : hip_fail(e, "launch");
}

}  // extern "C"
