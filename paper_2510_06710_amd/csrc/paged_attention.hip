// Attention of a ragged batch's new rows against a paged KV cache.
#include "paged.h"

namespace {

struct AttnArgs {
    PagedView pv;
    const char *q;
    char *out;
    float *lse;
    long q_stride, o_stride;
    int n_heads, group;
    float scale, cap;
    const float *slopes;
    const int32_t *prefix_len;
    int window, shared_len;
};

// One wave per (row, head), the dims over its lanes, one key after the other.
template <typename T>
__global__ void __launch_bounds__(64) paged_attention_simple_kernel(AttnArgs a) {
    const PagedView &pv = a.pv;
    const int row = blockIdx.x, h = blockIdx.y, lane = threadIdx.x, d = pv.d;
    const int s = paged_seq_of_row(pv, row);
    if (s >= pv.n_seq) return;
    const PagedSeq sq = paged_seq(pv, s);
    const int i = row - sq.r0, p = sq.len - sq.n + i;
    if (i < 0 || i >= sq.rows) return;
    const int prefix = a.prefix_len ? min(a.prefix_len[s], sq.keys) : 0;
    const int hi = p < 0 ? 0 : min(sq.keys, max(p + 1, prefix)), lo = a.window ? max(0, p + 1 - a.window) : 0, kh = h / a.group;
    float q[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
    for (int e = 0; e < 4; e++) q[e] = lane + 64 * e < d ? (float)((const T *)a.q)[row * a.q_stride + (size_t)h * d + lane + 64 * e] : 0.f;
    for (int j = 0; j < hi; j++) {
        if (!((j <= p && j >= lo) || j < prefix)) continue;
        const int page = pv.table[(size_t)(j < a.shared_len ? 0 : s) * pv.table_stride + (j >> pv.page_log)];
        const bool ok = (unsigned)page < (unsigned)pv.n_pages;
        const size_t at = ((((size_t)(ok ? page : 0) * pv.n_kv + kh) << pv.page_log) + (j & ((1 << pv.page_log) - 1))) * d;
        float x = 0.f, v[4];
        for (int e = 0; e < 4; e++) {
            const bool in = ok && lane + 64 * e < d;
            x += in ? q[e] * (float)((const T *)pv.k)[at + lane + 64 * e] : 0.f;
            v[e] = in ? (float)((const T *)pv.v)[at + lane + 64 * e] : 0.f;
        }
        x = vla_wave_sum(x) * a.scale;
        if (a.cap > 0.f) x = a.cap * tanhf(x / a.cap);
        if (a.slopes) x -= a.slopes[h] * (float)abs(p - j);
        const float top = fmaxf(m, x), f = expf(m - top), w = expf(x - top);
        l = l * f + w;
        for (int e = 0; e < 4; e++) o[e] = o[e] * f + w * v[e];
        m = top;
    }
    for (int e = 0; e < 4; e++)
        if (lane + 64 * e < d) ((T *)a.out)[row * a.o_stride + (size_t)h * d + lane + 64 * e] = (T)(l > 0.f ? o[e] / l : 0.f);
    if (a.lse && lane == 0) a.lse[(size_t)row * a.n_heads + h] = l > 0.f ? m + logf(l) : -INFINITY;
}

int check(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_paged_mask *mask, int n_heads, AttnArgs *a) {
    if (int rc = vla_check_paged("paged_attention", cache, batch, &a->pv)) return rc;
    if (!mask) { vla_set_error("paged_attention: mask is NULL"); return VLA_EINVAL; }
    if (n_heads <= 0 || n_heads % cache->n_kv_heads) {
        vla_set_error("paged_attention: n_heads %d is no multiple of n_kv_heads %d", n_heads, cache->n_kv_heads);
        return VLA_ESHAPE;
    }
    if (n_heads > 4096) { vla_set_error("paged_attention: n_heads %d unsupported (at most 4096)", n_heads); return VLA_ESHAPE; }
    if (!(mask->scale > 0.f) || !(mask->softcap >= 0.f) || !(mask->scale < INFINITY) || !(mask->softcap < INFINITY)) {
        vla_set_error("paged_attention: scale must be positive, softcap not negative, both finite");
        return VLA_EINVAL;
    }
    if (mask->window < 0 || mask->shared_len < 0) { vla_set_error("paged_attention: window and shared_len must not be negative"); return VLA_EINVAL; }
    if (mask->shared_len % cache->page_size || mask->shared_len > batch->max_len) {
        vla_set_error("paged_attention: shared_len %d is no multiple of page_size %d or exceeds max_len %d", mask->shared_len, cache->page_size, batch->max_len);
        return VLA_ESHAPE;
    }
    a->n_heads = n_heads; a->group = n_heads / cache->n_kv_heads;
    a->scale = mask->scale; a->cap = mask->softcap; a->slopes = mask->slopes; a->prefix_len = mask->prefix_len;
    a->window = mask->window; a->shared_len = mask->shared_len;
    return VLA_OK;
}

}  // namespace

extern "C" {

size_t vla_paged_attention_workspace_bytes(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_paged_mask *mask, int n_heads) {
    AttnArgs a{};
    if (check(cache, batch, mask, n_heads, &a)) return 0;
    return 256;
}

int vla_paged_attention(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_paged_mask *mask, const void *q, int n_heads,
                        int64_t q_stride, void *out, int64_t out_stride, float *lse, void *ws, size_t ws_bytes, void *stream) {
    AttnArgs a{};
    if (int rc = check(cache, batch, mask, n_heads, &a)) return rc;
    if (!q || !out || !ws) { vla_set_error("paged_attention: q, out or ws is NULL"); return VLA_EINVAL; }
    if ((uintptr_t)ws % 16) { vla_set_error("paged_attention: ws is not 16-byte aligned"); return VLA_EINVAL; }
    if (q_stride < (int64_t)n_heads * cache->head_dim || out_stride < (int64_t)n_heads * cache->head_dim) {
        vla_set_error("paged_attention: a row stride is shorter than its heads");
        return VLA_ESHAPE;
    }
    const size_t need = vla_paged_attention_workspace_bytes(cache, batch, mask, n_heads);
    if (ws_bytes < need) { vla_set_error("paged_attention: workspace %zu bytes, need %zu", ws_bytes, need); return VLA_EWORKSPACE; }
    if (batch->n_rows == 0) return VLA_OK;
    a.q = (const char *)q; a.out = (char *)out; a.lse = lse; a.q_stride = q_stride; a.o_stride = out_stride;
    hipStream_t st = (hipStream_t)stream;
    const dim3 grid(batch->n_rows, n_heads);
    if (cache->dtype == VLA_DTYPE_F32) paged_attention_simple_kernel<float><<<grid, 64, 0, st>>>(a);
    else paged_attention_simple_kernel<bf16_t><<<grid, 64, 0, st>>>(a);
    return vla_check_launch("paged_attention");
}

}  // extern "C"
