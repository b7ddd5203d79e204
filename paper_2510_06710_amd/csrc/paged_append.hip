// Appending to a paged KV cache: norm of each head of q and k, rotation, rounding, K and V to their pages.
//
// Memory bound: a row's (n_heads + 2 n_kv) heads are read once and written once.  A lane holds eight consecutive dims of a head
// (16 or 32 bytes in, 16 or 32 out), a wave 64 / (lanes a head) heads at a time; a lane's dims are the same for all its heads,
// so their cos, sin and gains stay in registers.  The sum of squares is folded over the head's lanes; the other half of a rotated pair comes
// from the neighbour in LDS (interleaved pairs lie in one lane).  Angles: position * inv_freq in fp64 turns, whose whole part is
// dropped before cos and sin, so far positions lose nothing; once per row and frequency.
//
// A row's place is a chain of dependent reads (its sequence, length, page), so its first heads, gains and frequencies are asked for before it.
// 18,432 rows of 96 heads of 128, fp32 to bf16: 262 us, 5.2 TB/s (with norms 261); 2000 rows of 20 heads of 80 with norms, fp32: 12.7 us, of
// which 7 would be the bytes at that rate (gains in single words, behind the chain: 19.6); one row of 48 heads: 4.4 us, the chain itself.
#include "paged.h"

namespace {

struct AppendArgs {
    PagedView pv;
    const char *q, *k, *v;
    char *q_out;
    long q_stride, k_stride, v_stride, o_stride;      // elements
    int n_heads;             // of q (0: none)
    const double *inv_freq;
    int half, interleaved;
    float scale, eps;
    const float *q_gain, *k_gain;
    int lanes_log;           // log2 of the lanes per head (d / 8 rounded up to a power of two)
    int aligned;             // every row and head of the inputs and of q_out starts at a multiple of 16 bytes
};

template <typename T> __device__ __forceinline__ void load8(float (&x)[8], const T *p, bool aligned) {
    if (aligned) {
        if constexpr (sizeof(T) == 4) {
            const f32x4_t a = *(const f32x4_t *)p, b = *(const f32x4_t *)(p + 4);
#pragma unroll
            for (int e = 0; e < 4; e++) { x[e] = a[e]; x[4 + e] = b[e]; }
        } else {
            const bf16x8_t a = *(const bf16x8_t *)p;
#pragma unroll
            for (int e = 0; e < 8; e++) x[e] = (float)a[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++) x[e] = (float)p[e];
    }
}
template <typename T> __device__ __forceinline__ void store8(T *p, const float (&x)[8], bool aligned) {
    if (aligned) {
        if constexpr (sizeof(T) == 4) {
            f32x4_t a, b;
#pragma unroll
            for (int e = 0; e < 4; e++) { a[e] = x[e]; b[e] = x[4 + e]; }
            *(f32x4_t *)p = a;
            *(f32x4_t *)(p + 4) = b;
        } else {
            bf16x8_t a;
#pragma unroll
            for (int e = 0; e < 8; e++) a[e] = (bf16_t)x[e];
            *(bf16x8_t *)p = a;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; e++) p[e] = (T)x[e];
    }
}

template <typename TI, typename TO>
__global__ void __launch_bounds__(256) paged_append_kernel(AppendArgs a) {
    __shared__ float2 turn[128];
    __shared__ __attribute__((aligned(16))) float xs[4][64 * 8];
    const PagedView &pv = a.pv;
    const int row = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int d = pv.d, lanes = 1 << a.lanes_log, c = lane & (lanes - 1), dim = c * 8, r = 2 * a.half;
    const int total = a.n_heads + 2 * pv.n_kv, per_wave = 64 >> a.lanes_log, step = 4 * gridDim.y * per_wave;
    const bool in = dim < d;
    auto fetch = [&](float (&x)[8], int h) {
        const int kh = h - a.n_heads, vh = kh - pv.n_kv;             // q, k or v
        if (in && h < total) {
            const TI *src = kh < 0 ? (const TI *)a.q + row * a.q_stride + (size_t)h * d
                          : vh < 0 ? (const TI *)a.k + row * a.k_stride + (size_t)kh * d : (const TI *)a.v + row * a.v_stride + (size_t)vh * d;
            load8(x, src + dim, a.aligned);
        }
    };
    // the first heads, gains and the frequency, on their way while the row's place is looked up; then always the next heads
    int h = (blockIdx.y * 4 + wave) * per_wave + (lane >> a.lanes_log);
    float next[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    fetch(next, h);
    float gq[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f}, gk[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    auto gains = [&](float (&g)[8], const float *p) {
        typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
        if (!p || !in) return;
        const f32x4_any lo = *(const f32x4_any *)(p + dim), hi = *(const f32x4_any *)(p + dim + 4);
#pragma unroll
        for (int e = 0; e < 4; e++) { g[e] = lo[e]; g[4 + e] = hi[e]; }
    };
    gains(gq, a.q_gain);
    gains(gk, a.k_gain);
    const double freq = (int)threadIdx.x < a.half ? a.inv_freq[threadIdx.x] : 0.0;
    const int s = paged_seq_of_row(pv, row);
    if (s >= pv.n_seq) return;                                        // padding
    const PagedSeq sq = paged_seq(pv, s);
    const int i = row - sq.r0, pos = sq.len - sq.n + i;
    if (i < 0 || i >= sq.rows || pos < 0 || pos >= pv.max_len) return;
    const int page = paged_int(pv.table, (size_t)s * pv.table_stride + (pos >> pv.page_log));
    const bool kept = (unsigned)page < (unsigned)pv.n_pages;
    if ((int)threadIdx.x < a.half) {
        double t = (double)pos * freq * 0.15915494309189533577, sn, cs;      // turns
        t -= rint(t);
        sincospi(2.0 * t, &sn, &cs);
        turn[threadIdx.x] = make_float2((float)cs * a.scale, (float)sn * a.scale);
    }
    __syncthreads();
    float cs[8], sn[8];
#pragma unroll
    for (int e = 0; e < 8; e++) {
        const int x = dim + e;
        const float2 t = x < r ? turn[a.interleaved ? x >> 1 : (x < a.half ? x : x - a.half)] : make_float2(1.f, 0.f);
        cs[e] = t.x;
        sn[e] = (a.interleaved ? (x & 1) == 0 : x < a.half) ? -t.y : t.y;      // y = x cos +- (the other of the pair) sin
    }
    const size_t page_at = ((size_t)(kept ? page : 0) * pv.n_kv << pv.page_log) + (pos & ((1 << pv.page_log) - 1));
    for (int h0 = (blockIdx.y * 4 + wave) * per_wave; h0 < total; h0 += step, h += step) {
        const bool active = in && h < total;
        const int kh = h - a.n_heads, vh = kh - pv.n_kv;
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; e++) { x[e] = next[e]; next[e] = 0.f; }
        fetch(next, h + step);
        if (a.q_gain || a.k_gain) {                                   // (uniform: all lanes take part in the fold)
            float ss = 0.f;
#pragma unroll
            for (int e = 0; e < 8; e++) ss += x[e] * x[e];
            for (int o = lanes >> 1; o > 0; o >>= 1) ss += __shfl_xor(ss, o, 64);
            const bool normed = kh < 0 ? a.q_gain != nullptr : vh < 0 && a.k_gain != nullptr;
            if (normed) {
                const float f = 1.0f / sqrtf(ss / (float)d + a.eps);
#pragma unroll
                for (int e = 0; e < 8; e++) x[e] = x[e] * f * (kh < 0 ? gq[e] : gk[e]);
            }
        }
        if (r) {
            float o[8];
            if (a.interleaved) {
#pragma unroll
                for (int e = 0; e < 8; e++) o[e] = x[e ^ 1];
            } else {
                float *xw = xs[wave];
#pragma unroll
                for (int e = 0; e < 8; e += 4) *(f32x4_t *)(xw + lane * 8 + e) = f32x4_t{x[e], x[e + 1], x[e + 2], x[e + 3]};
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // one wave's own LDS
                const float *head = xw + (lane - c) * 8;
#pragma unroll
                for (int e = 0; e < 8; e++) {
                    const int y = dim + e;
                    o[e] = y < r ? head[y < a.half ? y + a.half : y - a.half] : 0.f;
                }
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            }
            if (vh < 0) {
#pragma unroll
                for (int e = 0; e < 8; e++)
                    if (dim + e < r) x[e] = x[e] * cs[e] + o[e] * sn[e];
            }
        }
        if (!active) continue;
        if (kh < 0) store8((TO *)a.q_out + row * a.o_stride + (size_t)h * d + dim, x, a.aligned);
        else if (kept) {
            const size_t at = (page_at + ((size_t)(vh < 0 ? kh : vh) << pv.page_log)) * d + dim;
            store8((TO *)(vh < 0 ? pv.k : pv.v) + at, x, true);
        }
    }
}

template <typename T>
__global__ void __launch_bounds__(256) paged_embed_kernel(float *X, const int32_t *ids, const T *patch, int n_patch, const T *embed, int H, int vocab) {
    const int id = ids[blockIdx.x];
    const T *src = id < 0 && n_patch > 0 ? patch + (size_t)min(-(id + 1), n_patch - 1) * H : embed + (size_t)min(max(id, 0), vocab - 1) * H;
    for (int i = threadIdx.x; i < H; i += 256) X[(size_t)blockIdx.x * H + i] = (float)src[i];
}

// The last of each sequence's rows; zeros for a sequence without rows.
__global__ void __launch_bounds__(256) paged_last_rows_kernel(float *out, const float *X, const int32_t *row_start, int n_rows, int H) {
    const int s = blockIdx.x, r0 = min(max(row_start[s], 0), n_rows), r1 = min(max(row_start[s + 1], r0), n_rows);
    for (int i = threadIdx.x; i < H; i += 256) out[(size_t)s * H + i] = r1 > r0 ? X[(size_t)(r1 - 1) * H + i] : 0.f;
}

// theta^(-2 i / d), as vla_rope_entry has it
__global__ void rotary_freq_kernel(double *freq, int d, float theta) {
    if ((int)threadIdx.x < d / 2) freq[threadIdx.x] = pow((double)theta, -2.0 * (double)threadIdx.x / (double)d);
}

}  // namespace

template <typename T>
int launch_paged_embed(float *X, const int32_t *ids, const T *patch, int n_patch, const T *embed, int n_rows, int H, int vocab, hipStream_t st) {
    paged_embed_kernel<T><<<n_rows, 256, 0, st>>>(X, ids, patch, n_patch, embed, H, vocab);
    return vla_check_launch("paged_embed");
}
template int launch_paged_embed<float>(float *, const int32_t *, const float *, int, const float *, int, int, int, hipStream_t);
template int launch_paged_embed<bf16_t>(float *, const int32_t *, const bf16_t *, int, const bf16_t *, int, int, int, hipStream_t);
int launch_paged_last_rows(float *out, const float *X, const int32_t *row_start, int n_seq, int n_rows, int H, hipStream_t st) {
    paged_last_rows_kernel<<<n_seq, 256, 0, st>>>(out, X, row_start, n_rows, H);
    return vla_check_launch("paged_last_rows");
}
int launch_rotary_freq(double *freq, int d, float theta, hipStream_t st) {
    rotary_freq_kernel<<<1, 128, 0, st>>>(freq, d, theta);
    return vla_check_launch("rotary_freq");
}

int vla_check_paged(const char *what, const vla_paged_cache *c, const vla_paged_batch *b, PagedView *out) {
    if (!c || !b) { vla_set_error("%s: cache or batch is NULL", what); return VLA_EINVAL; }
    if (c->dtype != VLA_DTYPE_F32 && c->dtype != VLA_DTYPE_BF16) { vla_set_error("%s: unknown dtype %d", what, c->dtype); return VLA_EDTYPE; }
    if (!c->k || !c->v) { vla_set_error("%s: k or v of the cache is NULL", what); return VLA_EINVAL; }
    if (((uintptr_t)c->k | (uintptr_t)c->v) % 16) { vla_set_error("%s: the cache is not 16-byte aligned", what); return VLA_EINVAL; }
    if (c->n_pages <= 0 || c->n_kv_heads <= 0 || c->head_dim <= 0) { vla_set_error("%s: sizes of the cache must be positive", what); return VLA_EINVAL; }
    if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1))) {
        vla_set_error("%s: page_size %d unsupported (a power of two from 16 to 1024)", what, c->page_size);
        return VLA_ESHAPE;
    }
    if (c->head_dim % 16 != 0 || c->head_dim > 256) { vla_set_error("%s: head_dim %d unsupported (multiple of 16, at most 256)", what, c->head_dim); return VLA_ESHAPE; }
    if (c->n_kv_heads > 1024) { vla_set_error("%s: n_kv_heads %d unsupported (at most 1024)", what, c->n_kv_heads); return VLA_ESHAPE; }
    if (b->n_seq <= 0 || b->n_rows < 0 || b->max_rows < 0 || b->max_len < 0 || b->table_stride < 0) {
        vla_set_error("%s: n_seq must be positive, n_rows, max_rows, max_len and table_stride not negative", what);
        return VLA_EINVAL;
    }
    if (!b->row_start || !b->kv_len || !b->page_table) { vla_set_error("%s: row_start, kv_len or page_table is NULL", what); return VLA_EINVAL; }
    if (b->max_len > (1 << 30)) { vla_set_error("%s: max_len %d unsupported (at most 2^30)", what, b->max_len); return VLA_ESHAPE; }
    if (b->n_seq > 65536) { vla_set_error("%s: n_seq %d unsupported (at most 65,536)", what, b->n_seq); return VLA_ESHAPE; }
    if ((long)b->table_stride * c->page_size < b->max_len) {
        vla_set_error("%s: %d pages of %d per sequence hold fewer than max_len %d positions", what, b->table_stride, c->page_size, b->max_len);
        return VLA_ESHAPE;
    }
    *out = PagedView{(char *)c->k, (char *)c->v, c->n_pages, __builtin_ctz((unsigned)c->page_size), c->n_kv_heads, c->head_dim,
                     b->n_seq, b->n_rows, b->max_rows, b->max_len, b->table_stride, b->row_start, b->kv_len, b->page_table};
    return VLA_OK;
}

extern "C" int vla_paged_append(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_rotary *rotary, const void *q,
                                const void *k, const void *v, int in_dtype, int n_heads, int64_t q_stride, int64_t k_stride,
                                int64_t v_stride, void *q_out, int64_t q_out_stride, void *stream) {
    AppendArgs a{};
    if (int rc = vla_check_paged("paged_append", cache, batch, &a.pv)) return rc;
    if (in_dtype != VLA_DTYPE_F32 && in_dtype != VLA_DTYPE_BF16) { vla_set_error("paged_append: unknown dtype %d", in_dtype); return VLA_EDTYPE; }
    if (!rotary || (batch->n_rows > 0 && (!k || !v))) { vla_set_error("paged_append: rotary, k or v is NULL"); return VLA_EINVAL; }
    if (!q != !q_out) { vla_set_error("paged_append: q and q_out come together"); return VLA_EINVAL; }
    const int d = cache->head_dim, kv = cache->n_kv_heads;
    if (q && (n_heads <= 0 || n_heads > 65536)) { vla_set_error("paged_append: n_heads %d unsupported (1 .. 65,536)", n_heads); return VLA_ESHAPE; }
    if (rotary->rot_dim < 0 || rotary->rot_dim % 2 || rotary->rot_dim > d) {
        vla_set_error("paged_append: rot_dim %d unsupported (even, at most head_dim %d)", rotary->rot_dim, d);
        return VLA_ESHAPE;
    }
    if (rotary->rot_dim && !rotary->inv_freq) { vla_set_error("paged_append: inv_freq is NULL"); return VLA_EINVAL; }
    if ((rotary->q_gain || rotary->k_gain) && !(rotary->eps >= 0.f)) { vla_set_error("paged_append: eps must not be negative"); return VLA_EINVAL; }
    if (k_stride < (int64_t)kv * d || v_stride < (int64_t)kv * d || (q && (q_stride < (int64_t)n_heads * d || q_out_stride < (int64_t)n_heads * d))) {
        vla_set_error("paged_append: a row stride is shorter than its heads");
        return VLA_ESHAPE;
    }
    if (q && q == q_out && (in_dtype != cache->dtype || q_stride != q_out_stride)) {
        vla_set_error("paged_append: q_out is q, of another dtype or stride");
        return VLA_EINVAL;
    }
    if (batch->n_rows == 0) return VLA_OK;
    a.q = (const char *)q; a.k = (const char *)k; a.v = (const char *)v; a.q_out = (char *)q_out;
    a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.o_stride = q_out_stride;
    a.n_heads = q ? n_heads : 0;
    a.inv_freq = rotary->inv_freq; a.half = rotary->rot_dim / 2; a.interleaved = rotary->interleaved != 0;
    a.scale = rotary->scale; a.eps = rotary->eps; a.q_gain = q ? rotary->q_gain : nullptr; a.k_gain = rotary->k_gain;
    while ((8 << a.lanes_log) < d) a.lanes_log++;
    const size_t ei = in_dtype == VLA_DTYPE_F32 ? 4 : 2, eo = cache->dtype == VLA_DTYPE_F32 ? 4 : 2;
    size_t bits = (uintptr_t)k | (uintptr_t)v | (size_t)k_stride * ei | (size_t)v_stride * ei;
    if (q) bits |= (uintptr_t)q | (uintptr_t)q_out | (size_t)q_stride * ei | (size_t)q_out_stride * eo;
    a.aligned = bits % 16 == 0;
    const int units = (a.n_heads + 2 * kv + (64 >> a.lanes_log) - 1) / (64 >> a.lanes_log);          // heads of one wave at a time
    // few rows: a row's heads on several workgroups, one step each; many: one workgroup a row, whose angles serve all its heads (2000 rows: 20 us,
    // on two workgroups a row 30)
    const dim3 grid(batch->n_rows, batch->n_rows < 512 ? (units + 3) / 4 : 1);
    ProfScope ps("paged_append", (double)batch->n_rows * (a.n_heads + 2 * kv) * d * (double)(ei + eo), (hipStream_t)stream);
    hipStream_t st = (hipStream_t)stream;
    const bool fi = in_dtype == VLA_DTYPE_F32, fo = cache->dtype == VLA_DTYPE_F32;
    if (fi && fo) paged_append_kernel<float, float><<<grid, 256, 0, st>>>(a);
    else if (fi) paged_append_kernel<float, bf16_t><<<grid, 256, 0, st>>>(a);
    else if (fo) paged_append_kernel<bf16_t, float><<<grid, 256, 0, st>>>(a);
    else paged_append_kernel<bf16_t, bf16_t><<<grid, 256, 0, st>>>(a);
    return vla_check_launch("paged_append");
}
