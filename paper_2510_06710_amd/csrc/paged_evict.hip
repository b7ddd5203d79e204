// Eviction from a paged KV cache by accumulated attention weight: the weights of a call's rows summed per position, and a cache cut to the
// heaviest positions.
#include "paged_rows.h"

namespace {

// ---- weights -----------------------------------------------------------------------------------------------------------------
// One product, S = Q K^T (rows queries, columns keys, on 32 x 32 matrix instructions), so a lane owns a key: its weights' sum over the queries is a
// sum over the lane's registers (and lane ^ 32).  A wave keeps 32 keys in registers and takes the packed rows (query r / group, head
// r % group of a key head's group) that may see them 32 at a time.
struct WeightArgs {
    AttnArgs a;
    const float *lse_in;
    float *mass;
    long mass_stride;
};

constexpr int WEIGHT_WAVES = 4;
template <typename T, int DP, int MODE>
__global__ void __launch_bounds__(64 * WEIGHT_WAVES) paged_weights_kernel(WeightArgs w) {
    typedef typename FragOf<T>::type frag;
    constexpr int KS = DP / 16;
    __shared__ __attribute__((aligned(16))) float lse_at[WEIGHT_WAVES][32], slope_at[WEIGHT_WAVES][32];
    __shared__ __attribute__((aligned(16))) int pos_at[WEIGHT_WAVES][32];
    const AttnArgs &a = w.a;
    const PagedView &pv = a.pv;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, hh = lane >> 5;
    int id = blockIdx.x;
    const int kvh = id % pv.n_kv;
    id /= pv.n_kv;
    const int s = id % pv.n_seq, key0 = (id / pv.n_seq * WEIGHT_WAVES + wave) * 32;
    const PagedSeq sq = paged_seq(pv, s);
    if (key0 >= sq.keys) return;                              // (no barriers below)
    const int base = sq.len - sq.n, key = key0 + col;
    const int prefix = a.prefix_len ? min(max(paged_int(a.prefix_len, s), 0), sq.keys) : 0;
    // rows that may see one of the keys: positions key0 on, below key0 + 31 + window; all where the prefix reaches
    int i0 = max(0, key0 - base), i1 = sq.rows;
    if (a.window) i1 = min(i1, max(0, key0 + 31 + a.window - base));
    if (key0 < prefix) { i0 = 0; i1 = sq.rows; }
    if (i0 >= i1 && base > key0 + 31) return;                 // nothing to add, and no new position to set
    frag k[KS];
    {
        const int at = min(key, sq.keys - 1), page = paged_int(pv.table, (size_t)s * pv.table_stride + (min(key0 + (col & 16), sq.keys - 1) >> pv.page_log));
        const bool ok = (unsigned)page < (unsigned)pv.n_pages;
        const T *src = (const T *)(ok ? pv.k : (const char *)zero_rows) + (ok ? (((size_t)page * pv.n_kv + kvh << pv.page_log) + (at & ((1 << pv.page_log) - 1))) * pv.d : 0);
#pragma unroll
        for (int kk = 0; kk < KS; kk++) {
            const int dim = kk * 16 + hh * 8;
#pragma unroll
            for (int e = 0; e < 8; e++) k[kk][e] = (T)0.f;
            if (dim < pv.d) k[kk] = *(const frag *)(src + dim);
        }
    }
    const float unit = Rows<T, DP, MODE, false>::unit_of(a);
    float sum = 0.f;
    for (int r0 = i0 * a.group & ~31; r0 < i1 * a.group; r0 += 32) {
        // a lane's packed row of the 32
        const int r = r0 + col, i = r / a.group, head = kvh * a.group + r - i * a.group, row = sq.r0 + i;
        const bool in = r < sq.rows * a.group;
        if (hh == 0) {
            float l = in ? w.lse_in[(size_t)row * a.n_heads + head] : -INFINITY;
            // (a row that sees nothing adds nothing: its weights are exp2(x - inf))
            lse_at[wave][col] = l == -INFINITY ? INFINITY : l * LOG2E - a.offset;
            pos_at[wave][col] = base + i;
            if (MODE & BIASED) slope_at[wave][col] = in ? a.slopes[head] * LOG2E : 0.f;
        }
        const T *src = (const T *)a.q + (size_t)(in ? row : sq.r0) * a.q_stride + (size_t)(in ? head : 0) * pv.d;
        f32x16_t x;
#pragma unroll
        for (int e = 0; e < 16; e++) x[e] = 0.f;
#pragma unroll
        for (int kk = 0; kk < KS; kk++) {
            const int dim = kk * 16 + hh * 8;
            frag q;
#pragma unroll
            for (int e = 0; e < 8; e++) q[e] = (T)0.f;
            if (dim < pv.d && in) {
                if (a.aligned) {
                    q = *(const frag *)(src + dim);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; e++) q[e] = src[dim + e];
                }
            }
            x = mma(q, k[kk], x);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // one wave's own LDS
#pragma unroll
        for (int g = 0; g < 4; g++) {                         // register 4 g + e is packed row r0 + 8 g + 4 hh + e
            const f32x4_t l = *(const f32x4_t *)&lse_at[wave][8 * g + 4 * hh];
            const i32x4_v p = *(const i32x4_v *)&pos_at[wave][8 * g + 4 * hh];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                float z = x[4 * g + e];
                if (MODE & CAPPED) z = sizeof(T) == 4 ? tanhf(z * (a.scale / a.cap)) : -__builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * (2.f * LOG2E * a.scale / a.cap)));
                if (MODE & BIASED) {
                    const float factor = MODE & CAPPED ? (sizeof(T) == 4 ? 1.f : 2.f) * a.cap * LOG2E : a.scale * LOG2E;
                    z = __builtin_fmaf(-slope_at[wave][8 * g + 4 * hh + e], fabsf((float)(p[e] - key)), z * factor);
                }
                const bool see = key < sq.keys && ((key <= p[e] && (a.window == 0 || key > p[e] - a.window)) || key < prefix);
                sum += see ? __builtin_amdgcn_exp2f(__builtin_fmaf(z, unit, -l[e])) : 0.f;
            }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
    sum = vla_fold_step<32>(sum, VlaAdd());
    if (hh == 0 && key < sq.keys) {
        float *m = w.mass + ((size_t)s * pv.n_kv + kvh) * w.mass_stride + key;
        *m = key < base ? *m + sum : sum;
    }
}

int check_weights(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_paged_mask *mask, int n_heads, AttnArgs *a) {
    const char *what = "paged_weights";
    if (int rc = vla_check_paged(what, cache, batch, &a->pv)) return rc;
    if (!mask) { vla_set_error("%s: mask is NULL", what); return VLA_EINVAL; }
    if (n_heads <= 0 || n_heads % cache->n_kv_heads) { vla_set_error("%s: n_heads %d is no multiple of n_kv_heads %d", what, n_heads, cache->n_kv_heads); return VLA_ESHAPE; }
    if (n_heads > 4096) { vla_set_error("%s: n_heads %d unsupported (at most 4096)", what, n_heads); return VLA_ESHAPE; }
    if (!(mask->scale > 0.f) || !(mask->softcap >= 0.f) || !(mask->scale < INFINITY) || !(mask->softcap < INFINITY)) {
        vla_set_error("%s: scale must be positive, softcap not negative, both finite", what);
        return VLA_EINVAL;
    }
    if (mask->window < 0) { vla_set_error("%s: window must not be negative", what); return VLA_EINVAL; }
    if ((long)batch->n_rows * n_heads > 0x7fffffffL / 2) { vla_set_error("%s: %d rows of %d heads are too many", what, batch->n_rows, n_heads); return VLA_ESHAPE; }
    a->n_heads = n_heads; a->group = n_heads / cache->n_kv_heads;
    a->scale = mask->scale; a->cap = mask->softcap; a->slopes = mask->slopes; a->prefix_len = mask->prefix_len; a->window = mask->window;
    const long items = (long)cache->n_kv_heads * batch->n_seq * ((batch->max_len + 32 * WEIGHT_WAVES - 1) / (32 * WEIGHT_WAVES));
    if (items > 0x7fffffffL / 256) { vla_set_error("%s: %ld tiles of positions are too many: split the batch", what, items); return VLA_ESHAPE; }
    return VLA_OK;
}

template <typename T, int DP>
int launch_weights(const WeightArgs &w, hipStream_t st) {
    const PagedView &pv = w.a.pv;
    const unsigned blocks = (unsigned)pv.n_kv * pv.n_seq * ((pv.max_len + 32 * WEIGHT_WAVES - 1) / (32 * WEIGHT_WAVES));
    switch ((w.a.cap > 0.f ? CAPPED : 0) | (w.a.slopes ? BIASED : 0)) {
        case 0: paged_weights_kernel<T, DP, 0><<<blocks, 64 * WEIGHT_WAVES, 0, st>>>(w); break;
        case CAPPED: paged_weights_kernel<T, DP, CAPPED><<<blocks, 64 * WEIGHT_WAVES, 0, st>>>(w); break;
        case BIASED: paged_weights_kernel<T, DP, BIASED><<<blocks, 64 * WEIGHT_WAVES, 0, st>>>(w); break;
        default: paged_weights_kernel<T, DP, CAPPED | BIASED><<<blocks, 64 * WEIGHT_WAVES, 0, st>>>(w); break;
    }
    return vla_check_launch("paged_weights");
}
template <typename T>
int launch_weights_sized(const WeightArgs &w, hipStream_t st) {
    switch (padded_dim(w.a.pv.d)) {
        case 64: return launch_weights<T, 64>(w, st);
        case 128: return launch_weights<T, 128>(w, st);
        default: return launch_weights<T, 256>(w, st);
    }
}

// ---- eviction ----------------------------------------------------------------------------------------------------------------
struct EvictArgs {
    PagedView pv;
    const float *mass;
    float *mass_out;
    long mass_stride, out_stride;
    int keep, first, recent;
    const int32_t *to_table;
    int to_stride;
    int32_t *kept, *new_len;
};

// Masses as numbers that ascend with them; 0 for NaN.
__device__ __forceinline__ unsigned order_of(float x) {
    if (x != x) return 0;
    const unsigned u = __builtin_bit_cast(unsigned, x + 0.f);          // (-0 is 0)
    return u >> 31 ? ~u : u | 1u << 31;
}

constexpr int EVICT_THREADS = 1024;
__device__ __forceinline__ int evict_scan(int v, int *all, int *red) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int in = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int x = __shfl_up(in, o, 64); if (lane >= o) in += x; }
    __syncthreads();
    if (lane == 63) red[wave] = in;
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < EVICT_THREADS / 64; w++) { if (w < wave) before += red[w]; total += red[w]; }
    *all = total;
    return before + in - v;
}

// A workgroup for each (sequence, key head): the least mass that stays, digit by digit (eight bits a pass over the masses), then what is above it
// and the first of what equals it, in order.  A chunk's masses are read before any of it is written, and land no further back: mass_out may be mass.
__global__ void __launch_bounds__(EVICT_THREADS) paged_evict_select_kernel(EvictArgs a) {
    __shared__ int bins[256], red[EVICT_THREADS / 64], digit, rest;
    const PagedView &pv = a.pv;
    const int h = blockIdx.x % pv.n_kv, s = blockIdx.x / pv.n_kv, t = threadIdx.x;
    const PagedSeq sq = paged_seq(pv, s);
    const int n = sq.keys;
    const size_t at = (size_t)s * pv.n_kv + h;
    const float *mass = a.mass + at * a.mass_stride;
    float *out = a.mass_out + at * a.out_stride;
    int32_t *kept = a.kept + at * a.keep;
    if (h == 0 && t == 0 && a.new_len) a.new_len[s] = min(n, a.keep);
    if (n <= a.keep) {
        for (int i = t; i < a.keep; i += EVICT_THREADS) kept[i] = i < n ? i : -1;
        if (out != mass)
            for (int i = t; i < n; i += EVICT_THREADS) out[i] = mass[i];
        return;
    }
    const int lo = a.first, hi = n - a.recent;
    int want = a.keep - a.first - a.recent;
    unsigned prefix = 0, mask = 0;
    for (int shift = 24; shift >= 0 && want > 0; shift -= 8) {
        if (t < 256) bins[t] = 0;
        __syncthreads();
        for (int i = lo + t; i < hi; i += EVICT_THREADS) {
            const unsigned key = order_of(mass[i]);
            if ((key & mask) == prefix) atomicAdd(&bins[key >> shift & 255], 1);
        }
        __syncthreads();
        int all;
        const int c = t < 256 ? bins[255 - t] : 0, above = evict_scan(c, &all, red);
        if (t < 256 && above < want && above + c >= want) { digit = 255 - t; rest = want - above; }
        __syncthreads();
        want = rest;
        prefix |= (unsigned)digit << shift;
        mask |= 255u << shift;
        __syncthreads();
    }
    if (a.keep == a.first + a.recent) prefix = ~0u;          // (no mass is that: none is taken)
    int done = 0, equal = 0;
    for (int i0 = 0; i0 < n; i0 += EVICT_THREADS) {
        const int i = i0 + t;
        const float m = i < n ? mass[i] : 0.f;
        const unsigned key = order_of(m);
        const bool open = i >= lo && i < hi, tie = open && key == prefix;
        int ties, taken;
        const int e = evict_scan(tie, &ties, red);
        const bool take = i < n && (!open || key > prefix || (tie && equal + e < want));
        const int to = evict_scan(take, &taken, red);
        if (take) { kept[done + to] = i; out[done + to] = m; }
        done += taken;
        equal += ties;
    }
}

// K and V of the kept positions to their places: 16 bytes a lane, four rows of one key head on their way at once.
template <int U>
__global__ void __launch_bounds__(256) paged_evict_move_kernel(EvictArgs a, int chunks, int row_bytes) {
    const PagedView &pv = a.pv;
    const int h = blockIdx.y % pv.n_kv, s = blockIdx.y / pv.n_kv, t = threadIdx.x, per = 256 / chunks;
    const PagedSeq sq = paged_seq(pv, s);
    const int n = min(sq.keys, a.keep), c = t % chunks, in_page = (1 << pv.page_log) - 1;
    const int32_t *kept = a.kept + ((size_t)s * pv.n_kv + h) * a.keep;
    const int32_t *table = pv.table + (size_t)s * pv.table_stride, *to_table = a.to_table + (size_t)s * a.to_stride;
    if (t >= per * chunks) return;
    auto row = [&](int page, int pos) { return ((((size_t)page * pv.n_kv + h) << pv.page_log) + (pos & in_page)) * row_bytes + c * 16; };
    const int r0 = blockIdx.x * per * U + t / chunks;
    int from[U], src_page[U], dst_page[U];
#pragma unroll
    for (int u = 0; u < U; u++) from[u] = r0 + u * per < n ? kept[r0 + u * per] : -1;
#pragma unroll
    for (int u = 0; u < U; u++) {
        src_page[u] = from[u] >= 0 ? table[from[u] >> pv.page_log] : -1;
        dst_page[u] = from[u] >= 0 ? to_table[(r0 + u * per) >> pv.page_log] : -1;
    }
    i32x4_v k[U], v[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
        const bool ok = (unsigned)src_page[u] < (unsigned)pv.n_pages;
        const size_t at = ok ? row(src_page[u], from[u]) : 0;
        k[u] = ok ? *(const i32x4_v *)(pv.k + at) : i32x4_v{0, 0, 0, 0};
        v[u] = ok ? *(const i32x4_v *)(pv.v + at) : i32x4_v{0, 0, 0, 0};
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
        const int to = r0 + u * per;
        if ((unsigned)dst_page[u] >= (unsigned)pv.n_pages || (dst_page[u] == src_page[u] && to == from[u])) continue;
        const size_t at = row(dst_page[u], to);
        *(i32x4_v *)(pv.k + at) = k[u];
        *(i32x4_v *)(pv.v + at) = v[u];
    }
}

}  // namespace

extern "C" {

size_t vla_paged_weights_workspace_bytes(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_paged_mask *mask, int n_heads) {
    AttnArgs a{};
    return check_weights(cache, batch, mask, n_heads, &a) ? 0 : 256;
}

int vla_paged_weights(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_paged_mask *mask, const void *q, int n_heads,
                      int64_t q_stride, const float *lse, float *mass, int64_t mass_stride, void *ws, size_t ws_bytes, void *stream) {
    WeightArgs w{};
    AttnArgs &a = w.a;
    if (int rc = check_weights(cache, batch, mask, n_heads, &a)) return rc;
    if (!mass || (batch->n_rows > 0 && (!q || !lse || !ws))) { vla_set_error("paged_weights: q, lse, mass or ws is NULL"); return VLA_EINVAL; }
    if ((uintptr_t)ws % 16) { vla_set_error("paged_weights: ws is not 16-byte aligned"); return VLA_EINVAL; }
    if (q_stride < (int64_t)n_heads * cache->head_dim || mass_stride < batch->max_len) {
        vla_set_error("paged_weights: a row of q is shorter than its heads, or one of mass than max_len");
        return VLA_ESHAPE;
    }
    if (batch->n_rows > 0 && ws_bytes < 256) { vla_set_error("paged_weights: workspace %zu bytes, need %d", ws_bytes, 256); return VLA_EWORKSPACE; }
    if (batch->n_rows == 0 || batch->max_rows == 0 || batch->max_len == 0) return VLA_OK;
    const bool f32 = cache->dtype == VLA_DTYPE_F32;
    a.q = (const char *)q; a.q_stride = q_stride;
    a.aligned = ((uintptr_t)q | (size_t)q_stride * (f32 ? 4 : 2)) % 16 == 0;
    a.offset = !f32 ? a.cap * LOG2E : 0.f;
    w.lse_in = lse; w.mass = mass; w.mass_stride = mass_stride;
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps("paged_weights", 0.0, st);
    return f32 ? launch_weights_sized<float>(w, st) : launch_weights_sized<bf16_t>(w, st);
}

int vla_paged_evict(const vla_paged_cache *cache, const vla_paged_batch *batch, const float *mass, int64_t mass_stride, int keep, int first,
                    int recent, const int32_t *to_table, int to_stride, int32_t *kept, float *mass_out, int64_t mass_out_stride,
                    int32_t *new_len, void *stream) {
    EvictArgs a{};
    if (int rc = vla_check_paged("paged_evict", cache, batch, &a.pv)) return rc;
    if (!mass || !to_table || !kept || !mass_out) { vla_set_error("paged_evict: mass, to_table, kept or mass_out is NULL"); return VLA_EINVAL; }
    if (keep < 1 || keep > (1 << 30) || first < 0 || recent < 0 || (long)first + recent > keep) {
        vla_set_error("paged_evict: keep %d, first %d, recent %d (keep from 1 to 2^30, first + recent at most keep)", keep, first, recent);
        return VLA_EINVAL;
    }
    if ((long)to_stride * cache->page_size < keep) { vla_set_error("paged_evict: %d pages of %d per sequence hold fewer than keep %d positions", to_stride, cache->page_size, keep); return VLA_ESHAPE; }
    const int least = keep < batch->max_len ? keep : batch->max_len;
    if (mass_stride < batch->max_len || mass_out_stride < least || (mass == mass_out && mass_stride != mass_out_stride)) {
        vla_set_error("paged_evict: mass of %ld positions, mass_out of %ld (max_len %d, keep %d; the same array: the same stride)", (long)mass_stride, (long)mass_out_stride, batch->max_len, keep);
        return VLA_ESHAPE;
    }
    const long pairs = (long)batch->n_seq * cache->n_kv_heads;
    if (pairs > 65535) { vla_set_error("paged_evict: %ld sequences times key heads (at most 65,535): split the batch", pairs); return VLA_ESHAPE; }
    a.mass = mass; a.mass_out = mass_out; a.mass_stride = mass_stride; a.out_stride = mass_out_stride;
    a.keep = keep; a.first = first; a.recent = recent; a.to_table = to_table; a.to_stride = to_stride; a.kept = kept; a.new_len = new_len;
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps("paged_evict", 0.0, st);
    paged_evict_select_kernel<<<(unsigned)pairs, EVICT_THREADS, 0, st>>>(a);
    if (int rc = vla_check_launch("paged_evict")) return rc;
    if (least == 0) return VLA_OK;
    const int row_bytes = cache->head_dim * (cache->dtype == VLA_DTYPE_F32 ? 4 : 2), chunks = row_bytes / 16, per = 256 / chunks * 4;
    paged_evict_move_kernel<4><<<dim3((least + per - 1) / per, (unsigned)pairs), 256, 0, st>>>(a, chunks, row_bytes);
    return vla_check_launch("paged_evict move");
}

}  // extern "C"
