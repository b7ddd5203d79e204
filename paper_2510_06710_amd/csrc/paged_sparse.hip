// Sparse attention on a paged KV cache: bounds of each page's keys, the pages that a row's heads read, and the attention over them.
//
// For a key k of a page with lo <= k <= hi (dim by dim), q.k <= sum_d max(q_d lo_d, q_d hi_d).  Summed over the heads of a group that is
// (sum_h max(q_h, 0)) . hi + (sum_h min(q_h, 0)) . lo: two products a dim whatever the group, in fp64, where the sums of bf16 products are exact
// but for the last bits and the order of additions decides no border.
#include "paged_rows.h"
#include "paged_select.h"

namespace {

// ---- bounds ----------------------------------------------------------------------------------------------------------------
// A workgroup for each (page, sequence): its lanes each hold eight dims of one key head (16 bytes of bf16, 32 of fp32).  Reads the keys
// below kv_len of a page once and writes two rows a head; nothing is rounded.  Bound by memory: four prompts of up to 32,768 positions, 8 heads of 128, 181 MB in 38 us, 4.7 TB/s
// (plain reads reach 6.1; the first workgroups' look-ups and the last ones' end are a fifth of it); fp32, 362 MB, 76 us.
template <typename T>
__global__ void __launch_bounds__(256) paged_bounds_kernel(PagedView pv, T *bounds) {
    typedef T t8 __attribute__((ext_vector_type(8)));
    const int s = blockIdx.x, page_size = 1 << pv.page_log, chunks = pv.d / 8;
    const PagedSeq sq = paged_seq(pv, s);
    if (sq.rows == 0) return;
    const int number = (max(sq.len - sq.n, 0) >> pv.page_log) + blockIdx.y, key0 = number << pv.page_log;
    if (key0 >= sq.keys) return;
    const int page = paged_int(pv.table, (size_t)s * pv.table_stride + number), n = min(page_size, sq.keys - key0);
    if ((unsigned)page >= (unsigned)pv.n_pages) return;
    for (int x = threadIdx.x; x < pv.n_kv * chunks; x += 256) {
        const int h = x / chunks, c = x - h * chunks;
        const T *k = (const T *)pv.k + (((size_t)page * pv.n_kv + h) << pv.page_log) * pv.d + c * 8;
        float lo[8], hi[8];
#pragma unroll
        for (int e = 0; e < 8; e++) { lo[e] = INFINITY; hi[e] = -INFINITY; }
        for (int i = 0; i < n; i += 8) {                      // eight rows on their way at once (behind the last: the last again)
            t8 v[8];
#pragma unroll
            for (int u = 0; u < 8; u++) v[u] = *(const t8 *)(k + (size_t)min(i + u, n - 1) * pv.d);
#pragma unroll
            for (int u = 0; u < 8; u++)
#pragma unroll
                for (int e = 0; e < 8; e++) { lo[e] = fminf(lo[e], (float)v[u][e]); hi[e] = fmaxf(hi[e], (float)v[u][e]); }
        }
        T *to = bounds + ((size_t)page * pv.n_kv + h) * 2 * pv.d + c * 8;
        t8 a, b;
#pragma unroll
        for (int e = 0; e < 8; e++) { a[e] = (T)lo[e]; b[e] = (T)hi[e]; }
        *(t8 *)to = a;
        *(t8 *)(to + pv.d) = b;
    }
}

// ---- selection -------------------------------------------------------------------------------------------------------------
struct SelectArgs {
    PagedView pv;
    const void *bounds, *q;
    long q_stride;
    int group, n_select, first, recent;
    int pages;               // of a sequence at most
    unsigned long long *keys;  // [n_rows][n_kv][pages]: scores, in an order of whole numbers
    int32_t *selected;
};

// Scores as numbers that ascend with them; 0 for NaN.  Infinity is as 2^1022, above all sums of products of fp32 values: its own number begins with more ones than a cut's keys may (see cut_numbers).
__device__ __forceinline__ unsigned long long order_of(double x) {
    if (x != x) return 0;
    x = fmin(x, 0x1p1022);
    const unsigned long long u = __builtin_bit_cast(unsigned long long, x + 0.0);          // (-0 is 0)
    return u >> 63 ? ~u : u | 1ull << 63;
}

// A row's place: its sequence's table and the number of its page, -1 where it has none.
__device__ __forceinline__ int page_of_row(const PagedView &pv, int row, int *s) {
    *s = paged_seq_of_row(pv, row);
    if (*s >= pv.n_seq) return -2;                            // padding
    const PagedSeq sq = paged_seq(pv, *s);
    const int i = row - sq.r0, p = min(sq.len - sq.n + i, sq.keys - 1);
    if (i < 0 || i >= sq.rows) return -2;
    return p < 0 ? -1 : p >> pv.page_log;
}

// Sum over 2^lanes_log neighbouring lanes, by lane moves (the value of lane ^ o, in halves).
template <int CTRL> __device__ __forceinline__ double moved(double v) {
    const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
    const unsigned lo = __builtin_bit_cast(unsigned, vla_dpp<CTRL>(__builtin_bit_cast(float, (unsigned)u))), hi = __builtin_bit_cast(unsigned, vla_dpp<CTRL>(__builtin_bit_cast(float, (unsigned)(u >> 32))));
    return __builtin_bit_cast(double, (unsigned long long)hi << 32 | lo);
}
template <int O> __device__ __forceinline__ double paired(double v) {
    const unsigned long long u = __builtin_bit_cast(unsigned long long, v);
    const VlaPair lo = vla_pair<O>(__builtin_bit_cast(float, (unsigned)u)), hi = vla_pair<O>(__builtin_bit_cast(float, (unsigned)(u >> 32)));
    auto join = [](float h, float l) { return __builtin_bit_cast(double, (unsigned long long)__builtin_bit_cast(unsigned, h) << 32 | __builtin_bit_cast(unsigned, l)); };
    return join(hi.a, lo.a) + join(hi.b, lo.b);
}
__device__ __forceinline__ double lanes_sum(double v, int lanes_log) {
    if (lanes_log > 0) v += moved<0xb1>(v);                  // quad_perm 1 0 3 2
    if (lanes_log > 1) v += moved<0x4e>(v);                  // quad_perm 2 3 0 1
    if (lanes_log > 2) v += moved<0x141>(v);                 // row_half_mirror: lane ^ 7, which has what lane ^ 4 has once fours agree
    if (lanes_log > 3) v += moved<0x140>(v);                 // row_mirror: lane ^ 15
    if (lanes_log > 4) v = paired<16>(v);
    if (lanes_log > 5) v = paired<32>(v);
    return v;
}

// A page's bounds are 2 d values of lo and hi, 16 bytes a lane: `lanes` lanes (a power of two, at most 64) hold a page, so a wave's load has 64 / lanes of them, and eight loads are on their way at once
// (an fp32 page of more than 128 dims takes two loads a lane).  The parts of q that a lane multiplies by are the same for all pages.
// Where pages are few it is the chain of look-ups before the first load: 8 x 2048 pages of 512 bytes 7.3 us.  32 ragged rows of up to 1024 pages of 8 heads, 67 MB, take 23 us, 11 of them at the rate of reads;
// the rest is that chain and some 60 vector instructions a kilobyte, 8 of them products and 8 the bounds' widening to fp64, the others the bf16 values' unpacking and the sum over lanes.  In fp32 9.0 and 48 us.
// (One wave a page and load, q again for every four pages: 12 and 81.)
template <typename T>
__global__ void __launch_bounds__(256) paged_score_kernel(SelectArgs a, int lanes_log, int per_block) {
    constexpr int E = 16 / sizeof(T), U = 8, R = sizeof(T) == 4 ? 2 : 1;          // values of a load; pages of a lane at once; loads of a page
    typedef T vec __attribute__((ext_vector_type(E)));
    __shared__ double part[2 * 256];                         // what lo and hi are multiplied by: the group's negative and positive parts of q
    const PagedView &pv = a.pv;
    const int h = blockIdx.x % (unsigned)pv.n_kv, row = blockIdx.x / (unsigned)pv.n_kv, t = threadIdx.x, lanes = 1 << lanes_log;
    // (the first heads' q on their way while the row's place is looked up)
    constexpr int AHEAD = 8;
    const T *qs = (const T *)a.q + row * a.q_stride + (size_t)h * a.group * pv.d + min(t, pv.d - 1);
    float q[AHEAD];
#pragma unroll
    for (int g = 0; g < AHEAD; g++) q[g] = (float)qs[(size_t)min(g, a.group - 1) * pv.d];
    int s;
    const int last = page_of_row(pv, row, &s), n0 = blockIdx.y * per_block, n1 = min(n0 + per_block, last + 1);
    if (n0 >= n1) return;
    if (t < pv.d) {
        double up = 0.0, down = 0.0;
        auto add = [&](double x) {
            up += x > 0.0 ? x : 0.0;
            down += x > 0.0 ? 0.0 : x;
        };
#pragma unroll
        for (int g = 0; g < AHEAD; g++)
            if (g < a.group) add((double)q[g]);
        for (int g = AHEAD; g < a.group; g++) add((double)(float)qs[(size_t)g * pv.d]);
        part[t] = down;
        part[pv.d + t] = up;
    }
    __syncthreads();
    const int lane = t & (lanes - 1), chunks = 2 * pv.d / E;
    double w[R][E];
#pragma unroll
    for (int r = 0; r < R; r++)
#pragma unroll
        for (int e = 0; e < E; e++) w[r][e] = lane + r * lanes < chunks ? part[(lane + r * lanes) * E + e] : 0.0;
    const int32_t *table = pv.table + (size_t)s * pv.table_stride;
    unsigned long long *keys = a.keys + ((size_t)row * pv.n_kv + h) * a.pages;
    const int step = 256 >> lanes_log;                       // pages of one load of the workgroup
    int page[U];
    auto look = [&](int p0) {
#pragma unroll
        for (int u = 0; u < U; u++) page[u] = p0 + u * step < n1 ? table[p0 + u * step] : -1;
    };
    look(n0 + (t >> lanes_log));
    for (int p0 = n0 + (t >> lanes_log); __any(p0 < n1); p0 += U * step) {
        vec b[U][R];
#pragma unroll
        for (int u = 0; u < U; u++)
#pragma unroll
            for (int r = 0; r < R; r++)
                if ((unsigned)page[u] < (unsigned)pv.n_pages && lane + r * lanes < chunks)
                    b[u][r] = *(const vec *)((const T *)a.bounds + ((size_t)page[u] * pv.n_kv + h) * 2 * pv.d + (lane + r * lanes) * E);
                else
#pragma unroll
                    for (int e = 0; e < E; e++) b[u][r][e] = (T)0.f;          // (a page that is not there: zeros)
        look(p0 + U * step);                                  // (on their way while the products are formed)
        double x[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            x[u] = 0.0;
#pragma unroll
            for (int r = 0; r < R; r++)
                if (r == 0 || lanes + lane < chunks)          // (a zero times an infinite bound of no dim)
#pragma unroll
                    for (int e = 0; e < E; e++) x[u] = __builtin_fma((double)(float)b[u][r][e], w[r][e], x[u]);
        }
#pragma unroll
        for (int u = 0; u < U; u++) x[u] = lanes_sum(x[u], lanes_log);
#pragma unroll
        for (int u = 0; u < U; u++)
            if (lane == 0 && p0 + u * step < n1) keys[p0 + u * step] = order_of(x[u]);
    }
}

// A workgroup for each (row, key head): the keys to LDS, then the cut among those that are free to choose, [first, n - recent).  The bits that all of them share are found first: scores of one
// sign and about one size have a dozen, which no digit need be spent on.  Bound by the chain of its digits and barriers: 64 of 2048 pages for 8 lists 8 us, of up to 1024 for 256 lists 7.6.
__global__ void __launch_bounds__(256) paged_select_kernel(SelectArgs a) {
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ CutLds cut;
    __shared__ unsigned long long differ[4];
    unsigned long long *key = (unsigned long long *)lds;
    const PagedView &pv = a.pv;
    const int h = blockIdx.x % (unsigned)pv.n_kv, row = blockIdx.x / (unsigned)pv.n_kv, t = threadIdx.x;
    const unsigned long long *src = a.keys + ((size_t)row * pv.n_kv + h) * a.pages;
    constexpr int AHEAD = 8;                                 // of a lane, on their way while the row's place is looked up
    unsigned long long held[AHEAD];
    if (a.pages > a.n_select)
#pragma unroll
        for (int u = 0; u < AHEAD; u++) held[u] = src[min(t + u * 256, a.pages - 1)];
    int s;
    const int last = page_of_row(pv, row, &s), n = last + 1;
    if (last < -1) return;
    int32_t *out = a.selected + ((size_t)row * pv.n_kv + h) * a.n_select;
    if (n <= a.n_select) {
        for (int i = t; i < a.n_select; i += 256) out[i] = i < n ? i : -1;
        return;
    }
    const int lo = a.first, hi = n - a.recent, want = a.n_select - a.first - a.recent;
    Cut<unsigned long long> c{~0ull - 1, ~0ull, 0};          // (no score is that: what stays anyway alone is taken)
    {
        unsigned long long x = 0;
        const unsigned long long one = src[lo];
        auto hold = [&](int i, unsigned long long k) {
            if (i >= n) return;
            const bool open = i >= lo && i < hi;
            key[i] = open ? k : ~0ull;
            if (open) x |= k ^ one;
        };
#pragma unroll
        for (int u = 0; u < AHEAD; u++) hold(t + u * 256, held[u]);
        for (int i = t + AHEAD * 256; i < n; i += 256) hold(i, src[i]);
        for (int o = 32; o > 0; o >>= 1) x |= __shfl_xor(x, o, 64);
        if ((t & 63) == 0) differ[t >> 6] = x;
        __syncthreads();
        x = differ[0] | differ[1] | differ[2] | differ[3];
        if (want > 0)
            c = cut_keys<256, false, unsigned long long>([&](auto f) {
                for (int i = lo + t; i < hi; i += 256) f(key[i], 1);
            }, want, x ? 64 - __builtin_clzll(x) : 0, one, cut);
    }
    cut_numbers<256, 8>(n, c, [&](int i) { return key[i]; }, [](int, unsigned long long k) { return k; }, [&](int place, int i) { out[place] = i; }, cut);
}

// ---- attention over the selected pages ----------------------------------------------------------------------------------------
struct SparseArgs {
    AttnArgs a;
    const int32_t *selected;
    int n_select, heads_tiles;               // tiles of 32 heads of a group
};

// Keys are taken 16 at a time (a page's run of them), two such runs to a tile of 32, through the same ring and products as paged_decode_kernel.
// A workgroup is one wave: of one row and key head, up to 32 heads of its group, and a part of its list.  On a bf16 cache weights enter the product with v as a bf16 head and a bf16 tail (2^-16 of each is lost).
// Bound by memory: 32 rows of 64 pages of 32 positions, 8 heads of 128, 268 MB in 54 us, 5.0 TB/s; one row of 64 pages of 64 (17 MB) 8.8 us, and 4.3 for the join of its 64 parts.
// In fp32 168 us (3.2 TB/s; eight matrix instructions for one, most of whose columns are empty) and 17.4.
template <typename T, int DP, int MODE>
__global__ void __launch_bounds__(64) paged_sparse_kernel(SparseArgs x) {
    typedef Tile<T, DP> TL;
    constexpr int BYTES = 32 * TL::ROW, STAGE = 2 * BYTES, LOADS = 4 * 16 / TL::RPI;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const unsigned ring0 = (unsigned)(size_t)(lds_void *)lds;
    const AttnArgs &a = x.a;
    const PagedView &pv = a.pv;
    const int lane = threadIdx.x, part = blockIdx.y;
    const unsigned id = blockIdx.x / (unsigned)pv.n_kv;
    const int kvh = blockIdx.x % (unsigned)pv.n_kv, ht = id % (unsigned)x.heads_tiles, row = id / (unsigned)x.heads_tiles;
    const int32_t *list = x.selected + ((size_t)row * pv.n_kv + kvh) * x.n_select;
    const int entry = list[min(lane, x.n_select - 1)];       // (on its way while the row's place is looked up)
    const int s = paged_seq_of_row(pv, row);
    if (s >= pv.n_seq) return;
    const PagedSeq sq = paged_seq(pv, s);
    const int i = row - sq.r0;
    if (i < 0 || i >= sq.rows) return;
    const int p = min(sq.len - sq.n + i, sq.keys - 1);       // the last position it sees
    const int32_t *table = pv.table + (size_t)s * pv.table_stride;
    int m = 0;                                               // entries before the first negative one
    for (; m < x.n_select; m += 64) {
        const int e = m + lane;
        const unsigned long long ends = __ballot(e >= x.n_select || (m == 0 ? entry : list[min(e, x.n_select - 1)]) < 0);
        if (ends) { m += __builtin_ctzll(ends); break; }
    }
    m = __builtin_amdgcn_readfirstlane(min(m, x.n_select));
    const int per_log = pv.page_log - 4, runs = p < 0 ? 0 : m << per_log, tiles = (runs + 1) / 2;
    const int share = __builtin_amdgcn_readfirstlane((unsigned)(tiles + a.parts - 1) / (unsigned)a.parts), t0 = min(part * share, tiles), t1 = min(t0 + share, tiles);
    // run r: where its 16 keys begin, and their page; a run that nothing sees begins behind p
    auto run_of = [&](int r, int *page) __attribute__((always_inline)) {
        *page = -1;
        if (r >= runs) return p + 1;
        const int e = r >> per_log, number = paged_int(list, e), before = e ? paged_int(list, e - 1) : -1;
        const long key = ((long)number << pv.page_log) + (r & ((1 << per_log) - 1)) * 16;
        if (number <= before || key > p) return p + 1;
        *page = paged_int(table, number);
        return (int)key;
    };
    typename TL::template Offsets<false, 16> off_k;
    typename TL::template Offsets<true, 16> off_v;
    off_k.start(pv, 0);
    off_v.start(pv, 0);
    const Place place(pv, kvh, sizeof(T));
    int begin[2][2];                                         // of the tiles in the ring's stages
    auto load_run = [&](unsigned at, int key, int page) __attribute__((always_inline)) {
        if (key + 15 <= p || key > p) {                      // (behind p: zeros)
            const size_t from = place.at(pv, page, key);
            off_k.load(at, place.in(pv, pv.k, key > p ? -1 : page, from));
            off_v.load(at + BYTES, place.in(pv, pv.v, key > p ? -1 : page, from));
        } else {
            const Span sp{key, p + 1, 0, 0};
            TL::template load<false, 16>(at, pv.k, pv, page, kvh, key, sp);
            TL::template load<true, 16>(at + BYTES, pv.v, pv, page, kvh, key, sp);
        }
    };
    auto load = [&](int t, int stage) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < 2; u++) {
            int page;
            const int key = run_of(2 * t + u, &page);
            if (stage) begin[1][u] = key; else begin[0][u] = key;
            load_run(ring0 + stage * STAGE + u * 16 * TL::ROW, key, page);
        }
    };
    if (t0 < t1) load(t0, 0);
    Query y{};
    y.row = row;
    y.valid = ht * 32 + (lane & 31) < a.group;
    y.head = kvh * a.group + min(ht * 32 + (lane & 31), a.group - 1);
    Rows<T, DP, MODE, sizeof(T) == 2> rows;
    rows.start(a, y);
    auto step = [&](int t, int stage) __attribute__((always_inline)) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (t + 1 < t1) { load(t + 1, stage ^ 1); vm_wait<LOADS>(); }
        else vm_wait<0>();
        const char *kt = lds + stage * STAGE;
        f32x16_t z;
        typename Rows<T, DP, MODE, sizeof(T) == 2>::Weights w;
        rows.scores(z, kt);
#pragma unroll
        for (int k = 0; k < 16; k++) z[k] = rows.shaped(z[k], a, y, 0, k);
        const int hh = (lane >> 5) & 1;
#pragma unroll
        for (int u = 0; u < 2; u++)
            if (begin[stage][u] + 15 > p) {
#pragma unroll
                for (int k = 0; k < 8; k++)
                    if (begin[stage][u] + 8 * (k / 4) + 4 * hh + k % 4 > p) z[8 * u + k] = -INFINITY;
            }
        rows.move_to(rows.largest(z, rows.unit_of(a)));
        rows.weights(w, z, rows.unit_of(a));
        rows.values(w, kt + BYTES);
    };
    for (int t = t0; t < t1; t += 2) {
        step(t, 0);
        if (t + 1 < t1) step(t + 1, 1);
    }
    rows.finish(a, y, part);
}

int check_bounds(const char *what, const void *bounds) {
    if (!bounds) { vla_set_error("%s: bounds is NULL", what); return VLA_EINVAL; }
    if ((uintptr_t)bounds % 16) { vla_set_error("%s: bounds is not 16-byte aligned", what); return VLA_EINVAL; }
    return VLA_OK;
}
int check_pages(const PagedView &pv, SelectArgs *a) {
    a->pv = pv;
    a->pages = (pv.max_len + (1 << pv.page_log) - 1) >> pv.page_log;
    if (a->pages > VLA_SELECT_PAGES) { vla_set_error("paged_select: %d pages of a sequence (at most %d)", a->pages, VLA_SELECT_PAGES); return VLA_ESHAPE; }
    if ((long)pv.n_rows * pv.n_kv > 0x7fffffffL / 256) { vla_set_error("paged_select: %d rows of %d key heads are too many", pv.n_rows, pv.n_kv); return VLA_ESHAPE; }
    return VLA_OK;
}
size_t select_bytes(const SelectArgs &a) { return round_up((size_t)a.pv.n_rows * a.pv.n_kv * a.pages * 8 + 1); }

int check_sparse(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_paged_mask *mask, int n_heads, int n_select, SparseArgs *x) {
    AttnArgs &a = x->a;
    const char *what = "paged_sparse_attention";
    if (int rc = vla_check_paged(what, cache, batch, &a.pv)) return rc;
    if (!mask) { vla_set_error("%s: mask is NULL", what); return VLA_EINVAL; }
    if (n_heads <= 0 || n_heads % cache->n_kv_heads) { vla_set_error("%s: n_heads %d is no multiple of n_kv_heads %d", what, n_heads, cache->n_kv_heads); return VLA_ESHAPE; }
    if (n_heads > 4096) { vla_set_error("%s: n_heads %d unsupported (at most 4096)", what, n_heads); return VLA_ESHAPE; }
    if (!(mask->scale > 0.f) || !(mask->softcap >= 0.f) || !(mask->scale < INFINITY) || !(mask->softcap < INFINITY)) {
        vla_set_error("%s: scale must be positive, softcap not negative, both finite", what);
        return VLA_EINVAL;
    }
    if (mask->slopes || mask->prefix_len || mask->window || mask->shared_len) {
        vla_set_error("%s: slopes, prefix_len, window and shared_len have no meaning here", what);
        return VLA_EINVAL;
    }
    if (n_select < 1 || n_select > VLA_SELECT_PAGES) { vla_set_error("%s: n_select %d unsupported (1 .. %d)", what, n_select, VLA_SELECT_PAGES); return VLA_ESHAPE; }
    a.n_heads = n_heads; a.group = n_heads / cache->n_kv_heads;
    a.scale = mask->scale; a.cap = mask->softcap;
    x->n_select = n_select;
    x->heads_tiles = (a.group + 31) / 32;
    if ((long)batch->n_rows * cache->n_kv_heads * x->heads_tiles > 0x7fffffffL / 256 || (long)batch->n_rows * n_heads > 0x7fffffffL / 2) {
        vla_set_error("%s: %d rows of %d heads are too many", what, batch->n_rows, n_heads);
        return VLA_ESHAPE;
    }
    return VLA_OK;
}
// Waves enough to fill the chip, each with two tiles at least.
void plan_sparse(SparseArgs *x, bool f32) {
    AttnArgs &a = x->a;
    const long items = (long)a.pv.n_rows * a.pv.n_kv * x->heads_tiles;
    long pages = (a.pv.max_len + (1 << a.pv.page_log) - 1) >> a.pv.page_log;
    if (pages > x->n_select) pages = x->n_select;
    const long tiles = ((pages << a.pv.page_log) + 31) / 32;
    const int fit = 128 / ((128 * padded_dim(a.pv.d) * (f32 ? 4 : 2) + 1279) / 1280);
    const long waves = 256 * (fit > 8 ? 8 : fit);
    long parts = items > 0 ? waves / items : 1;
    if (parts > tiles / 2) parts = tiles / 2;
    a.parts = (int)(parts < 1 ? 1 : parts);
}
size_t lay_out(AttnArgs *a, char *base) {
    if (a->parts <= 1) return 256;
    const size_t slots = (size_t)a->pv.n_rows * a->n_heads * a->parts, ml = round_up(slots * sizeof(float2));
    a->ml = (float2 *)base;
    a->o_part = (float *)(base + ml);
    return ml + round_up(slots * a->pv.d * sizeof(float));
}

template <typename T, int DP, int MODE>
int launch(const SparseArgs &x, hipStream_t st) {
    const AttnArgs &a = x.a;
    constexpr size_t bytes = 2 * 2 * 32 * Tile<T, DP>::ROW;
    if (int rc = vla_allow_lds((const void *)paged_sparse_kernel<T, DP, MODE>, bytes)) return rc;
    paged_sparse_kernel<T, DP, MODE><<<dim3(a.pv.n_rows * a.pv.n_kv * x.heads_tiles, a.parts), 64, bytes, st>>>(x);
    if (int rc = vla_check_launch("paged_sparse_attention")) return rc;
    if (a.parts == 1) return VLA_OK;
    const int heads = (2048 + a.pv.n_rows - 1) / a.pv.n_rows;
    paged_join_kernel<T, DP><<<dim3(a.pv.n_rows, heads < a.n_heads ? heads : a.n_heads), 256, 0, st>>>(a);
    return vla_check_launch("paged_sparse_attention join");
}
template <typename T, int MODE>
int launch_sized(const SparseArgs &x, hipStream_t st) {
    switch (padded_dim(x.a.pv.d)) {
        case 64: return launch<T, 64, MODE>(x, st);
        case 128: return launch<T, 128, MODE>(x, st);
        default: return launch<T, 256, MODE>(x, st);
    }
}
template <typename T> int launch_typed(const SparseArgs &x, hipStream_t st) { return x.a.cap > 0.f ? launch_sized<T, CAPPED>(x, st) : launch_sized<T, 0>(x, st); }

}  // namespace

extern "C" {

int vla_paged_bounds(const vla_paged_cache *cache, const vla_paged_batch *batch, void *bounds, void *stream) {
    PagedView pv;
    if (int rc = vla_check_paged("paged_bounds", cache, batch, &pv)) return rc;
    if (int rc = check_bounds("paged_bounds", bounds)) return rc;
    if (pv.n_rows == 0 || pv.max_rows == 0 || pv.max_len == 0) return VLA_OK;
    // pages that max_rows rows may touch, whatever the first one's place in its page
    const int size = 1 << pv.page_log, all = (pv.max_len + size - 1) >> pv.page_log, some = (int)(((long)pv.max_rows + size - 2) >> pv.page_log) + 1, pages = some < all ? some : all;
    if (pages > 65535) { vla_set_error("paged_bounds: rows on %d pages of a sequence (at most 65,535)", pages); return VLA_ESHAPE; }
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps("paged_bounds", 0.0, st);
    if (cache->dtype == VLA_DTYPE_F32) paged_bounds_kernel<float><<<dim3(pv.n_seq, pages), 256, 0, st>>>(pv, (float *)bounds);
    else paged_bounds_kernel<bf16_t><<<dim3(pv.n_seq, pages), 256, 0, st>>>(pv, (bf16_t *)bounds);
    return vla_check_launch("paged_bounds");
}

size_t vla_paged_select_workspace_bytes(const vla_paged_cache *cache, const vla_paged_batch *batch) {
    PagedView pv;
    SelectArgs a{};
    if (vla_check_paged("paged_select", cache, batch, &pv) || check_pages(pv, &a)) return 0;
    return select_bytes(a);
}

int vla_paged_select(const vla_paged_cache *cache, const vla_paged_batch *batch, const void *bounds, const void *q, int n_heads,
                     int64_t q_stride, int n_select, int first, int recent, int32_t *selected, void *ws, size_t ws_bytes, void *stream) {
    PagedView pv;
    SelectArgs a{};
    if (int rc = vla_check_paged("paged_select", cache, batch, &pv)) return rc;
    if (int rc = check_pages(pv, &a)) return rc;
    if (int rc = check_bounds("paged_select", bounds)) return rc;
    if (n_heads <= 0 || n_heads % cache->n_kv_heads) { vla_set_error("paged_select: n_heads %d is no multiple of n_kv_heads %d", n_heads, cache->n_kv_heads); return VLA_ESHAPE; }
    if (n_heads > 4096) { vla_set_error("paged_select: n_heads %d unsupported (at most 4096)", n_heads); return VLA_ESHAPE; }
    if (first < 0 || recent < 1 || n_select > VLA_SELECT_PAGES || (long)first + recent > n_select) {
        vla_set_error("paged_select: n_select %d, first %d, recent %d (recent at least 1, n_select from first + recent to %d)", n_select, first, recent, VLA_SELECT_PAGES);
        return VLA_EINVAL;
    }
    if (batch->n_rows > 0 && (!q || !selected || !ws)) { vla_set_error("paged_select: q, selected or ws is NULL"); return VLA_EINVAL; }
    if ((uintptr_t)ws % 16) { vla_set_error("paged_select: ws is not 16-byte aligned"); return VLA_EINVAL; }
    if (q_stride < (int64_t)n_heads * cache->head_dim) { vla_set_error("paged_select: a row stride is shorter than its heads"); return VLA_ESHAPE; }
    if (batch->n_rows > 0 && ws_bytes < select_bytes(a)) { vla_set_error("paged_select: workspace %zu bytes, need %zu", ws_bytes, select_bytes(a)); return VLA_EWORKSPACE; }
    if (batch->n_rows == 0 || batch->max_rows == 0) return VLA_OK;
    a.bounds = bounds; a.q = q; a.q_stride = q_stride; a.group = n_heads / cache->n_kv_heads;
    a.n_select = n_select; a.first = first; a.recent = recent; a.keys = (unsigned long long *)ws; a.selected = selected;
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps("paged_select", 0.0, st);
    const int items = pv.n_rows * pv.n_kv;
    if (a.pages > n_select) {
        // workgroups for two rounds of four a CU, each with one step of the loop at least
        const bool f32 = cache->dtype == VLA_DTYPE_F32;
        const int chunks = 2 * pv.d * (f32 ? 4 : 2) / 16;
        int lanes_log = 0;
        while (lanes_log < 6 && (1 << lanes_log) < chunks) lanes_log++;
        const int step = 8 * (256 >> lanes_log);
        int y = (2048 + items - 1) / items;
        if (y > (a.pages + step - 1) / step) y = (a.pages + step - 1) / step;
        const int per_block = ((a.pages + y - 1) / y + step - 1) / step * step;
        y = (a.pages + per_block - 1) / per_block;
        if (f32) paged_score_kernel<float><<<dim3(items, y), 256, 0, st>>>(a, lanes_log, per_block);
        else paged_score_kernel<bf16_t><<<dim3(items, y), 256, 0, st>>>(a, lanes_log, per_block);
        if (int rc = vla_check_launch("paged_select scores")) return rc;
    }
    const size_t lds = (size_t)a.pages * 8;
    if (int rc = vla_allow_lds((const void *)paged_select_kernel, VLA_SELECT_PAGES * 8)) return rc;
    paged_select_kernel<<<items, 256, lds, st>>>(a);
    return vla_check_launch("paged_select");
}

size_t vla_paged_sparse_attention_workspace_bytes(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_paged_mask *mask,
                                                  int n_heads, int n_select) {
    SparseArgs x{};
    if (check_sparse(cache, batch, mask, n_heads, n_select, &x)) return 0;
    plan_sparse(&x, cache->dtype == VLA_DTYPE_F32);
    return lay_out(&x.a, nullptr);
}

int vla_paged_sparse_attention(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_paged_mask *mask,
                               const int32_t *selected, int n_select, const void *q, int n_heads, int64_t q_stride, void *out,
                               int64_t out_stride, float *lse, void *ws, size_t ws_bytes, void *stream) {
    SparseArgs x{};
    AttnArgs &a = x.a;
    if (int rc = check_sparse(cache, batch, mask, n_heads, n_select, &x)) return rc;
    const bool f32 = cache->dtype == VLA_DTYPE_F32;
    if (batch->n_rows > 0 && (!selected || !q || !out || !ws)) { vla_set_error("paged_sparse_attention: selected, q, out or ws is NULL"); return VLA_EINVAL; }
    if ((uintptr_t)ws % 16) { vla_set_error("paged_sparse_attention: ws is not 16-byte aligned"); return VLA_EINVAL; }
    if (q_stride < (int64_t)n_heads * cache->head_dim || out_stride < (int64_t)n_heads * cache->head_dim) {
        vla_set_error("paged_sparse_attention: a row stride is shorter than its heads");
        return VLA_ESHAPE;
    }
    plan_sparse(&x, f32);
    const size_t need = lay_out(&a, (char *)ws);
    if (batch->n_rows > 0 && ws_bytes < need) { vla_set_error("paged_sparse_attention: workspace %zu bytes, need %zu", ws_bytes, need); return VLA_EWORKSPACE; }
    if (batch->n_rows == 0 || batch->max_rows == 0) return VLA_OK;
    const size_t es = f32 ? 4 : 2;
    x.selected = selected;
    a.q = (const char *)q; a.out = (char *)out; a.lse = lse; a.q_stride = q_stride; a.o_stride = out_stride;
    a.aligned = ((uintptr_t)q | (uintptr_t)out | (size_t)q_stride * es | (size_t)out_stride * es) % 16 == 0;
    a.offset = !f32 ? a.cap * LOG2E : 0.f;
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps("paged_sparse_attention", 0.0, st);
    return f32 ? launch_typed<float>(x, st) : launch_typed<bf16_t>(x, st);
}

}  // extern "C"
