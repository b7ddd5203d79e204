// Attention of a ragged batch's new rows against a paged KV cache.
//
// Both products run transposed, on 32 x 32 matrix instructions: S^T = K Q^T (rows keys, columns queries) and O^T = V^T P^T (rows head
// dims), so a lane owns one query: its running maximum, sum and limits of visibility are scalars of the lane (and of lane ^ 32, which
// has the other half of the keys), and S^T's accumulators are P^T's operand as they lie once the sixteen keys of a lane pair are
// taken as the instruction's slots.  K and V go from memory to LDS without registers in between (global_load_lds, one kilobyte an instruction, 16 rows of
// one page at a time), V's columns come out of LDS transposed (ds_read_b64_tr_b16).  fp32 caches run the same code on
// v_mfma_f32_32x32x2_f32, eight instructions for one.
//
// The queries of a key head's group are rows like any others: row r of a sequence's "packed rows" is query r / group, head
// r % group.  Two forms: paged_prompt_kernel (128 packed rows, four waves of 32, one tile of keys for all) and paged_decode_kernel
// (up to 32 packed rows; every wave walks key tiles of its own through a ring of its own, no barriers).  Keys are split over workgroups where rows are
// few; the parts (maximum, sum, unscaled output) are joined in order by paged_join_kernel.  A prefix that all sequences share is a
// part of its own, whose packed rows are those of the whole batch.
//
// Weights are exp2 of scores in units of log2 e; the reference of a row moves only when its maximum has grown by more than 2^8, so
// sums stay below 2^8 times the count and most tiles rescale nothing.  P is rounded to bf16 once (relative 2^-8 of each weight, as the
// tolerances count it; the sum that divides is that of the unrounded weights).
#include "paged.h"

#include <type_traits>

namespace {

typedef float f32x8_t __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void lds_void;
typedef __attribute__((address_space(3))) bf16x4_t lds_bf16x4;

template <typename T> struct FragOf;
template <> struct FragOf<bf16_t> { typedef bf16x8_t type; };
template <> struct FragOf<float> { typedef f32x8_t type; };

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
    float offset;            // what scores lack, in log2 units (see Rows::tile): lse alone knows it
    int aligned;             // rows of q and out start at multiples of 16 bytes
    // this launch
    int whole;               // packed rows of the whole batch against the shared positions
    int row_tiles;           // tiles of packed rows per sequence (whole: in all)
    int chunk;               // keys per part
    int part0, parts;        // number of this launch's first part; parts of all launches (1: the output is written here)
    float2 *ml;              // [parts][n_rows][n_heads]: maximum (log2 units) and sum
    float *o_part;           // [parts][n_rows][n_heads][d]
};

// 16 bytes of zeros and more: what rows of pages that are not there are read from.
__device__ __attribute__((aligned(16))) float zero_row[256];

__device__ __forceinline__ f32x16_t mma(const bf16x8_t &x, const bf16x8_t &y, f32x16_t c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0); }
__device__ __forceinline__ f32x16_t mma(const f32x8_t &x, const f32x8_t &y, f32x16_t c) {
#pragma unroll
    for (int e = 0; e < 8; e++) c = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], c, 0, 0, 0);
    return c;
}

// One kilobyte: 16 bytes a lane from base + off to LDS at at + 16 lane.  No register is written; the waits are the caller's: the
// compiler, were it to know of the load, would wait for all of them before any read of LDS.  (Nothing else in these kernels uses m0.)
__device__ __forceinline__ void dma16(unsigned at, unsigned off, const char *base) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(at), "v"(off), "s"(base) : "memory");
}
template <int N> __device__ __forceinline__ void vm_wait() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N < 63 ? N : 63) : "memory"); }

// The keys of a part: [lo, hi) but for [g0, g1) (g0 = g1: all of them), a gap between a prefix and the windows behind it.
struct Span {
    int lo, hi, g0, g1;
    // the page of the 16 keys from key0 on
    __device__ __forceinline__ int page(const int32_t *table, int page_log, int key0) const {
        int k = min(max(key0, lo), hi - 1);
        if (key0 >= g0 && key0 + 15 < g1) k = g1;
        else if (k >= g0 && k < g1) k = key0 >= g0 || key0 + 15 >= g1 ? g1 : g0 - 1;
        return table[k >> page_log];
    }
};

// A tile of keys in LDS: rows of CPR 16-byte chunks; chunk c of row r sits at c ^ fk(r) (K: the 32 rows of an operand read in eight
// and sixteen lanes at a time fall on different banks) or c ^ fv(r) (V: four rows by 32 bytes of a transposing read do).
template <typename T, int DP> struct Tile {
    static constexpr int CPR = DP * (int)sizeof(T) / 16, ROW = CPR * 16, RPI = 64 / CPR;
    __device__ static int fk(int r) { return r & (CPR < 16 ? CPR - 1 : 15); }
    __device__ static int fv(int r) {
        if constexpr (sizeof(T) == 4) return 0;
        return 2 * (CPR < 16 ? r & 3 : (r & 3) | (r & 1) << 2);
    }
    // 16 rows from key0 on (a multiple of 16: one page) of K or V.  Keys that no query of the tile sees are not read: outside [lo, hi)
    // the nearest one inside takes their place, in [g0, g1) the nearest one outside.
    template <bool V>
    __device__ static void load16(unsigned at, const char *pool, const PagedView &pv, int page, int kvh, int key0, const Span &sp) {
        const int lane = threadIdx.x & 63, row_bytes = pv.d * (int)sizeof(T), chunks = row_bytes >> 4;
        const bool ok = (unsigned)page < (unsigned)pv.n_pages;
        const char *base = ok ? pool + (((size_t)page * pv.n_kv + kvh) << pv.page_log) * row_bytes : (const char *)zero_row;
        const int in_page = ok ? (1 << pv.page_log) - 1 : 0;
#pragma unroll
        for (int i = 0; i < 16 / RPI; i++) {
            const int r = i * RPI + lane / CPR;
            int key = min(max(key0 + r, sp.lo), sp.hi - 1);
            if (key >= sp.g0 && key < sp.g1) key = key0 >= sp.g0 || key0 + 15 >= sp.g1 ? sp.g1 : sp.g0 - 1;
            const int c = min((lane % CPR) ^ (V ? fv(r) : fk(r)), chunks - 1);
            dma16(at + i * 1024, (unsigned)((key & in_page) * row_bytes + c * 16), base);
        }
    }
};

constexpr int CAPPED = 1, BIASED = 2;          // bits of MODE

// What one lane knows of its query.
struct Query {
    int row, head;           // of the call
    int p, lo, hi, pre;      // visible keys: [lo, hi) and [0, pre)
    bool valid;
    float slope;
};

template <int MODE>
__device__ __forceinline__ Query make_query(const AttnArgs &a, int kvh, int s, int row, int i, const PagedSeq &sq, int hg, bool valid) {
    Query q;
    q.row = row;
    q.head = kvh * a.group + hg;
    q.valid = valid;
    q.p = sq.len - sq.n + i;
    q.pre = a.prefix_len && valid ? min(a.prefix_len[s], sq.keys) : 0;
    q.hi = min(sq.keys, q.p + 1);
    q.lo = a.whole ? 0 : a.shared_len;
    if (a.window) q.lo = max(0, q.p + 1 - a.window);
    else { q.hi = max(q.hi, q.pre); q.pre = 0; }
    q.slope = (MODE & BIASED) && valid ? a.slopes[q.head] : 0.f;
    if (!valid) { q.hi = 0x7fffffff; q.lo = 0; }
    return q;
}

template <typename T, int DP, int MODE> struct Rows {
    typedef typename FragOf<T>::type frag;
    typedef Tile<T, DP> TL;
    static constexpr int KS = DP / 16, DB = DP / 32;
    frag q[KS];
    f32x16_t o[DB];
    float m, l;

    __device__ __forceinline__ void start(const AttnArgs &a, const Query &y) {
        const int hh = (threadIdx.x >> 5) & 1, d = a.pv.d;
        const T *src = (const T *)a.q + y.row * a.q_stride + (size_t)y.head * d;
#pragma unroll
        for (int kk = 0; kk < KS; kk++) {
            const int dim = kk * 16 + hh * 8;
#pragma unroll
            for (int e = 0; e < 8; e++) q[kk][e] = (T)0.f;
            if (y.valid && dim < d) {
                if (a.aligned) {
                    if constexpr (sizeof(T) == 2) q[kk] = *(const frag *)(src + dim);
                    else {
                        const f32x4_t x = *(const f32x4_t *)(src + dim), z = *(const f32x4_t *)(src + dim + 4);
                        q[kk] = __builtin_shufflevector(x, z, 0, 1, 2, 3, 4, 5, 6, 7);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 8; e++) q[kk][e] = src[dim + e];
                }
            }
        }
#pragma unroll
        for (int b = 0; b < DB; b++)
#pragma unroll
            for (int i = 0; i < 16; i++) o[b][i] = 0.f;
        m = -INFINITY;
        l = 0.f;
    }

    // 32 NB keys from key0 on, K and V at kt and vt in LDS.  masked: some query may not see some key.
    template <int NB>
    __device__ __forceinline__ void tile(const AttnArgs &a, const Query &y, const char *kt, const char *vt, int key0, bool masked) {
        const int lane = threadIdx.x & 63, col = lane & 31, hh = lane >> 5;
        f32x16_t x[NB];
#pragma unroll
        for (int n = 0; n < NB; n++) {
#pragma unroll
            for (int i = 0; i < 16; i++) x[n][i] = 0.f;
#pragma unroll
            for (int kk = 0; kk < KS; kk++) {
                const char *row = kt + (n * 32 + col) * TL::ROW;
                frag k;
                if constexpr (sizeof(T) == 2) k = *(const frag *)(row + ((2 * kk + hh) ^ TL::fk(col)) * 16);
                else {
                    const f32x4_t u = *(const f32x4_t *)(row + ((4 * kk + 2 * hh) ^ TL::fk(col)) * 16), w = *(const f32x4_t *)(row + ((4 * kk + 2 * hh + 1) ^ TL::fk(col)) * 16);
                    k = __builtin_shufflevector(u, w, 0, 1, 2, 3, 4, 5, 6, 7);
                }
                x[n] = mma(k, q[kk], x[n]);
            }
        }
        // scores in log2 units are x unit (+ AttnArgs::offset, which changes no weight)
        constexpr float LOG2E = 1.4426950408889634f;
        float unit = a.scale * LOG2E;
        if (MODE & CAPPED) {
            if constexpr (sizeof(T) == 4) {
                const float back = a.scale / a.cap;
                unit = a.cap * LOG2E;
#pragma unroll
                for (int n = 0; n < NB; n++)
#pragma unroll
                    for (int i = 0; i < 16; i++) x[n][i] = tanhf(x[n][i] * back);
            } else {                                         // tanh t = 1 - 2 / (1 + e^2t); the 1 is the offset
                const float twice = 2.f * LOG2E * a.scale / a.cap;
                unit = 2.f * a.cap * LOG2E;
#pragma unroll
                for (int n = 0; n < NB; n++)
#pragma unroll
                    for (int i = 0; i < 16; i++) x[n][i] = -__builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x[n][i] * twice));
            }
        }
        if (MODE & BIASED) {
            const float slope = -y.slope * LOG2E, away = (float)(y.p - key0 - 4 * hh);
#pragma unroll
            for (int n = 0; n < NB; n++)
#pragma unroll
                for (int i = 0; i < 16; i++) x[n][i] = __builtin_fmaf(slope, fabsf(away - (float)(n * 32 + 8 * (i / 4) + i % 4)), x[n][i] * unit);
            unit = 1.f;
        }
        if (masked) {
#pragma unroll
            for (int n = 0; n < NB; n++)
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    const int j = key0 + n * 32 + 8 * (i / 4) + 4 * hh + i % 4;
                    if (!((j < y.hi && j >= y.lo) || j < y.pre)) x[n][i] = -INFINITY;
                }
        }
        float top = x[0][0];
#pragma unroll
        for (int n = 0; n < NB; n++)
#pragma unroll
            for (int i = 0; i < 16; i++) top = fmaxf(top, x[n][i]);
        top = vla_fold_step<32>(top, VlaMax()) * unit;
        if (__any(top > m + 8.f)) {                          // (m = -inf at first: any visible key)
            const float to = fmaxf(m, top), f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - to);
            l *= f;
#pragma unroll
            for (int b = 0; b < DB; b++)
#pragma unroll
                for (int i = 0; i < 16; i++) o[b][i] *= f;
            m = to;
        }
        const float ref = m == -INFINITY ? 0.f : m;
        frag p[2 * NB];
#pragma unroll
        for (int n = 0; n < NB; n++)
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(x[n][i], unit, -ref));
                l += w;
                p[2 * n + i / 8][i % 8] = (T)w;
            }
#pragma unroll
        for (int u = 0; u < 2 * NB; u++)
#pragma unroll
            for (int b = 0; b < DB; b++) {
                frag v;
                if constexpr (sizeof(T) == 2) {
                    const int l16 = lane & 15, r = u * 16 + 4 * hh + (l16 >> 2);
                    const int c = (b * 4 + ((lane >> 4) & 1) * 2 + ((l16 & 3) >> 1)) ^ TL::fv(l16 >> 2);
                    const char *at = vt + r * TL::ROW + c * 16 + (l16 & 1) * 8;
                    const auto v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)at), v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4 *)(at + 8 * TL::ROW));
                    v = __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; e++)
                        v[e] = *(const float *)(vt + (u * 16 + 8 * (e / 4) + 4 * hh + e % 4) * TL::ROW + (b * 32 + col) * 4);
                }
                o[b] = mma(v, p[u], o[b]);
            }
    }

    // One part's result: the output itself where there is one part, else the part's sums.
    __device__ __forceinline__ void finish(const AttnArgs &a, const Query &y, int part) {
        write(a, y, part, m, vla_fold_step<32>(l, VlaAdd()), (threadIdx.x >> 5) & 1);
    }
    __device__ __forceinline__ void write(const AttnArgs &a, const Query &y, int part, float m_, float sum, int hh) {
        const int d = a.pv.d;
        if (!y.valid) return;
        const size_t at = (size_t)y.row * a.n_heads + y.head, slot = (size_t)part * a.pv.n_rows * a.n_heads + at;
        if (a.parts > 1) {
            if (hh == 0) a.ml[slot] = make_float2(m_, sum);
            if (!(sum > 0.f)) return;                        // (the join reads nothing of an empty part)
            float *dst = a.o_part + slot * d;
#pragma unroll
            for (int b = 0; b < DB; b++)
#pragma unroll
                for (int g = 0; g < 4; g++) {
                    const int dim = b * 32 + g * 8 + hh * 4;
                    if (dim < d) *(f32x4_t *)(dst + dim) = f32x4_t{o[b][4 * g], o[b][4 * g + 1], o[b][4 * g + 2], o[b][4 * g + 3]};
                }
            return;
        }
        const float f = sum > 0.f ? 1.f / sum : 0.f;
        if (a.lse && hh == 0) a.lse[at] = sum > 0.f ? (m_ + a.offset + log2f(sum)) * 0.6931471805599453f : -INFINITY;
        T *dst = (T *)a.out + y.row * a.o_stride + (size_t)y.head * d;
#pragma unroll
        for (int b = 0; b < DB; b++)
#pragma unroll
            for (int g = 0; g < 4; g++) {
                const int dim = b * 32 + g * 8 + hh * 4;
                if (dim >= d) continue;
                if (a.aligned) {
                    typedef T t4 __attribute__((ext_vector_type(4)));
                    t4 w;
#pragma unroll
                    for (int e = 0; e < 4; e++) w[e] = (T)(o[b][4 * g + e] * f);
                    *(t4 *)(dst + dim) = w;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; e++) dst[dim + e] = (T)(o[b][4 * g + e] * f);
                }
            }
    }
};

// Packed rows first .. first + n - 1 of a launch's item -> the lane's query, and the keys any of them may see.
struct Item { int s, kvh, first, lo, hi, g0, g1; PagedSeq sq; };

__device__ __forceinline__ bool find_item(const AttnArgs &a, int id, int rows_per_tile, Item *it) {
    const PagedView &pv = a.pv;
    it->kvh = id % pv.n_kv;
    it->g0 = it->g1 = 0;
    id /= pv.n_kv;
    if (a.whole) {
        it->s = 0;
        it->first = id * rows_per_tile;
        it->lo = 0;
        it->hi = a.shared_len;
        it->sq = paged_seq(pv, 0);
        return it->first < min(pv.row_start[pv.n_seq], pv.n_rows) * a.group;
    }
    it->s = id % pv.n_seq;
    it->first = (a.row_tiles - 1 - id / pv.n_seq) * rows_per_tile;      // the last rows, which see most keys, first
    it->sq = paged_seq(pv, it->s);
    const int rows = it->sq.rows;
    if (it->first >= rows * a.group) return false;
    const int i0 = it->first / a.group, i1 = min(rows - 1, (it->first + rows_per_tile - 1) / a.group), p0 = it->sq.len - it->sq.n;
    const int prefix = a.prefix_len ? min(max(a.prefix_len[it->s], 0), it->sq.keys) : 0;
    it->hi = min(it->sq.keys, max(p0 + i1 + 1, prefix));
    const int from = a.window ? max(0, p0 + i0 + 1 - a.window) : 0;          // the first row's window, the lowest
    it->lo = max(a.shared_len, prefix == 0 ? from : 0);
    if (prefix > 0 && a.window) { it->g0 = prefix; it->g1 = max(prefix, min(from, it->hi - 1)); }
    return true;
}

template <int MODE>
__device__ __forceinline__ Query find_query(const AttnArgs &a, const Item &it, int r) {
    const int i = r / a.group, hg = r - i * a.group;
    if (!a.whole) return make_query<MODE>(a, it.kvh, it.s, it.sq.r0 + i, i, it.sq, hg, i < it.sq.rows);
    // row i of the batch: its sequence, by halving (row_start ascends)
    int lo = 0, hi = a.pv.n_seq;                              // row_start[lo] <= i < row_start[hi], if i is a row at all
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (a.pv.row_start[mid] <= i) lo = mid; else hi = mid;
    }
    const PagedSeq sq = paged_seq(a.pv, lo);
    const int at = i - sq.r0;
    Query q = make_query<MODE>(a, it.kvh, lo, i, at, sq, hg, at >= 0 && at < sq.rows);
    if (q.valid) { q.hi = min(q.hi, a.shared_len); q.pre = min(q.pre, a.shared_len); }
    return q;
}

__device__ __forceinline__ bool sees_all(const Query &y, int k0, int k1) { return (k1 <= y.hi && k0 >= y.lo) || k1 <= y.pre; }
__device__ __forceinline__ bool sees_none(const Query &y, int k0, int k1) { return !y.valid || ((k0 >= y.hi || k1 <= y.lo) && k0 >= y.pre); }

template <typename T, int DP, int MODE>
__global__ void __launch_bounds__(256) paged_prompt_kernel(AttnArgs a) {
    typedef Tile<T, DP> TL;
    constexpr int NB = sizeof(T) == 2 ? 2 : 1, KT = 32 * NB, BYTES = KT * TL::ROW, GROUPS = KT / 16;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const unsigned lds0 = (unsigned)(size_t)(lds_void *)lds;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Item it;
    if (!find_item(a, blockIdx.x, 128, &it)) return;
    const Query y = find_query<MODE>(a, it, it.first + wave * 32 + (threadIdx.x & 31));
    const int part = a.part0 + blockIdx.y, base = it.lo & ~(KT - 1), lo = max(it.lo, base + (int)blockIdx.y * a.chunk), hi = min(it.hi, base + ((int)blockIdx.y + 1) * a.chunk);
    Rows<T, DP, MODE> rows;
    rows.start(a, y);
    if (lo < hi) {
        const int32_t *table = a.pv.table + (size_t)it.s * a.pv.table_stride;
        const int t0 = lo / KT, t1 = (hi + KT - 1) / KT;
        const Span sp{lo, hi, it.g0, it.g1};
        auto page_of = [&](int t, int g) { return sp.page(table, a.pv.page_log, t * KT + g * 16); };
        // a wave's share of a tile: 16 rows of K and the same of V, or (GROUPS = 2) of one of them
        const int g = wave % GROUPS;
        auto load = [&](int t, int page) {
            const unsigned at = lds0 + (t & 1) * 2 * BYTES + g * 16 * TL::ROW;
            if (GROUPS == 4 || wave < 2) TL::template load16<false>(at, a.pv.k, a.pv, page, it.kvh, t * KT + g * 16, sp);
            if (GROUPS == 4 || wave >= 2) TL::template load16<true>(at + BYTES, a.pv.v, a.pv, page, it.kvh, t * KT + g * 16, sp);
        };
        load(t0, page_of(t0, g));
        int page = page_of(min(t0 + 1, t1 - 1), g);
        for (int t = t0; t < t1; t++) {
            // this tile has landed and everyone is through with the one before, whose place the next one takes
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
            if (t + 1 < t1) {
                load(t + 1, page);
                page = page_of(min(t + 2, t1 - 1), g);
            }
            const int k0 = t * KT;
            if (__all(sees_none(y, k0, k0 + KT))) continue;
            const char *kt = lds + (t & 1) * 2 * BYTES;
            rows.template tile<NB>(a, y, kt, kt + BYTES, k0, !__all(sees_all(y, max(k0, lo), k0 + KT) && k0 + KT <= hi && k0 >= lo));
        }
    }
    rows.finish(a, y, part);
}

template <typename T, int DP, int NW, int MODE>
__global__ void __launch_bounds__(64 * NW) paged_decode_kernel(AttnArgs a) {
    typedef Tile<T, DP> TL;
    constexpr int KT = 32, BYTES = KT * TL::ROW, STAGE = 2 * BYTES, LOADS = 4 * 16 / TL::RPI;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    char *ring = lds + wave * 2 * STAGE;
    const unsigned ring0 = (unsigned)(size_t)(lds_void *)ring;
    Item it;
    if (!find_item(a, blockIdx.x, 32, &it)) return;
    const Query y = find_query<MODE>(a, it, it.first + (lane & 31));
    const int part = a.part0 + blockIdx.y, base = it.lo & ~(KT - 1), lo = max(it.lo, base + (int)blockIdx.y * a.chunk), hi = min(it.hi, base + ((int)blockIdx.y + 1) * a.chunk);
    Rows<T, DP, MODE> rows;
    rows.start(a, y);
    const int t0 = lo / KT, t1 = lo < hi ? (hi + KT - 1) / KT : t0;
    if (t0 + wave < t1) {
        const int32_t *table = a.pv.table + (size_t)it.s * a.pv.table_stride;
        const Span sp{lo, hi, it.g0, it.g1};
        auto page_of = [&](int t, int g) { return sp.page(table, a.pv.page_log, t * KT + g * 16); };
        auto load = [&](int t, int stage, int p0, int p1) {
            const unsigned at = ring0 + stage * STAGE;
            TL::template load16<false>(at, a.pv.k, a.pv, p0, it.kvh, t * KT, sp);
            TL::template load16<false>(at + 16 * TL::ROW, a.pv.k, a.pv, p1, it.kvh, t * KT + 16, sp);
            TL::template load16<true>(at + BYTES, a.pv.v, a.pv, p0, it.kvh, t * KT, sp);
            TL::template load16<true>(at + BYTES + 16 * TL::ROW, a.pv.v, a.pv, p1, it.kvh, t * KT + 16, sp);
        };
        int t = t0 + wave, stage = 0;
        load(t, 0, page_of(t, 0), page_of(t, 1));
        int p0 = page_of(t + NW, 0), p1 = page_of(t + NW, 1);
        for (; t < t1; t += NW, stage ^= 1) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // the reads of the stage that is loaded again are through
            if (t + NW < t1) {
                load(t + NW, stage ^ 1, p0, p1);
                p0 = page_of(t + 2 * NW, 0);
                p1 = page_of(t + 2 * NW, 1);
                vm_wait<LOADS>();
            } else vm_wait<0>();
            const int k0 = t * KT;
            const char *kt = ring + stage * STAGE;
            rows.template tile<1>(a, y, kt, kt + BYTES, k0, !__all(sees_all(y, k0, k0 + KT) && k0 + KT <= hi && k0 >= lo));
        }
    }
    if constexpr (NW > 1) {
        // the waves' sums, joined by the first: maxima and sums through LDS, then the outputs, 32 dims at a time
        const float sum = vla_fold_step<32>(rows.l, VlaAdd());
        __syncthreads();
        float *x = (float *)lds;
        float2 *ml = (float2 *)(x + NW * 64 * 16);
        if (lane < 32) ml[wave * 32 + lane] = make_float2(rows.m, sum);
        __syncthreads();
        float top = -INFINITY, total = 0.f;
        for (int w = 0; w < NW; w++) top = fmaxf(top, ml[w * 32 + (lane & 31)].x);
        for (int w = 0; w < NW; w++) {
            const float2 v = ml[w * 32 + (lane & 31)];
            total += v.x == -INFINITY ? 0.f : v.y * __builtin_amdgcn_exp2f(v.x - top);
        }
        const float f = rows.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(rows.m - top);
#pragma unroll
        for (int b = 0; b < DP / 32; b++) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 16; i++) x[(wave * 16 + i) * 64 + lane] = rows.o[b][i] * f;
            __syncthreads();
            if (wave == 0) {
#pragma unroll
                for (int i = 0; i < 16; i++) {
                    float v = 0.f;
                    for (int w = 0; w < NW; w++) v += x[(w * 16 + i) * 64 + lane];
                    rows.o[b][i] = v;
                }
            }
        }
        if (wave == 0) rows.write(a, y, part, top, total, lane >> 5);
    } else rows.finish(a, y, part);
}

// The parts of one (row, head), joined by one workgroup: DP / 4 lanes a part, so 1024 / DP parts at a time, whose sums are added in one order.
// (One wave a pair and part after part: 41 us for 64 parts of 32 pairs, a memory latency each.)
template <typename T, int DP>
__global__ void __launch_bounds__(256) paged_join_kernel(AttnArgs a) {
    constexpr int LANES = DP / 4, AT_ONCE = 256 / LANES;
    __shared__ f32x4_t sums[256];
    const PagedView &pv = a.pv;
    const int row = blockIdx.x, h = blockIdx.y, t = threadIdx.x, lane = t & 63, d = pv.d;
    const int s = paged_seq_of_row(pv, row);
    if (s >= pv.n_seq) return;
    const PagedSeq sq = paged_seq(pv, s);
    if (row - sq.r0 < 0 || row - sq.r0 >= sq.rows) return;
    const size_t step = (size_t)pv.n_rows * a.n_heads, at = (size_t)row * a.n_heads + h;
    float top = -INFINITY, sum = 0.f;
    for (int z = lane; z < a.parts; z += 64) top = fmaxf(top, a.ml[z * step + at].x);
    top = vla_wave_fold(top, VlaMax());
    auto share = [&](float2 v) { return v.y > 0.f ? __builtin_amdgcn_exp2f(v.x - top) : 0.f; };
    for (int z = lane; z < a.parts; z += 64) { const float2 v = a.ml[z * step + at]; sum += share(v) * v.y; }
    sum = vla_wave_sum(sum);
    const int dim = (t % LANES) * 4;
    f32x4_t o = {0.f, 0.f, 0.f, 0.f};
    if (dim < d)
#pragma unroll 4
        for (int z = t / LANES; z < a.parts; z += AT_ONCE) {
            const float f = share(a.ml[z * step + at]);
            if (f > 0.f) {
                const f32x4_t v = *(const f32x4_t *)(a.o_part + (z * step + at) * d + dim);
#pragma unroll
                for (int e = 0; e < 4; e++) o[e] += f * v[e];
            }
        }
    sums[t] = o;
    __syncthreads();
    if (t >= LANES || dim >= d) return;
    for (int i = 1; i < AT_ONCE; i++) {
        const f32x4_t v = sums[i * LANES + t];
#pragma unroll
        for (int e = 0; e < 4; e++) o[e] += v[e];
    }
    const float f = sum > 0.f ? 1.f / sum : 0.f;
    T *dst = (T *)a.out + row * a.o_stride + (size_t)h * d + dim;
#pragma unroll
    for (int e = 0; e < 4; e++) dst[e] = (T)(o[e] * f);
    if (a.lse && t == 0) a.lse[at] = sum > 0.f ? (top + a.offset + log2f(sum)) * 0.6931471805599453f : -INFINITY;
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
    if (mask->window && mask->shared_len) { vla_set_error("paged_attention: a window and a shared prefix exclude each other"); return VLA_EINVAL; }
    if (mask->shared_len % cache->page_size || mask->shared_len > batch->max_len) {
        vla_set_error("paged_attention: shared_len %d is no multiple of page_size %d or exceeds max_len %d", mask->shared_len, cache->page_size, batch->max_len);
        return VLA_ESHAPE;
    }
    if ((long)batch->n_rows * n_heads > 0x7fffffffL / 2) { vla_set_error("paged_attention: %d rows of %d heads are too many", batch->n_rows, n_heads); return VLA_ESHAPE; }
    a->n_heads = n_heads; a->group = n_heads / cache->n_kv_heads;
    a->scale = mask->scale; a->cap = mask->softcap; a->slopes = mask->slopes; a->prefix_len = mask->prefix_len;
    a->window = mask->window; a->shared_len = mask->shared_len;
    return VLA_OK;
}

// One launch: which kernel, its tiles of packed rows and its parts.
struct Launch { bool prompt; int nw, row_tiles, parts, chunk; long items; };
struct Plan { Launch own, whole; int parts; bool has_whole; };

int padded_dim(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

Launch plan_launch(const AttnArgs &a, bool f32, bool whole) {
    Launch p{};
    const int dp = padded_dim(a.pv.d), row = dp * (f32 ? 4 : 2);
    const long packed = (long)(whole ? a.pv.n_rows : a.pv.max_rows) * a.group;
    p.prompt = packed > 32;
    // the longest range of keys of one tile of rows; it starts at a multiple of 64 unless a window or a short shared prefix moves it
    long keys = whole ? a.shared_len : a.pv.max_len - a.shared_len;
    if (a.window && !a.prefix_len && keys > (long)a.window + (p.prompt ? 128 : 32)) keys = a.window + (p.prompt ? 128 : 32);
    if (!whole && (a.window || a.shared_len % 64)) keys += 63;
    p.row_tiles = (int)((packed + (p.prompt ? 127 : 31)) / (p.prompt ? 128 : 32));
    p.items = (long)p.row_tiles * (whole ? 1 : a.pv.n_seq) * a.pv.n_kv;
    // A decode wave's ring is 128 rows: four waves a workgroup where four rings fit a CU's LDS and there are keys enough for each
    p.nw = !p.prompt && row <= 256 && keys > 512 ? 4 : 1;
    // Parts: as many as fill the chip, none under 256 keys
    const long want = p.prompt ? 512 : p.nw == 4 ? 512 : 1024, most = (keys + 255) / 256;
    long parts = p.items > 0 ? (want + p.items - 1) / p.items : 1;
    if (parts > most) parts = most;
    if (parts < 1) parts = 1;
    p.chunk = (int)(((keys + parts - 1) / parts + 63) / 64 * 64);
    if (p.chunk < 64) p.chunk = 64;
    p.parts = (int)((keys + p.chunk - 1) / p.chunk);
    if (p.parts < 1) p.parts = 1;
    return p;
}
Plan plan(const AttnArgs &a, bool f32) {
    Plan p{};
    p.own = plan_launch(a, f32, false);
    p.has_whole = a.shared_len > 0;
    if (p.has_whole) p.whole = plan_launch(a, f32, true);
    p.parts = p.own.parts + (p.has_whole ? p.whole.parts : 0);
    return p;
}
size_t workspace(const AttnArgs &a, const Plan &p) {
    const size_t slots = (size_t)a.pv.n_rows * a.n_heads * p.parts;
    return p.parts > 1 ? ((slots * sizeof(float2) + 255) / 256 * 256) + slots * a.pv.d * sizeof(float) : 256;
}

template <typename T, int DP, int MODE>
int launch_form(const AttnArgs &a, const Launch &p, hipStream_t st) {
    typedef Tile<T, DP> TL;
    const dim3 grid((unsigned)p.items, p.parts);
    if (p.prompt) {
        constexpr size_t bytes = 2 * 2 * (sizeof(T) == 2 ? 64 : 32) * TL::ROW;
        if (int rc = vla_allow_lds((const void *)paged_prompt_kernel<T, DP, MODE>, bytes)) return rc;
        paged_prompt_kernel<T, DP, MODE><<<grid, 256, bytes, st>>>(a);
    } else if (p.nw == 4) {
        if constexpr (TL::ROW <= 256) {
            constexpr size_t bytes = 4 * 2 * 2 * 32 * TL::ROW;
            static_assert(bytes >= 4 * 64 * 16 * 4 + 4 * 32 * 8, "the join's panel");
            if (int rc = vla_allow_lds((const void *)paged_decode_kernel<T, DP, 4, MODE>, bytes)) return rc;
            paged_decode_kernel<T, DP, 4, MODE><<<grid, 256, bytes, st>>>(a);
        }
    } else {
        constexpr size_t bytes = 2 * 2 * 32 * TL::ROW;
        if (int rc = vla_allow_lds((const void *)paged_decode_kernel<T, DP, 1, MODE>, bytes)) return rc;
        paged_decode_kernel<T, DP, 1, MODE><<<grid, 64, bytes, st>>>(a);
    }
    return vla_check_launch("paged_attention");
}
template <typename T, int MODE>
int launch_sized(const AttnArgs &a, const Launch &p, hipStream_t st) {
    switch (padded_dim(a.pv.d)) {
        case 64: return launch_form<T, 64, MODE>(a, p, st);
        case 128: return launch_form<T, 128, MODE>(a, p, st);
        default: return launch_form<T, 256, MODE>(a, p, st);
    }
}
template <typename T>
int launch_typed(const AttnArgs &a, const Launch &p, hipStream_t st) {
    switch ((a.cap > 0.f ? CAPPED : 0) | (a.slopes ? BIASED : 0)) {
        case 0: return launch_sized<T, 0>(a, p, st);
        case CAPPED: return launch_sized<T, CAPPED>(a, p, st);
        case BIASED: return launch_sized<T, BIASED>(a, p, st);
        default: return launch_sized<T, CAPPED | BIASED>(a, p, st);
    }
}
template <typename T>
int attend(AttnArgs a, const Plan &p, void *ws, hipStream_t st) {
    a.parts = p.parts;
    const size_t slots = (size_t)a.pv.n_rows * a.n_heads * p.parts;
    a.ml = (float2 *)ws;
    a.o_part = (float *)((char *)ws + (slots * sizeof(float2) + 255) / 256 * 256);
    int rc;
    if (p.has_whole) {
        AttnArgs w = a;
        w.whole = 1; w.row_tiles = p.whole.row_tiles; w.chunk = p.whole.chunk; w.part0 = p.own.parts;
        if ((rc = launch_typed<T>(w, p.whole, st))) return rc;
    }
    a.row_tiles = p.own.row_tiles; a.chunk = p.own.chunk;
    if ((rc = launch_typed<T>(a, p.own, st))) return rc;
    if (p.parts == 1) return VLA_OK;
    const dim3 grid(a.pv.n_rows, a.n_heads);
    switch (padded_dim(a.pv.d)) {
        case 64: paged_join_kernel<T, 64><<<grid, 256, 0, st>>>(a); break;
        case 128: paged_join_kernel<T, 128><<<grid, 256, 0, st>>>(a); break;
        default: paged_join_kernel<T, 256><<<grid, 256, 0, st>>>(a);
    }
    return vla_check_launch("paged_attention join");
}

}  // namespace

extern "C" {

size_t vla_paged_attention_workspace_bytes(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_paged_mask *mask, int n_heads) {
    AttnArgs a{};
    if (check(cache, batch, mask, n_heads, &a)) return 0;
    return workspace(a, plan(a, cache->dtype == VLA_DTYPE_F32));
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
    const bool f32 = cache->dtype == VLA_DTYPE_F32;
    const Plan p = plan(a, f32);
    const size_t need = workspace(a, p);
    if (ws_bytes < need) { vla_set_error("paged_attention: workspace %zu bytes, need %zu", ws_bytes, need); return VLA_EWORKSPACE; }
    if (batch->n_rows == 0 || batch->max_rows == 0) return VLA_OK;
    if (p.own.items > 0x7fffffffL) { vla_set_error("paged_attention: %ld tiles of rows are too many: split the batch", p.own.items); return VLA_ESHAPE; }
    const size_t es = f32 ? 4 : 2;
    a.q = (const char *)q; a.out = (char *)out; a.lse = lse; a.q_stride = q_stride; a.o_stride = out_stride;
    a.aligned = ((uintptr_t)q | (uintptr_t)out | (size_t)q_stride * es | (size_t)out_stride * es) % 16 == 0;
    a.offset = !f32 ? a.cap * 1.4426950408889634f : 0.f;
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps("paged_attention", 0.0, st);
    return f32 ? attend<float>(a, p, ws, st) : attend<bf16_t>(a, p, ws, st);
}

}  // extern "C"
