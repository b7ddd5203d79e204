// What the attention kernels of the paged cache (paged_attention.hip, paged_sparse.hip) and the sums of their weights (paged_evict.hip) share: tiles of keys in LDS, the two products with
// the online softmax between them, the sums of parts and their join.  The mathematics is described at the top of paged_attention.hip.
#pragma once
#include "paged.h"

#include <type_traits>

namespace {

// A window that reaches before every position (there are 2^30 at most) is one of 2^30: positions less a window, rows at negative ones among them, stay numbers of 32 bits.
int mask_window(const vla_paged_mask &mask) { return mask.window < 1 << 30 ? mask.window : 1 << 30; }
int padded_dim(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }
size_t round_up(size_t v) { return (v + 255) / 256 * 256; }

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
    const int32_t *seen;     // drafted trees: [n_rows][words], bit j of a row: it sees its sequence's new row j
    int words;
    float offset;            // what scores lack, in log2 units (see Rows::shaped): lse alone knows it
    int aligned;             // rows of q and out start at multiples of 16 bytes
    // this launch
    int decode;              // the new rows' own keys in decode form
    int whole;               // packed rows of the whole batch against the shared positions
    int row_tiles;           // tiles of packed rows per sequence (whole: in all)
    int chunk;               // keys per part
    int part0, parts;        // number of this launch's first part; parts of all launches (1: the output is written here)
    int waves, packed;       // decode: waves among which a key head's tiles are divided (0: one per sequence and key head); packed rows of a sequence at most
    int2 *seq_waves;         // [n_seq]: the first wave that has a sequence, and how many have
    float2 *wave_ml;         // [waves][n_kv][2][packed]: parts of sequences that several waves share
    float *wave_o;           // [waves][n_kv][2][packed][d]
    float2 *ml;              // [parts][n_rows][n_heads]: maximum (log2 units) and sum
    float *o_part;           // [parts][n_rows][n_heads][d]
};

__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = min(v, __shfl_xor(v, o, 64));
    return __builtin_amdgcn_readfirstlane(v);
}
__device__ __forceinline__ int wave_sum(int v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}

// What rows of pages that are not there are read from: 16 of the longest.
__device__ __attribute__((aligned(16))) float zero_rows[16 * 256];

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
        return paged_int(table, k >> page_log);
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
    // ROWS rows from row r0 on of the 16 keys from key0 on (a multiple of 16: one page), of K or V.  Keys that no query of the tile sees are not read: outside [lo, hi)
    // the nearest one inside takes their place, in [g0, g1) the nearest one outside.
    template <bool V, int ROWS>
    __device__ __forceinline__ static void load(unsigned at, const char *pool, const PagedView &pv, int page, int kvh, int key0, const Span &sp, int r0 = 0) {
        const int lane = threadIdx.x & 63, row_bytes = pv.d * (int)sizeof(T), chunks = row_bytes >> 4;
        const bool ok = (unsigned)page < (unsigned)pv.n_pages;
        const char *base = ok ? pool + (((size_t)page * pv.n_kv + kvh) << pv.page_log) * row_bytes : (const char *)zero_rows;
        const int in_page = ok ? (1 << pv.page_log) - 1 : 0;
#pragma unroll
        for (int i = 0; i < ROWS / RPI; i++) {
            const int r = r0 + i * RPI + lane / CPR;
            int key = min(max(key0 + r, sp.lo), sp.hi - 1);
            if (key >= sp.g0 && key < sp.g1) key = key0 >= sp.g0 || key0 + 15 >= sp.g1 ? sp.g1 : sp.g0 - 1;
            const int c = min((lane % CPR) ^ (V ? fv(r) : fk(r)), chunks - 1);
            dma16(at + i * 1024, (unsigned)((key & in_page) * row_bytes + c * 16), base);
        }
    }
    // The same where all of the rows are read: a lane's offsets do not change from tile to tile.
    template <bool V, int ROWS> struct Offsets {
        unsigned off[ROWS / RPI];
        __device__ __forceinline__ void start(const PagedView &pv, int r0) {
            const int lane = threadIdx.x & 63, row_bytes = pv.d * (int)sizeof(T), chunks = row_bytes >> 4;
#pragma unroll
            for (int i = 0; i < ROWS / RPI; i++) {
                const int r = r0 + i * RPI + lane / CPR;
                off[i] = r * row_bytes + min((lane % CPR) ^ (V ? fv(r) : fk(r)), chunks - 1) * 16;
            }
        }
        __device__ __forceinline__ void load(unsigned at, const char *rows) const {
#pragma unroll
            for (int i = 0; i < ROWS / RPI; i++) dma16(at + i * 1024, off[i], rows);
        }
    };
};
// Where the 16 keys from key0 on begin in k and in v.
struct Place {
    unsigned page_bytes, head_bytes, row_bytes;
    __device__ __forceinline__ Place(const PagedView &pv, int kvh, int size) {
        row_bytes = pv.d * size;
        head_bytes = ((unsigned)kvh << pv.page_log) * row_bytes;
        page_bytes = ((unsigned)pv.n_kv << pv.page_log) * row_bytes;
    }
    __device__ __forceinline__ size_t at(const PagedView &pv, int page, int key0) const {
        return (size_t)(unsigned)page * page_bytes + head_bytes + (key0 & ((1 << pv.page_log) - 1)) * row_bytes;
    }
    __device__ __forceinline__ const char *in(const PagedView &pv, const char *pool, int page, size_t at) const {
        return (unsigned)page < (unsigned)pv.n_pages ? pool + at : (const char *)zero_rows;
    }
};

constexpr float LOG2E = 1.4426950408889634f;
constexpr int CAPPED = 1, BIASED = 2, TREE = 4;          // bits of MODE

// What one lane knows of its query.
struct Query {
    int row, head;           // of the call
    int p, lo, hi, pre;      // visible keys: [lo, hi) and [0, pre)
    bool valid;
    float slope;
    const int32_t *seen;     // TREE: its bits; position of the first new row, keys there are
    int base, keys, words;
    // Which of the 32 keys from key0 on are new rows that it sees.
    __device__ __forceinline__ unsigned drafts(int key0) const {
        const int first = key0 - base, w = first >> 5, off = first & 31, left = keys - key0;
        const unsigned lo = w >= 0 && w < words ? seen[w] : 0u, hi = off && w + 1 >= 0 && w + 1 < words ? seen[w + 1] : 0u;
        const unsigned bits = off ? lo >> off | hi << (32 - off) : lo;
        return left <= 0 ? 0u : left < 32 ? bits & ((1u << left) - 1u) : bits;
    }
};

template <int MODE>
__device__ __forceinline__ Query make_query(const AttnArgs &a, int kvh, int s, int row, int i, const PagedSeq &sq, int hg, bool valid) {
    Query q;
    q.row = row;
    q.head = kvh * a.group + hg;
    q.valid = valid;
    q.p = sq.len - sq.n + i;
    q.pre = a.prefix_len && valid ? min(paged_int(a.prefix_len, s), sq.keys) : 0;
    q.hi = min(sq.keys, q.p + 1);
    q.lo = a.whole ? 0 : a.shared_len;
    if constexpr (MODE & TREE) {
        q.base = sq.len - sq.n;
        q.keys = sq.keys;
        q.words = valid ? a.words : 0;
        q.seen = a.seen + (size_t)row * a.words;
        q.hi = min(sq.keys, q.base);
        q.pre = 0;
    } else if (a.window) q.lo = max(0, q.p + 1 - a.window);
    else { q.hi = max(q.hi, q.pre); q.pre = 0; }
    q.slope = (MODE & BIASED) && valid ? a.slopes[q.head] : 0.f;
    if (!valid) { q.hi = 0x7fffffff; q.lo = 0; }
    return q;
}

// ln of a row's sum of exponentials; -inf where it sees no key.
__device__ __forceinline__ float lse_of(const AttnArgs &a, float m, float sum) { return sum == 0.f ? -INFINITY : (m + a.offset + log2f(sum)) * 0.6931471805599453f; }

// TAILS (bf16): weights enter the product with V as head and tail.
template <typename T, int DP, int MODE, bool TAILS> struct Rows {
    typedef typename FragOf<T>::type frag;
    typedef Tile<T, DP> TL;
    static constexpr int KS = DP / 16, DB = DP / 32, HALVES = TAILS ? 2 : 1;
    // A lane's weights of a tile as matrix operands: bf16 head (and tail), or the fp32 weights.
    struct Weights {
        frag p[HALVES][2];
        __device__ __forceinline__ void put(int i, float w) {
            p[0][i / 8][i % 8] = (T)w;
            if constexpr (HALVES == 2) p[1][i / 8][i % 8] = (T)(w - (float)p[0][i / 8][i % 8]);
        }
    };
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
        // (here the compiler waits for them: left to the first use, inside the loop over tiles, it would wait for everything in flight at every tile)
#pragma unroll
        for (int kk = 0; kk < KS; kk++) asm volatile("" : "+v"(q[kk]));
#pragma unroll
        for (int b = 0; b < DB; b++)
#pragma unroll
            for (int i = 0; i < 16; i++) o[b][i] = 0.f;
        m = -INFINITY;
        l = 0.f;
    }

    // The steps of a tile of 32 keys from key0 on, K and V at kt and vt in LDS.  Scores: a lane's query against 16 of the keys,
    // register i is key 8 (i / 4) + 4 hh + i % 4.
    __device__ __forceinline__ static frag key(const char *kt, int kk) {
        const int lane = threadIdx.x & 63, col = lane & 31, hh = lane >> 5;
        const char *row = kt + col * TL::ROW;
        if constexpr (sizeof(T) == 2) return *(const frag *)(row + ((2 * kk + hh) ^ TL::fk(col)) * 16);
        else {
            const f32x4_t u = *(const f32x4_t *)(row + ((4 * kk + 2 * hh) ^ TL::fk(col)) * 16), w = *(const f32x4_t *)(row + ((4 * kk + 2 * hh + 1) ^ TL::fk(col)) * 16);
            return __builtin_shufflevector(u, w, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
    __device__ __forceinline__ void scores(f32x16_t &x, const char *kt) const {
#pragma unroll
        for (int i = 0; i < 16; i++) x[i] = 0.f;
#pragma unroll
        for (int kk = 0; kk < KS; kk++) x = mma(key(kt, kk), q[kk], x);
    }
    // scores(next, kt) and weights(p, x) in turn: a matrix instruction, then the vector work it covers (left to itself the compiler
    // puts all of the one before all of the other).  The operands come out of LDS three instructions ahead.
    __device__ __forceinline__ void scores_and_weights(f32x16_t &next, const char *kt, Weights &p, const f32x16_t &x, float unit) {
        constexpr int EACH = 16 / KS, AHEAD = KS < 3 ? KS : 3;
        const float ref = m == -INFINITY ? 0.f : m;
        frag k[AHEAD];
#pragma unroll
        for (int kk = 0; kk < AHEAD; kk++) k[kk] = key(kt, kk);
#pragma unroll
        for (int i = 0; i < 16; i++) next[i] = 0.f;
#pragma unroll
        for (int kk = 0; kk < KS; kk++) {
            __builtin_amdgcn_sched_barrier(0);
            next = mma(k[kk % AHEAD], q[kk], next);
            if (kk + AHEAD < KS) k[kk % AHEAD] = key(kt, kk + AHEAD);
#pragma unroll
            for (int i = kk * EACH; i < (kk + 1) * EACH; i++) {
                const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], unit, -ref));
                l += w;
                p.put(i, w);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    }
    // values(p, vt), and in its cover shape and the largest of `next`.  Two products by heads, then the same two by tails: none waits for the one before it.
    __device__ __forceinline__ float values_and_largest(const Weights &p, const char *vt, f32x16_t &next, const AttnArgs &a, const Query &y, int key0) {
        constexpr int N = 2 * DB, EACH = (16 + N * HALVES - 1) / (N * HALVES), AHEAD = TAILS ? 4 : 3;
        frag v[AHEAD];
        float top = -INFINITY;
#pragma unroll
        for (int s = 0; s < AHEAD; s++) v[s] = value(vt, s / DB, s % DB);
#pragma unroll
        for (int n = 0; n < N * HALVES; n++) {
            const int half = n / 2 % HALVES, s = n / (2 * HALVES) * 2 + n % 2;
            __builtin_amdgcn_sched_barrier(0);
            o[s % DB] = mma(v[s % AHEAD], p.p[half][s / DB], o[s % DB]);
            if (half == HALVES - 1 && s + AHEAD < N) v[s % AHEAD] = value(vt, (s + AHEAD) / DB, (s + AHEAD) % DB);
#pragma unroll
            for (int i = n * EACH; i < (n + 1) * EACH && i < 16; i++) {
                next[i] = shaped(next[i], a, y, key0, i);
                top = fmaxf(top, next[i]);
            }
        }
        __builtin_amdgcn_sched_barrier(0);
        return vla_fold_step<32>(top, VlaMax()) * unit_of(a);
    }
    // Scores in log2 units are x unit (+ AttnArgs::offset, which changes no weight).
    __device__ __forceinline__ static float unit_of(const AttnArgs &a) {
        if (MODE & BIASED) return 1.f;
        if (MODE & CAPPED) return (sizeof(T) == 4 ? 1.f : 2.f) * a.cap * LOG2E;
        return a.scale * LOG2E;
    }
    // One score of the tile from key0 on; i as in scores.
    __device__ __forceinline__ static float shaped(float x, const AttnArgs &a, const Query &y, int key0, int i) {
        float unit = a.scale * LOG2E;
        if (MODE & CAPPED) {
            if constexpr (sizeof(T) == 4) {
                unit = a.cap * LOG2E;
                x = tanhf(x * (a.scale / a.cap));
            } else {                                         // tanh t = 1 - 2 / (1 + e^2t); the 1 is the offset
                unit = 2.f * a.cap * LOG2E;
                x = -__builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(x * (2.f * LOG2E * a.scale / a.cap)));
            }
        }
        if (MODE & BIASED) {
            const float away = (float)(y.p - key0 - 4 * (int)((threadIdx.x >> 5) & 1));
            x = __builtin_fmaf(-y.slope * LOG2E, fabsf(away - (float)(8 * (i / 4) + i % 4)), x * unit);
        }
        return x;
    }
    __device__ __forceinline__ static void hide(f32x16_t &x, const Query &y, int key0) {
        const int j0 = key0 + 4 * (int)((threadIdx.x >> 5) & 1);
        unsigned drafts = 0u;
        if constexpr (MODE & TREE) drafts = y.drafts(key0) >> (j0 - key0);
#pragma unroll
        for (int i = 0; i < 16; i++) {
            const int at = 8 * (i / 4) + i % 4, j = j0 + at;
            if constexpr (MODE & TREE) {
                if (!((j < y.hi && j >= y.lo) || (drafts >> at & 1u))) x[i] = -INFINITY;
            } else if (!((j < y.hi && j >= y.lo) || j < y.pre)) x[i] = -INFINITY;
        }
    }
    // The largest of a query's scores, in log2 units.
    __device__ __forceinline__ static float largest(const f32x16_t &x, float unit) {
        float top = x[0];
#pragma unroll
        for (int i = 1; i < 16; i++) top = fmaxf(top, x[i]);
        return vla_fold_step<32>(top, VlaMax()) * unit;
    }
    __device__ __forceinline__ void move_to(float top) {
        if (__any(top > m + 8.f)) {                          // (m = -inf at first: any visible key)
            const float to = fmaxf(m, top), f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - to);
            l *= f;
#pragma unroll
            for (int b = 0; b < DB; b++)
#pragma unroll
                for (int i = 0; i < 16; i++) o[b][i] *= f;
            m = to;
        }
    }
    __device__ __forceinline__ void weights(Weights &p, const f32x16_t &x, float unit) {
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int i = 0; i < 16; i++) {
            const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(x[i], unit, -ref));
            l += w;
            p.put(i, w);
        }
    }
    __device__ __forceinline__ static frag value(const char *vt, int u, int b) {
        const int lane = threadIdx.x & 63, col = lane & 31, hh = lane >> 5;
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
        return v;
    }
    __device__ __forceinline__ void values(const Weights &p, const char *vt) {
#pragma unroll
        for (int u = 0; u < 2; u++)
#pragma unroll
            for (int b = 0; b < DB; b++) {
                const frag v = value(vt, u, b);
#pragma unroll
                for (int half = 0; half < HALVES; half++) o[b] = mma(v, p.p[half][u], o[b]);
            }
    }
    // masked: some query may not see some key.
    __device__ __forceinline__ void tile(const AttnArgs &a, const Query &y, const char *kt, const char *vt, int key0, bool masked) {
        f32x16_t x;
        Weights p;
        scores(x, kt);
#pragma unroll
        for (int i = 0; i < 16; i++) x[i] = shaped(x[i], a, y, key0, i);
        if (masked) hide(x, y, key0);
        move_to(largest(x, unit_of(a)));
        weights(p, x, unit_of(a));
        values(p, vt);
    }

    // A part's sums.  (It is empty where its sum is zero: a sum that is no number belongs to the output.)
    __device__ __forceinline__ void keep(const AttnArgs &a, float2 *ml, float *dst, float sum, int hh) {
        if (hh == 0) *ml = make_float2(m, sum);
        if (sum == 0.f) return;                              // (the join reads nothing of an empty part)
#pragma unroll
        for (int b = 0; b < DB; b++)
#pragma unroll
            for (int g = 0; g < 4; g++) {
                const int dim = b * 32 + g * 8 + hh * 4;
                if (dim < a.pv.d) *(f32x4_t *)(dst + dim) = f32x4_t{o[b][4 * g], o[b][4 * g + 1], o[b][4 * g + 2], o[b][4 * g + 3]};
            }
    }
    // The output itself where there is one part, else the part's sums.
    __device__ __forceinline__ void finish(const AttnArgs &a, const Query &y, int part) {
        const int d = a.pv.d, hh = (threadIdx.x >> 5) & 1;
        const float sum = vla_fold_step<32>(l, VlaAdd());
        if (!y.valid) return;
        const size_t at = (size_t)y.row * a.n_heads + y.head, slot = (size_t)part * a.pv.n_rows * a.n_heads + at;
        if (a.parts > 1) {
            keep(a, a.ml + slot, a.o_part + slot * d, sum, hh);
            return;
        }
        const float f = sum == 0.f ? 0.f : 1.f / sum;
        if (a.lse && hh == 0) a.lse[at] = lse_of(a, m, sum);
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

// The parts of a row's heads.  FEW or less, as where a prompt's keys are in two parts or a decode wave's end falls into a sequence: DP / 4 lanes
// a (row, head) read them at once (4000 rows of 16 heads in two parts: 11 us; a workgroup for each 90).  More: a workgroup for each (row, head),
// DP / 4 lanes a part, so 1024 / DP parts at a time, whose sums are added in one order.  (One wave and part after part: 41 us for 64 parts of 32
// pairs, a memory latency each.)  The parts of all rows' layout (ml, o_part) come first, then those of the waves that shared the sequence.
constexpr int FEW = 4;
constexpr float EMPTY = -1.f;                    // of a part without a visible key, where weights stand
constexpr int JOIN_PARTS = 2048 + 512;          // of waves, and of own and shared ranges, at most
template <typename T, int DP>
__global__ void __launch_bounds__(256) paged_join_kernel(AttnArgs a) {
    constexpr int LANES = DP / 4, AT_ONCE = 256 / LANES;
    __shared__ f32x4_t sums[256];
    __shared__ float weights[JOIN_PARTS];
    const PagedView &pv = a.pv;
    const int t = threadIdx.x, lane = t & 63, d = pv.d;
    const int s = a.decode ? blockIdx.x / pv.max_rows : paged_seq_of_row(pv, blockIdx.x);
    if (s >= pv.n_seq) return;
    const PagedSeq sq = paged_seq(pv, s);
    const int i0 = a.decode ? blockIdx.x % pv.max_rows : blockIdx.x - sq.r0, row = sq.r0 + i0;
    if (i0 < 0 || i0 >= sq.rows) return;
    int w0 = 0, first = 0, shared = 0;                       // parts of ml from `first` on; those of waves w0 .. w0 + shared - 1
    if (a.waves) {
        w0 = a.seq_waves[s].x;
        shared = a.seq_waves[s].y;
        if (shared == 1) {                                   // one wave had it all
            if (a.parts == 1) return;
            shared = 0;
        } else first = 1;
    }
    const int n = a.parts - first, total = n + shared, dim = (t % LANES) * 4;
    const size_t step = (size_t)pv.n_rows * a.n_heads;
    // (the wave that begins a sequence holds it as its last, the others as their first)
    auto wave_slot = [&](int h, int z) { return (((size_t)(w0 + z) * pv.n_kv + h / a.group) * 2 + (z == 0 ? 1 : 0)) * a.packed + i0 * a.group + h % a.group; };
    auto ml_at = [&](int h, int z) { return z < n ? a.ml[(z + first) * step + (size_t)row * a.n_heads + h] : a.wave_ml[wave_slot(h, z - n)]; };
    auto sums_at = [&](int h, int z) { return *(const f32x4_t *)((z < n ? a.o_part + ((z + first) * step + (size_t)row * a.n_heads + h) * d : a.wave_o + wave_slot(h, z - n) * d) + dim); };
    if (total <= FEW) {                                      // every DP / 4 lanes a head of their own, whose parts they read themselves
        for (int h = blockIdx.y * AT_ONCE + t / LANES; h < a.n_heads; h += gridDim.y * AT_ONCE) {
            float2 ml[FEW];
            f32x4_t v[FEW], o = {0.f, 0.f, 0.f, 0.f};
            float top = -INFINITY, sum = 0.f;
#pragma unroll
            for (int z = 0; z < FEW; z++) {
                ml[z] = z < total ? ml_at(h, z) : make_float2(-INFINITY, 0.f);
                if (z < total && dim < d) v[z] = sums_at(h, z);
                top = fmaxf(top, ml[z].x);
            }
#pragma unroll
            for (int z = 0; z < FEW; z++) {
                const float f = ml[z].y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml[z].x - top);
                sum += f * ml[z].y;
#pragma unroll
                for (int e = 0; e < 4; e++) o[e] += ml[z].y == 0.f ? 0.f : f * v[z][e];          // (an empty part has no sums, whatever lies there)
            }
            if (dim >= d) continue;
            const float f = sum == 0.f ? 0.f : 1.f / sum;
            T *dst = (T *)a.out + row * a.o_stride + (size_t)h * d + dim;
#pragma unroll
            for (int e = 0; e < 4; e++) dst[e] = (T)(o[e] * f);
            if (a.lse && dim == 0) a.lse[(size_t)row * a.n_heads + h] = lse_of(a, top, sum);
        }
        return;
    }
    for (int h = blockIdx.y; h < a.n_heads; h += gridDim.y) {
        const size_t at = (size_t)row * a.n_heads + h;
        auto ml_of = [&](int z) { return ml_at(h, z); };
        float top = -INFINITY, sum = 0.f;
        for (int z = lane; z < total; z += 64) top = fmaxf(top, ml_of(z).x);
        top = vla_wave_fold(top, VlaMax());
        __syncthreads();
        for (int z = lane; z < total; z += 64) {
            const float2 v = ml_of(z);
            const float f = v.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(v.x - top);
            sum += f * v.y;
            if (t < 64) weights[z] = v.y == 0.f ? EMPTY : f;
        }
        sum = vla_wave_sum(sum);
        __syncthreads();
        f32x4_t o = {0.f, 0.f, 0.f, 0.f};
        if (dim < d)
#pragma unroll 8
            for (int z = t / LANES; z < total; z += AT_ONCE) {
                const float f = weights[z];
                const f32x4_t v = sums_at(h, z);
#pragma unroll
                for (int e = 0; e < 4; e++) o[e] += f == EMPTY ? 0.f : f * v[e];
            }
        sums[t] = o;
        __syncthreads();
        if (t < LANES && dim < d) {
            for (int i = 1; i < AT_ONCE; i++) {
                const f32x4_t v = sums[i * LANES + t];
#pragma unroll
                for (int e = 0; e < 4; e++) o[e] += v[e];
            }
            const float f = sum == 0.f ? 0.f : 1.f / sum;
            T *dst = (T *)a.out + row * a.o_stride + (size_t)h * d + dim;
#pragma unroll
            for (int e = 0; e < 4; e++) dst[e] = (T)(o[e] * f);
            if (a.lse && t == 0) a.lse[at] = lse_of(a, top, sum);
        }
    }
}

}  // namespace
