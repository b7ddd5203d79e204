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
// sums stay below 2^8 times the count and most tiles rescale nothing.  Of a decode form's weights the product with a bf16 V takes a bf16 head and a
// bf16 tail (2^-16 of the weight is lost, as in attn_mfma.hip): the step waits for memory, and is 1 % longer (behind a shared prefix 8 %).  A prompt's are rounded to
// bf16 once (2^-8 of each, as the tolerances count it), for the third product would take 8192 rows from 550 to 745 us: outputs are off by 1.4 times what their own rounding
// costs (rms 0.0023 of them for 0.0017).  The sum that divides is that of the fp32 weights.
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
    __device__ static void load(unsigned at, const char *pool, const PagedView &pv, int page, int kvh, int key0, const Span &sp, int r0 = 0) {
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
    q.pre = a.prefix_len && valid ? min(paged_int(a.prefix_len, s), sq.keys) : 0;
    q.hi = min(sq.keys, q.p + 1);
    q.lo = a.whole ? 0 : a.shared_len;
    if (a.window) q.lo = max(0, q.p + 1 - a.window);
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
#pragma unroll
        for (int i = 0; i < 16; i++) {
            const int j = j0 + 8 * (i / 4) + i % 4;
            if (!((j < y.hi && j >= y.lo) || j < y.pre)) x[i] = -INFINITY;
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

// Packed rows first .. first + n - 1 of a launch's item -> the lane's query, and the keys any of them may see.
struct Item { int s, kvh, first, lo, hi, g0, g1; PagedSeq sq; };

// The keys that packed rows first .. first + n - 1 of sequence s may see (it->sq is there; false: there are no such rows).
__device__ __forceinline__ bool range_of(const AttnArgs &a, int s, int first, int n, Item *it) {
    it->s = s;
    it->first = first;
    it->g0 = it->g1 = 0;
    const int rows = it->sq.rows;
    if (first >= rows * a.group) return false;
    const int i0 = first / a.group, i1 = min(rows - 1, (first + n - 1) / a.group), p0 = it->sq.len - it->sq.n;
    const int prefix = a.prefix_len ? min(max(paged_int(a.prefix_len, s), 0), it->sq.keys) : 0;
    it->hi = min(it->sq.keys, max(p0 + i1 + 1, prefix));
    const int from = a.window ? max(0, p0 + i0 + 1 - a.window) : 0;          // the first row's window, the lowest
    it->lo = max(a.shared_len, prefix == 0 ? from : 0);
    if (prefix > 0 && a.window) { it->g0 = prefix; it->g1 = max(prefix, min(from, it->hi - 1)); }
    return true;
}

__device__ __forceinline__ bool find_item(const AttnArgs &a, int id, int rows_per_tile, Item *it) {
    const PagedView &pv = a.pv;
    it->kvh = id % pv.n_kv;
    id /= pv.n_kv;
    if (a.whole) {
        it->sq = paged_seq(pv, 0);
        it->s = it->lo = it->g0 = it->g1 = 0;
        it->first = id * rows_per_tile;
        it->hi = a.shared_len;
        return it->first < min(paged_int(pv.row_start, pv.n_seq), pv.n_rows) * a.group;
    }
    const int s = id % pv.n_seq;
    it->sq = paged_seq(pv, s);
    return range_of(a, s, (a.row_tiles - 1 - id / pv.n_seq) * rows_per_tile, rows_per_tile, it);      // the last rows, which see most keys, first
}

// starts: a copy of row_start in LDS, or row_start itself.
template <int MODE>
__device__ __forceinline__ Query find_query(const AttnArgs &a, const Item &it, int r, const int32_t *starts) {
    const int i = r / a.group, hg = r - i * a.group;
    if (!a.whole) return make_query<MODE>(a, it.kvh, it.s, it.sq.r0 + i, i, it.sq, hg, i < it.sq.rows);
    // row i of the batch: its sequence, by halving (row_start ascends)
    int lo = 0, hi = a.pv.n_seq;                              // row_start[lo] <= i < row_start[hi], if i is a row at all
    while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if (starts[mid] <= i) lo = mid; else hi = mid;
    }
    const PagedSeq sq = paged_seq(a.pv, lo);
    const int at = i - sq.r0;
    Query q = make_query<MODE>(a, it.kvh, lo, i, at, sq, hg, at >= 0 && at < sq.rows);
    if (q.valid) { q.hi = min(q.hi, a.shared_len); q.pre = min(q.pre, a.shared_len); }
    return q;
}

__device__ __forceinline__ bool sees_all(const Query &y, int k0, int k1) { return (k1 <= y.hi && k0 >= y.lo) || k1 <= y.pre; }

// Four waves of 32 packed rows each, all walking the same keys, 32 at a time.  K and V move through rings of RING tiles, K one tile before V: while
// tile t's weights are formed on the vector units its successor's scores are on the matrix pipe, instruction by instruction in turn,
// and while its values are summed the successor's largest is found.
// Bound by the matrix pipe and the vector work beside it: 8192 causal rows of 32 heads of 128, 8 key heads: 540-555 us, 1.0 PFLOP/s where a plain matrix
// product reaches 1.39 on this card; heads of 64: 333 us, of 256: 1.32 ms; capped 650; fp32, 2048 rows, heads of 128: 323 us, 107 of 154 TFLOP/s.  (Scores and
// weights one after the other: 637 us; in turn, but every step with its checks: 654.)  A ragged batch of 13 chunks of up to 613 rows: 33 us, a few rounds of
// workgroups, each with its chain of dependent loads.
constexpr int LDS_STARTS = 2048;
template <typename T, int DP> constexpr int RING = 32 * Tile<T, DP>::ROW * 8 <= 64 * 1024 ? 4 : 2;
template <typename T, int DP, int MODE, bool TAILS>
__global__ void __launch_bounds__(256, sizeof(T) * DP <= 256 ? 2 : 1) paged_prompt_kernel(AttnArgs a) {
    typedef Tile<T, DP> TL;
    typedef Rows<T, DP, MODE, TAILS> R;
    constexpr int KT = 32, BYTES = KT * TL::ROW, RG = RING<T, DP>, LOADS = 2 * 8 / TL::RPI;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const unsigned lds0 = (unsigned)(size_t)(lds_void *)lds;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Item it;
    if (!find_item(a, blockIdx.x, 128, &it)) return;
    const int part = a.part0 + blockIdx.y, base = it.lo & ~63, lo = max(it.lo, base + (int)blockIdx.y * a.chunk), hi = min(it.hi, base + ((int)blockIdx.y + 1) * a.chunk);
    const int32_t *table = a.pv.table + (size_t)it.s * a.pv.table_stride;
    const int t0 = lo / KT, t1 = lo < hi ? (hi + KT - 1) / KT : t0;
    const Span sp{lo, hi, it.g0, it.g1};
    // a wave's share of a tile: eight rows of K and of V
    const int g = wave / 2, r0 = wave % 2 * 8;
    const unsigned lds_k = lds0 + wave * 8 * TL::ROW, lds_v = lds_k + RG * BYTES;
    typename TL::template Offsets<false, 8> off_k;
    typename TL::template Offsets<true, 8> off_v;
    off_k.start(a.pv, r0);
    off_v.start(a.pv, r0);
    const Place place(a.pv, it.kvh, sizeof(T));
    const int in0 = (lo + KT - 1) / KT, in1 = it.g0 == it.g1 ? hi / KT : 0;          // tiles that are read whole: [in0, in1)
    auto page_of = [&](int t) { return sp.page(table, a.pv.page_log, t * KT + g * 16); };
    auto load_k = [&](int t, unsigned stage_at, int page) {
        if (t >= in0 && t < in1) off_k.load(lds_k + stage_at, place.in(a.pv, a.pv.k, page, place.at(a.pv, page, t * KT + g * 16)));
        else TL::template load<false, 8>(lds_k + stage_at, a.pv.k, a.pv, page, it.kvh, t * KT + g * 16, sp, r0);
    };
    auto load_v = [&](int t, unsigned stage_at, int page) {
        if (t >= in0 && t < in1) off_v.load(lds_v + stage_at, place.in(a.pv, a.pv.v, page, place.at(a.pv, page, t * KT + g * 16)));
        else TL::template load<true, 8>(lds_v + stage_at, a.pv.v, a.pv, page, it.kvh, t * KT + g * 16, sp, r0);
    };
    // Tile t lies in stage (t - t0) % RG of either ring.  In order: K0 V0 K1 V1 K2 V2 K3 (two stages: K0 V0 K1), then one V and one K a step.
    // The first are on their way before the queries are looked for.
#pragma unroll
    for (int i = 0; i < RG; i++)
        if (t0 + i < t1) {
            const int page = page_of(t0 + i);
            load_k(t0 + i, i * BYTES, page);
            if (i < RG - 1) load_v(t0 + i, i * BYTES, page);
        }
    // (the search of a row's sequence is a chain of loads, one per halving: from LDS, behind the rings)
    const int32_t *starts = a.pv.row_start;
    if (a.whole && a.pv.n_seq <= LDS_STARTS) {
        int32_t *copy = (int32_t *)(lds + 2 * RG * BYTES);
        for (int i = threadIdx.x; i < a.pv.n_seq; i += 256) copy[i] = starts[i];
        __syncthreads();
        starts = copy;
    }
    const Query y = find_query<MODE>(a, it, it.first + wave * 32 + (threadIdx.x & 31), starts);
    R rows;
    rows.start(a, y);
    if (lo < hi) {
        // tiles whose keys all of the wave's queries see: [seen0, seen1) and [in0, pre1)
        const int seen0 = (max(-wave_min(-y.lo), lo) + KT - 1) / KT, seen1 = min(wave_min(y.hi), hi) / KT;
        const int pre1 = max(0, min(wave_min(y.valid ? y.pre : 0x7fffffff), hi)) / KT;
        auto masked = [&](int t) { return !((t >= seen0 && t < seen1) || (t >= in0 && t < pre1)); };
        const float unit = R::unit_of(a);
        int page_v = page_of(t0 + RG - 1), page_k = page_of(t0 + RG);          // (clamped to pages that there are)
        if (t0 + RG - 1 < t1) vm_wait<(RG - 1) * LOADS>();
        else vm_wait<0>();
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        f32x16_t x, next;
        rows.scores(x, lds);
#pragma unroll
        for (int i = 0; i < 16; i++) x[i] = R::shaped(x[i], a, y, t0 * KT, i);
        if (masked(t0)) R::hide(x, y, t0 * KT);
        float top = R::largest(x, unit);
        int t = t0;
        size_t at_v = place.at(a.pv, page_v, (t0 + RG - 1) * KT + g * 16);          // of the 16 keys whose V comes next
        typename R::Weights p;
        // plain steps, from `from` to before `upto`: everything is there to load, whole, and all see all of tile t + 1
        const int from = max(in0, seen0), upto = min(min(in1, t1) - RG - 1, seen1 - 1);
        // The step of tile t, in the stage of that number (a constant: what lies where is known when this is compiled)
        auto step = [&](int stage, f32x16_t &x, f32x16_t &next) __attribute__((always_inline)) {
            const unsigned now = stage * BYTES, after = stage == RG - 1 ? 0 : now + BYTES, before = stage == 0 ? (RG - 1) * BYTES : now - BYTES;
            const bool plain = t >= from && t < upto;
            // K of t + 1 and V of t have landed, and everyone is through with K of t and V of t - 1, whose places are loaded again
            if (t + RG - 1 < t1) vm_wait<(RG - 2) * LOADS>();
            else vm_wait<0>();
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
            if (plain) {
                off_v.load(lds_v + before, place.in(a.pv, a.pv.v, page_v, at_v));
                at_v = place.at(a.pv, page_k, (t + RG) * KT + g * 16);
                off_k.load(lds_k + now, place.in(a.pv, a.pv.k, page_k, at_v));
                page_v = page_k;
                page_k = paged_int(table, ((t + 1 + RG) * KT + g * 16) >> a.pv.page_log);
            } else {
                if (t + RG - 1 < t1) load_v(t + RG - 1, before, page_v);
                if (t + RG < t1) load_k(t + RG, now, page_k);
                at_v = place.at(a.pv, page_k, (t + RG) * KT + g * 16);
                page_v = page_k;
                page_k = page_of(t + 1 + RG);
            }
            rows.move_to(top);
            rows.scores_and_weights(next, lds + after, p, x, unit);
            top = rows.values_and_largest(p, lds + RG * BYTES + now, next, a, y, (t + 1) * KT);
            if (!plain && masked(t + 1)) {                           // (behind the last tile `next` is of no use to anyone)
                R::hide(next, y, (t + 1) * KT);
                top = R::largest(next, unit);
            }
            return ++t < t1;
        };
        for (;;) {
            if (!step(0, x, next) || !step(1, next, x)) break;
            if constexpr (RG == 4)
                if (!step(2, x, next) || !step(3, next, x)) break;
        }
    }
    rows.finish(a, y, part);
}

// Key tiles of 32 of a sequence's rows in decode form, at least one where there are rows (their output has to be written).
__device__ __forceinline__ int tiles_of(const AttnArgs &a, int s) {
    Item it;
    it.sq = paged_seq(a.pv, s);
    if (!range_of(a, s, 0, 32, &it)) return 0;
    return max(1, (it.hi + 31) / 32 - it.lo / 32);
}
// A wave's share of its key head's tiles.  No wave has less than two.  (The plan keeps all sums of tiles below 2^30.)
__device__ __forceinline__ int share_of(const AttnArgs &a, int all) { return max(2, (int)((unsigned)(all + a.waves - 1) / (unsigned)a.waves)); }

// A run of one sequence's tiles of one key head.
struct Run {
    Item it;
    int t0, t1;              // (t0 = t1: its rows see nothing)
    int tiles, took;         // of the sequence; of these, here
    bool first, whole;       // from its first tile on; all of them
};
struct Walk {
    int kvh, s, skip, left;
    __device__ __forceinline__ bool next(const AttnArgs &a, Run *r) {
        while (left > 0 && s < a.pv.n_seq) {
            r->it.sq = paged_seq(a.pv, s);
            r->it.kvh = kvh;
            if (!range_of(a, s++, 0, 32, &r->it)) continue;
            const int t = r->it.lo / 32, n = max(0, (r->it.hi + 31) / 32 - t), all = max(1, n), take = min(all - skip, left);
            r->t0 = t + min(skip, n);
            r->t1 = t + min(skip + take, n);
            r->tiles = all;
            r->took = take;
            r->first = skip == 0;
            r->whole = skip == 0 && take == all;
            left -= take;
            skip = 0;
            return true;
        }
        return false;
    }
};

// One wave a workgroup, as many as their rings fit the chip; each takes one key head's equal run of the key tiles of all sequences, whatever
// their lengths, and streams through it, the next tile on its way whether it is of the same sequence or not.  A sequence's tiles that
// fall to several waves leave parts for the join (a wave has at most two: of the sequence it begins within, and of the one it ends within).
// Neighbouring waves have the same run of different heads, whose rows lie side by side in the pages.
// Memory bound: 32 sequences of 2048 keys, 32 heads, 192 us, 5.6 TB/s; 256 of 294 keys 229 us, 5.4; one of 32768 keys, 8 key heads, 27 us and 6 for
// the join of 128 parts; 48 ragged ones of up to 8192 keys with capped scores and a bias 80 us.  (One workgroup of 1, 2 or 4 waves per sequence,
// key head and even part of max_len: 200, 259, 30 + 5 and 125 to 155 us.)
template <typename T, int DP, int MODE>
__global__ void __launch_bounds__(64) paged_decode_kernel(AttnArgs a) {
    typedef Tile<T, DP> TL;
    constexpr int KT = 32, BYTES = KT * TL::ROW, STAGE = 2 * BYTES, LOADS = 4 * 16 / TL::RPI;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    const unsigned ring0 = (unsigned)(size_t)(lds_void *)lds;
    Walk walk{(int)(blockIdx.x % a.pv.n_kv), 0, 0, 0};
    int share = 0x3fffffff, done = 0;                        // tiles of its share; that it has walked past
    if (a.waves) {
        const int lane = threadIdx.x & 63;
        int all = 0, c = 0;
        for (int s = lane; s < a.pv.n_seq; s += 64) all += c = tiles_of(a, s);
        all = __builtin_amdgcn_readfirstlane(wave_sum(all));
        share = share_of(a, all);
        int rest = blockIdx.x / a.pv.n_kv * share;
        walk.left = min(share, all - rest);
        if (walk.left <= 0) return;
        // the sequence in which it begins
        for (int s0 = 0; s0 < a.pv.n_seq; s0 += 64) {
            if (a.pv.n_seq > 64) c = s0 + lane < a.pv.n_seq ? tiles_of(a, s0 + lane) : 0;
            int in = c;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) { const int v = __shfl_up(in, o, 64); if (lane >= o) in += v; }
            const unsigned long long past = __ballot(in > rest);
            if (past) {
                const int l = __builtin_ctzll(past);
                walk.s = __builtin_amdgcn_readfirstlane(s0 + l);
                walk.skip = __builtin_amdgcn_readfirstlane(rest - __shfl(in - c, l, 64));
                break;
            }
            rest -= __builtin_amdgcn_readlane(in, 63);
        }
    } else {
        walk.s = blockIdx.x / a.pv.n_kv;
        walk.left = tiles_of(a, walk.s);
    }
    Run run, ahead;
    Walk lead = walk;                                        // one tile before what is computed
    bool more = lead.next(a, &ahead);
    int t = 0, p0 = 0, p1 = 0, stage = 0;                    // the lead's next tile and its pages
    Span sp{0, 0, 0, 0};
    auto pages = [&]() {
        const int32_t *table = a.pv.table + (size_t)ahead.it.s * a.pv.table_stride;
        p0 = sp.page(table, a.pv.page_log, t * KT);
        p1 = sp.page(table, a.pv.page_log, t * KT + 16);
    };
    auto settle = [&]() {                                    // on to a tile that there is
        while (more && ahead.t0 == ahead.t1) more = lead.next(a, &ahead);
        if (!more) return;
        t = ahead.t0;
        sp = Span{ahead.it.lo, ahead.it.hi, ahead.it.g0, ahead.it.g1};
        pages();
    };
    typename TL::template Offsets<false, 16> off_k;
    typename TL::template Offsets<true, 16> off_v;
    off_k.start(a.pv, 0);
    off_v.start(a.pv, 0);
    const Place place(a.pv, walk.kvh, sizeof(T));
    auto load = [&](int to) {
        const unsigned at = ring0 + to * STAGE;
        if (t * KT >= sp.lo && (t + 1) * KT <= sp.hi && sp.g0 == sp.g1) {
            const size_t x = place.at(a.pv, p0, t * KT), z = place.at(a.pv, p1, t * KT + 16);
            off_k.load(at, place.in(a.pv, a.pv.k, p0, x));
            off_k.load(at + 16 * TL::ROW, place.in(a.pv, a.pv.k, p1, z));
            off_v.load(at + BYTES, place.in(a.pv, a.pv.v, p0, x));
            off_v.load(at + BYTES + 16 * TL::ROW, place.in(a.pv, a.pv.v, p1, z));
        } else {
            TL::template load<false, 16>(at, a.pv.k, a.pv, p0, ahead.it.kvh, t * KT, sp);
            TL::template load<false, 16>(at + 16 * TL::ROW, a.pv.k, a.pv, p1, ahead.it.kvh, t * KT + 16, sp);
            TL::template load<true, 16>(at + BYTES, a.pv.v, a.pv, p0, ahead.it.kvh, t * KT, sp);
            TL::template load<true, 16>(at + BYTES + 16 * TL::ROW, a.pv.v, a.pv, p1, ahead.it.kvh, t * KT + 16, sp);
        }
        if (++t < ahead.t1) pages();
        else { more = lead.next(a, &ahead); settle(); }
    };
    settle();
    if (more) load(0);
    Rows<T, DP, MODE, sizeof(T) == 2> rows;
    while (walk.next(a, &run)) {
        const int packed = threadIdx.x & 31;
        if (a.waves) {
            // for the join: the waves that have this sequence, told by the one that begins it
            if (run.first && run.it.kvh == 0 && threadIdx.x == 0) a.seq_waves[run.it.s] = make_int2(blockIdx.x / a.pv.n_kv, (int)((unsigned)(done + run.tiles - 1) / (unsigned)share) + 1);
            done += run.took;
        }
        const Query y = find_query<MODE>(a, run.it, packed, a.pv.row_start);
        rows.start(a, y);
        for (int u = run.t0; u < run.t1; u++, stage ^= 1) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // the reads of the stage that is loaded again are through
            if (more) { load(stage ^ 1); vm_wait<LOADS>(); }
            else vm_wait<0>();
            const int k0 = u * KT;
            const char *kt = lds + stage * STAGE;
            rows.tile(a, y, kt, kt + BYTES, k0, !__all(sees_all(y, k0, k0 + KT) && k0 + KT <= run.it.hi && k0 >= run.it.lo));
        }
        if (run.whole) rows.finish(a, y, 0);
        else {
            const size_t slot = ((size_t)blockIdx.x * 2 + (run.first ? 1 : 0)) * a.packed + packed;
            const float sum = vla_fold_step<32>(rows.l, VlaAdd());
            if (y.valid) rows.keep(a, a.wave_ml + slot, a.wave_o + slot * a.pv.d, sum, (threadIdx.x >> 5) & 1);
        }
    }
}

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

// The launches of a call: the new rows against what is their sequence's alone, in prompt or in decode form, and against the shared prefix.
struct Prompt { int row_tiles, parts, chunk; long items; };
struct Plan {
    bool decode;
    int waves;               // decode: among which a key head's tiles are divided, 0: a wave per sequence and key head
    Prompt own, whole;       // own: unless decode
    int parts;               // in ml and o_part
};

int padded_dim(int d) { return d <= 64 ? 64 : d <= 128 ? 128 : 256; }

// Tiles of 128 packed rows, their keys in parts by an estimate in cycles: rounds of workgroups, each a fixed time (its dependent loads, the first
// tile, the writing out: 8 us) and its keys at the matrix and vector work of a tile; and the parts' sums, written and read again, and the launch
// that joins them (with a shared prefix there is one anyway).
Prompt plan_prompt(const AttnArgs &a, bool f32, bool whole) {
    Prompt p{};
    const int row = padded_dim(a.pv.d) * (f32 ? 4 : 2);
    const long packed = (long)(whole ? a.pv.n_rows : a.pv.max_rows) * a.group;
    // the longest range of keys of one tile of rows; it starts at a multiple of 64 unless a window or a short shared prefix moves it
    long keys = whole ? a.shared_len : a.pv.max_len - a.shared_len;
    if (a.window && !a.prefix_len && keys > (long)a.window + 128) keys = a.window + 128;
    if (!whole && (a.window || a.shared_len % 64)) keys += 63;
    p.row_tiles = (int)((packed + 127) / 128);
    p.items = (long)p.row_tiles * (whole ? 1 : a.pv.n_seq) * a.pv.n_kv;
    p.parts = 1;
    p.chunk = 64;
    const double pairs = (double)a.pv.n_rows * a.n_heads;
    const int per_cu = row <= 256 ? 2 : 1;
    double best = 0.0;
    for (long parts = 1; parts <= 256; parts++) {
        const long chunk = keys > 0 ? (((keys + parts - 1) / parts) + 63) / 64 * 64 : 64, n = keys > 0 ? (keys + chunk - 1) / chunk : 1;
        if (n < parts) continue;
        const double rounds = (double)((p.items * n + 256 * per_cu - 1) / (256 * per_cu));
        const double cost = rounds * (20e3 + chunk * 33.0 * per_cu * row / 256) + (n > 1 ? n * pairs * a.pv.d * 8.0 / 2000.0 + (whole ? 0.0 : 12e3) : 0.0);
        if (best == 0.0 || cost < best) { best = cost; p.chunk = (int)chunk; p.parts = (int)n; }
    }
    return p;
}
Plan plan(const AttnArgs &a, bool f32) {
    Plan p{};
    // Decode form: up to 32 packed rows a sequence (a matrix instruction's columns).  (Every wave looks at all sequences' lengths: not for many thousands.)
    p.decode = (long)a.pv.max_rows * a.group <= 32 && a.pv.n_seq <= 2048 && (long)a.pv.n_seq * (a.pv.max_len / 32 + 2) < 1L << 30;
    if (p.decode) {
        // as many waves as their rings, 128 rows of K or V each, fit the CUs' LDS (handed out in units of 1280 bytes: four of 32 KB)
        const int fit = 128 / ((128 * padded_dim(a.pv.d) * (f32 ? 4 : 2) + 1279) / 1280);
        const int all = 256 * (fit > 8 ? 8 : fit), waves = all / a.pv.n_kv;
        // Not divided, a wave per sequence and key head, which saves the search for a share and most of the join: where these are enough to fill the chip and
        // the longest is no long tail behind the others.  1024 waves, 32 key heads: 256 sequences of 294 keys 226 us (divided 248), of 1024 744 (801), ragged up to
        // 1024 399 (430); 16 of up to 512 26 both ways; but 16 ragged ones of up to 1024 42 (36), 64 of up to 2048 235 (222).
        const long pairs = (long)a.pv.n_seq * a.pv.n_kv, longest = a.pv.max_len - a.shared_len;
        const bool divided = longest > (pairs >= 4 * all ? 1024 : 2 * pairs >= all ? 512 : 128);
        p.waves = divided ? (waves > 0 ? waves : 1) : 0;
        p.parts = 1;
    } else {
        p.own = plan_prompt(a, f32, false);
        p.parts = p.own.parts;
    }
    if (a.shared_len > 0) {
        p.whole = plan_prompt(a, f32, true);
        p.parts += p.whole.parts;
    }
    return p;
}
int check_plan(const Plan &p) {
    const long most = p.own.items > p.whole.items ? p.own.items : p.whole.items;
    if (most > 0x7fffffffL / 256) { vla_set_error("paged_attention: %ld tiles of rows are too many: split the batch", most); return VLA_ESHAPE; }
    return VLA_OK;
}
size_t round_up(size_t v) { return (v + 255) / 256 * 256; }
// Lays the workspace out from `base` (NULL: only its size).
size_t lay_out(AttnArgs *a, const Plan &p, char *base) {
    size_t off = 0;
    auto take = [&](size_t bytes) { char *at = base + off; off += round_up(bytes); return at; };
    a->parts = p.parts;
    a->waves = p.waves;
    a->decode = p.decode;
    a->packed = a->pv.max_rows * a->group;
    if (p.parts > 1) {
        const size_t slots = (size_t)a->pv.n_rows * a->n_heads * p.parts;
        a->ml = (float2 *)take(slots * sizeof(float2));
        a->o_part = (float *)take(slots * a->pv.d * sizeof(float));
    }
    if (p.waves) {
        const size_t slots = (size_t)p.waves * a->pv.n_kv * 2 * a->packed;
        a->seq_waves = (int2 *)take(a->pv.n_seq * sizeof(int2));
        a->wave_ml = (float2 *)take(slots * sizeof(float2));
        a->wave_o = (float *)take(slots * a->pv.d * sizeof(float));
    }
    return off ? off : 256;
}

template <typename T, int DP, int MODE, bool TAILS>
int launch_prompt(AttnArgs a, const Prompt &p, bool whole, int part0, hipStream_t st) {
    const size_t bytes = 2 * RING<T, DP> * 32 * Tile<T, DP>::ROW + (whole && a.pv.n_seq <= LDS_STARTS ? a.pv.n_seq * sizeof(int32_t) : 0);
    if (int rc = vla_allow_lds((const void *)paged_prompt_kernel<T, DP, MODE, TAILS>, 2 * RING<T, DP> * 32 * Tile<T, DP>::ROW + LDS_STARTS * sizeof(int32_t))) return rc;
    a.whole = whole; a.row_tiles = p.row_tiles; a.chunk = p.chunk; a.part0 = part0;
    paged_prompt_kernel<T, DP, MODE, TAILS><<<dim3((unsigned)p.items, p.parts), 256, bytes, st>>>(a);
    return vla_check_launch("paged_attention");
}
template <typename T, int DP, int MODE>
int launch(const AttnArgs &a, const Plan &p, hipStream_t st) {
    int rc;
    constexpr bool BF16 = sizeof(T) == 2;
    if (a.shared_len > 0 && (rc = p.decode ? launch_prompt<T, DP, MODE, BF16>(a, p.whole, true, 1, st) : launch_prompt<T, DP, MODE, false>(a, p.whole, true, p.own.parts, st))) return rc;
    if (p.decode) {
        constexpr size_t bytes = 2 * 2 * 32 * Tile<T, DP>::ROW;
        if ((rc = vla_allow_lds((const void *)paged_decode_kernel<T, DP, MODE>, bytes))) return rc;
        paged_decode_kernel<T, DP, MODE><<<(p.waves ? p.waves : a.pv.n_seq) * a.pv.n_kv, 64, bytes, st>>>(a);
        rc = vla_check_launch("paged_attention");
    } else rc = launch_prompt<T, DP, MODE, false>(a, p.own, false, 0, st);
    if (rc || (p.parts == 1 && !p.waves)) return rc;
    const int rows = p.decode ? a.pv.n_seq * a.pv.max_rows : a.pv.n_rows;
    const int heads = (2048 + rows - 1) / rows;              // of a row, that get a workgroup of their own
    paged_join_kernel<T, DP><<<dim3(rows, heads < a.n_heads ? heads : a.n_heads), 256, 0, st>>>(a);
    return vla_check_launch("paged_attention join");
}
template <typename T, int MODE>
int launch_sized(const AttnArgs &a, const Plan &p, hipStream_t st) {
    switch (padded_dim(a.pv.d)) {
        case 64: return launch<T, 64, MODE>(a, p, st);
        case 128: return launch<T, 128, MODE>(a, p, st);
        default: return launch<T, 256, MODE>(a, p, st);
    }
}
template <typename T>
int launch_typed(const AttnArgs &a, const Plan &p, hipStream_t st) {
    switch ((a.cap > 0.f ? CAPPED : 0) | (a.slopes ? BIASED : 0)) {
        case 0: return launch_sized<T, 0>(a, p, st);
        case CAPPED: return launch_sized<T, CAPPED>(a, p, st);
        case BIASED: return launch_sized<T, BIASED>(a, p, st);
        default: return launch_sized<T, CAPPED | BIASED>(a, p, st);
    }
}

}  // namespace

extern "C" {

size_t vla_paged_attention_workspace_bytes(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_paged_mask *mask, int n_heads) {
    AttnArgs a{};
    if (check(cache, batch, mask, n_heads, &a)) return 0;
    const Plan p = plan(a, cache->dtype == VLA_DTYPE_F32);
    return check_plan(p) ? 0 : lay_out(&a, p, nullptr);
}

int vla_paged_attention(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_paged_mask *mask, const void *q, int n_heads,
                        int64_t q_stride, void *out, int64_t out_stride, float *lse, void *ws, size_t ws_bytes, void *stream) {
    AttnArgs a{};
    if (int rc = check(cache, batch, mask, n_heads, &a)) return rc;
    if (batch->n_rows > 0 && (!q || !out || !ws)) { vla_set_error("paged_attention: q, out or ws is NULL"); return VLA_EINVAL; }
    if ((uintptr_t)ws % 16) { vla_set_error("paged_attention: ws is not 16-byte aligned"); return VLA_EINVAL; }
    if (q_stride < (int64_t)n_heads * cache->head_dim || out_stride < (int64_t)n_heads * cache->head_dim) {
        vla_set_error("paged_attention: a row stride is shorter than its heads");
        return VLA_ESHAPE;
    }
    const bool f32 = cache->dtype == VLA_DTYPE_F32;
    const Plan p = plan(a, f32);
    if (int rc = check_plan(p)) return rc;
    const size_t need = lay_out(&a, p, (char *)ws);
    if (batch->n_rows > 0 && ws_bytes < need) { vla_set_error("paged_attention: workspace %zu bytes, need %zu", ws_bytes, need); return VLA_EWORKSPACE; }
    if (batch->n_rows == 0 || batch->max_rows == 0) return VLA_OK;
    const size_t es = f32 ? 4 : 2;
    a.q = (const char *)q; a.out = (char *)out; a.lse = lse; a.q_stride = q_stride; a.o_stride = out_stride;
    a.aligned = ((uintptr_t)q | (uintptr_t)out | (size_t)q_stride * es | (size_t)out_stride * es) % 16 == 0;
    a.offset = !f32 ? a.cap * 1.4426950408889634f : 0.f;
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps("paged_attention", 0.0, st);               // (how much there is to do stands in arrays of the device)
    return f32 ? launch_typed<float>(a, p, st) : launch_typed<bf16_t>(a, p, st);
}

}  // extern "C"
