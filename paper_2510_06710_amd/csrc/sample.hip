// Sampling from rows of logits with temperature, top-k, top-p and min-p, from given random numbers.
//
// A token's place in the order "largest first, lowest id first among equals" is its rank; 64 bits hold (value, id) so that a
// larger number comes earlier.  Every cut keeps a leading run of that order, so the kept set is one threshold on that
// number.  Masses are w = exp((z - max) / T) in fp64, rounded to multiples of 2^-44 and summed as whole numbers: the sums are exact,
// in any order, and the border cases of top-p and of u fall alike every time (2^18 tokens of mass 1 stay below 2^63).
//
// One workgroup a row.  A row of up to SHORT tokens is sorted whole in LDS; the cuts are then places in a running sum.  Longer rows: with
// top-k, a count over bins of 1/32 in log2 units finds the bin of the k-th token, and the list is all tokens down to that bin.  With top-p
// alone, masses over the same bins find the bin in which the cut falls, and the list is that bin's tokens.  The row is read again from the
// caches for each step: its maximum; the bins; the list and the kept mass of every segment of ids; and the segment in which u falls.
//
// 256 rows of 128,000 fp32 logits, every setting in turn: 112 us (read once at the rate of a large copy: 27).  Of a row with top-p alone 18 us
// are the maximum, at the rate of the memory; 31 the bins and 40 the list and segments, both bound by the issue of the vector ALU, where fp64
// instructions of the masses are most; 14 the sort and the choice.  Small rows are bound by the steps behind each other: 256 of 256 bins 9.5 us; one row of 128,000, on one CU, 63.
#include "vla_internal.h"

namespace {

constexpr double UNIT = 17592186044416.0;      // 2^44
constexpr int LIST = 4096, SHORT = 512, BINS = 2048, SEGMENTS = 512;
typedef unsigned long long u64;

struct SampleArgs {
    const char *logits;
    long stride;
    int n, vocab;
    const float *temperature;
    const int32_t *top_k;
    const float *top_p, *min_p, *u;
    int32_t *token;
    float *logp, *logp_kept;
    int32_t *n_kept;
};

// Values in ascending order as unsigned numbers; those that are never kept (NaN, -inf) are 0.
__device__ __forceinline__ unsigned order_of(float z) {
    if (!(z > -INFINITY)) return 0u;
    const unsigned b = __builtin_bit_cast(unsigned, z == 0.f ? 0.f : z);      // (both zeros are one value)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float value_of(unsigned o) { return __builtin_bit_cast(float, o & 0x80000000u ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ u64 rank_key(unsigned order, int id) { return (u64)order << 32 | (unsigned)~id; }
__device__ __forceinline__ int id_of(u64 key) { return (int)~(unsigned)key; }
__device__ __forceinline__ float value_at(u64 key) { return value_of((unsigned)(key >> 32)); }

// Over the 64 lanes by lane moves of the vector ALU (through LDS a step of a 64-bit value takes some 150 cycles): running sums of rows of 16
// lanes, then of 32 and 64.
template <int CTRL, int ROWS> __device__ __forceinline__ u64 moved(u64 v) {
    const unsigned lo = __builtin_amdgcn_update_dpp(0, (int)(unsigned)v, CTRL, ROWS, 0xf, false), hi = __builtin_amdgcn_update_dpp(0, (int)(unsigned)(v >> 32), CTRL, ROWS, 0xf, false);
    return (u64)hi << 32 | lo;
}
template <typename F> __device__ __forceinline__ u64 wave_run(u64 v, F f) {
    v = f(v, moved<0x111, 0xf>(v));          // row_shr 1, 2, 4, 8
    v = f(v, moved<0x112, 0xf>(v));
    v = f(v, moved<0x114, 0xf>(v));
    v = f(v, moved<0x118, 0xf>(v));
    v = f(v, moved<0x142, 0xa>(v));          // row_bcast 15, 31
    return f(v, moved<0x143, 0xc>(v));
}
__device__ __forceinline__ u64 last_lane(u64 v) {
    return (u64)(unsigned)__builtin_amdgcn_readlane((int)(unsigned)(v >> 32), 63) << 32 | (unsigned)__builtin_amdgcn_readlane((int)(unsigned)v, 63);
}
__device__ __forceinline__ u64 wave_scan(u64 v) { return wave_run(v, [](u64 a, u64 b) { return a + b; }); }
__device__ __forceinline__ u64 wave_sum(u64 v) { return last_lane(wave_scan(v)); }
__device__ __forceinline__ u64 wave_max(u64 v) { return last_lane(wave_run(v, [](u64 a, u64 b) { return a > b ? a : b; })); }

// 2^y for y <= 0, relative error below 1e-14: 2^f by its series in f ln 2 (|f ln 2| <= 0.347), the last term left out 6e-15.
__device__ __forceinline__ double exp2_neg(double y) {
    const double n = __builtin_rint(y), x = (y - n) * 0.69314718055994530942;
    double p = 1.0 / 39916800.0;
    p = __builtin_fma(p, x, 1.0 / 3628800.0);
    p = __builtin_fma(p, x, 1.0 / 362880.0);
    p = __builtin_fma(p, x, 1.0 / 40320.0);
    p = __builtin_fma(p, x, 1.0 / 5040.0);
    p = __builtin_fma(p, x, 1.0 / 720.0);
    p = __builtin_fma(p, x, 1.0 / 120.0);
    p = __builtin_fma(p, x, 1.0 / 24.0);
    p = __builtin_fma(p, x, 1.0 / 6.0);
    p = __builtin_fma(p, x, 0.5);
    p = __builtin_fma(p, x, 1.0);
    p = __builtin_fma(p, x, 1.0);
    return __builtin_ldexp(p, n < -2000.0 ? -2000 : (int)n);
}
// w in [0, 1] to multiples of 2^-44: added to 2^52 its rounded multiple stands in the low bits.
__device__ __forceinline__ u64 units_of(double w) { return __builtin_bit_cast(u64, __builtin_fma(w, UNIT, 4503599627370496.0)) & 0xfffffffffffffull; }

// A row's masses: w = 2^y, y = (z - max) rate.  2^y = 2^e table[j] 2^r with y = e + j / 32 + r, |r| <= 1/64: table[j] = 2^(j/32), and five
// terms of the series of 2^r, the next of which is below 1.3e-12.  Without a table eleven terms (256 rows of 128,000 logits: 75 of 180 us were
// fp64 instructions); 32 entries are one for each pair of LDS banks, so that no lookup waits for another (256 entries and a term less were 121 us with top-p, 107 so).
constexpr int TABLE = 32;
struct Scale {
    double zmax, rate;       // (of table steps: 32 log2 e / T)
    const double *table;
    // Steps below the largest, and the whole number of them.  Added to 1.5 2^52 a number is rounded to a whole one, which stands in the low bits
    // (fp64 conversions and ldexp run at a quarter of the rate).
    struct Steps { double v, n; int k; };
    __device__ __forceinline__ Steps steps(float z) const {
        constexpr double MAGIC = 6755399441055744.0;
        Steps s;
        s.v = fmax(((double)z - zmax) * rate, -32000.0);          // (NaN and -inf too: a weight of 2^-1000)
        const double m = s.v + MAGIC;
        s.k = (int)(unsigned)__builtin_bit_cast(u64, m);
        s.n = m - MAGIC;
        return s;
    }
    __device__ __forceinline__ double weight_of(const Steps &s) const {
        constexpr double C = 0.69314718055994530942 / TABLE, C2 = C * C / 2.0, C3 = C2 * C / 3.0, C4 = C3 * C / 4.0;
        const double r = s.v - s.n;
        const u64 p = __builtin_bit_cast(u64, __builtin_fma(__builtin_fma(__builtin_fma(__builtin_fma(r, C4, C3), r, C2), r, C), r, 1.0) * table[s.k & (TABLE - 1)]);
        return __builtin_bit_cast(double, (u64)((unsigned)(p >> 32) + ((unsigned)(s.k >> 5) << 20)) << 32 | (unsigned)p);      // times 2^(k / 32)
    }
    __device__ __forceinline__ double weight(float z) const { return weight_of(steps(z)); }
    __device__ __forceinline__ u64 units(float z) const { return units_of(weight(z)); }
    // one bin per step, never descending in -z; below 2^-63 all one
    __device__ __forceinline__ int bin_of(const Steps &s) const { return min(-s.k, BINS - 1); }
};
__device__ __forceinline__ void fill_table(double *table) {
    for (int j = threadIdx.x; j < TABLE; j += blockDim.x) table[j] = j == 0 ? 1.0 : 2.0 * exp2_neg((double)j / TABLE - 1.0);
}

struct Both { u64 count, mass; };
template <int THREADS> struct Block {
    u64 red[2][THREADS / 64];
    // Sums (or the maximum of `count`) over the workgroup, to all threads.
    __device__ Both both(Both v, bool largest = false) {
        v.count = largest ? wave_max(v.count) : wave_sum(v.count);
        v.mass = wave_sum(v.mass);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) { red[0][threadIdx.x >> 6] = v.count; red[1][threadIdx.x >> 6] = v.mass; }
        __syncthreads();
        Both r{0, 0};
        for (int i = 0; i < THREADS / 64; i++) {
            r.count = largest ? (red[0][i] > r.count ? red[0][i] : r.count) : r.count + red[0][i];
            r.mass += red[1][i];
        }
        return r;
    }
    // What lies before this thread's value, in thread order.
    __device__ u64 before(u64 v) {
        const u64 in = wave_scan(v);
        __syncthreads();
        if ((threadIdx.x & 63) == 63) red[0][threadIdx.x >> 6] = in;
        __syncthreads();
        u64 b = in - v;
        for (int i = 0; i < (int)(threadIdx.x >> 6); i++) b += red[0][i];
        return b;
    }
};

// LDS of a workgroup.
template <int THREADS> struct Room {
    u64 keys[LIST];              // the list, sorted: largest key first; zeros behind it
    union { u64 mass[BINS]; unsigned count[BINS]; u64 bucket[BINS]; };
    u64 segment[SEGMENTS];
    double table[TABLE];
    Block<THREADS> block;
    int n;                       // tokens that asked for a place in the list
    int found;
    u64 found_before;
};

// keys[0 .. P), P a power of two, from the largest to the smallest.  Pairs of a distance up to 64 lie in the 128 keys of one wave's
// threads, whose LDS accesses take place in order: only longer distances need the workgroup's barrier.
// Up to 256 keys: each thread counts how many are larger than its own (a microsecond; in steps three).
template <int THREADS> __device__ void sort_keys(u64 *keys, int P) {
    const int t = threadIdx.x;
    __syncthreads();
    if (P <= 256) {
        typedef u64 u64x2 __attribute__((ext_vector_type(2)));
        u64 mine = 0;
        int place = 0;
        if (t < P) {
            mine = keys[t];
            if (!mine) keys[t] = P - t;                      // (below every key, and no two alike)
        }
        __syncthreads();
        if (t < P) {
            const u64 key = keys[t];
#pragma unroll 8
            for (int i = 0; i < P; i += 2) {
                const u64x2 k = *(const u64x2 *)(keys + i);
                place += (k[0] > key) + (k[1] > key);
            }
        }
        __syncthreads();
        if (t < P) keys[place] = mine;
        __syncthreads();
        return;
    }
    for (int k = 2; k <= P; k <<= 1)
        for (int j = k >> 1; j > 0; j >>= 1) {
            if (j >= 128 && j == k >> 1) __syncthreads();
            for (int q = threadIdx.x; q < P / 2; q += THREADS) {
                const int i = ((q & ~(j - 1)) << 1) | (q & (j - 1));
                const u64 x = keys[i], y = keys[i + j];
                if (((i & k) == 0) == (x < y)) { keys[i] = y; keys[i + j] = x; }
            }
            if (j >= 128) __syncthreads();
            else asm volatile("" ::: "memory");
        }
    __syncthreads();
}

// A segment's tokens, SEGMENT ids, in the registers of a wave: 16 bytes a load.
template <int SEGMENT, typename T> struct Segment {
    static constexpr int W = SEGMENT / 64 < 16 / (int)sizeof(T) ? SEGMENT / 64 : 16 / (int)sizeof(T), STEPS = SEGMENT / (64 * W);
    typedef T tw __attribute__((ext_vector_type(W), aligned(sizeof(T))));
    typedef const __attribute__((address_space(1))) tw *global;          // (not a flat load, which waits with LDS)
    typedef const __attribute__((address_space(1))) T *global_one;
    tw v[STEPS];
    __device__ __forceinline__ void load(const T *z, int V, int segment) {
        const int i0 = segment * SEGMENT + (threadIdx.x & 63) * W;
        if (segment * SEGMENT + SEGMENT <= V) {
#pragma unroll
            for (int s = 0; s < STEPS; s++) v[s] = *(global)(z + i0 + s * 64 * W);
        } else
#pragma unroll
            for (int s = 0; s < STEPS; s++)
#pragma unroll
                for (int e = 0; e < W; e++) v[s][e] = i0 + s * 64 * W + e < V ? ((global_one)z)[i0 + s * 64 * W + e] : (T)-INFINITY;
    }
    // f(value, number) of the lane's tokens; id_at: a number's id
    template <typename F> __device__ __forceinline__ void each(F f) const {
#pragma unroll
        for (int s = 0; s < STEPS; s++)
#pragma unroll
            for (int e = 0; e < W; e++) f((float)v[s][e], s * W + e);
    }
    __device__ static int id_at(int segment, int n) { return segment * SEGMENT + (threadIdx.x & 63) * W + n / W * 64 * W + n % W; }
};
// All tokens of the row (and -inf for ids behind it) to f(value, number, segment), a wave's segment after segment, the next one on its way meanwhile; end(segment) behind each.
template <int THREADS, int SEGMENT, typename T, typename F, typename E> __device__ __forceinline__ void each_token(const T *z, int V, F f, E end) {
    constexpr int WAVES = THREADS / 64;
    const int n = (V + SEGMENT - 1) / SEGMENT;
    int s = threadIdx.x >> 6;
    if (s >= n) return;
    Segment<SEGMENT, T> a, b;
    a.load(z, V, s);
    for (;;) {
        if (s + WAVES < n) b.load(z, V, s + WAVES);
        a.each([&](float v, int n) { f(v, n, s); });
        end(s);
        if ((s += WAVES) >= n) return;
        if (s + WAVES < n) a.load(z, V, s + WAVES);
        b.each([&](float v, int n) { f(v, n, s); });
        end(s);
        if ((s += WAVES) >= n) return;
    }
}
template <int THREADS, int SEGMENT, typename T, typename F> __device__ __forceinline__ void each_token(const T *z, int V, F f) {
    each_token<THREADS, SEGMENT>(z, V, f, [](int) {});
}

// Whether a token of mass w, with `run` before it in id order, is the one: the first whose sum exceeds `want`; the last with mass
// should none (u that is no number below 1).
__device__ __forceinline__ bool falls_in(u64 run, u64 w, double want, u64 total) {
    const bool over = (double)(run + w) > want;
    return w && (over ? run == 0 || !((double)run > want) : run + w == total);
}

// What the other ways decline (infinite logits; more than LIST tokens in one bin of a cut, as where logits are flat or few values): each cut by the 50 bits of
// the order, ten a pass over the row: the counts or masses of the tokens that agree in the higher digits, by the next one.  (256 rows of 128,000 logits
// N(0, 0.05) with top-p: 1.0 ms; a bit a pass was some fifty such passes a cut.)
template <int THREADS, typename T> __device__ void sample_by_digits(const SampleArgs &a, const T *z, int row, u64 first, Room<THREADS> &room) {
    const int t = threadIdx.x, V = a.vocab;
    Block<THREADS> &block = room.block;
    u64 *scan = room.mass;
    const float zmax = value_at(first);
    const float T0 = a.temperature ? a.temperature[row] : 1.f;
    const bool infinite = zmax == INFINITY;
    const bool greedy = !(T0 > 0.f) || !a.u;
    const Scale sc{infinite ? 0.0 : (double)zmax, 1.4426950408889634074 * TABLE / (T0 > 0.f ? (double)T0 : 1.0), room.table};
    auto weight = [&](float v) { return infinite ? (v == INFINITY ? 1.0 : 0.0) : sc.weight(v); };
    auto units = [&](float v) { return units_of(weight(v)); };
    // count and mass of what lies at or above a threshold
    auto above = [&](u64 least) {
        Both b{0, 0};
        for (int i = t; i < V; i += THREADS) {
            const float v = (float)z[i];
            const unsigned o = order_of(v);
            if (o && rank_key(o, i) >= least) { b.count++; b.mass += units(v); }
        }
        return block.both(b);
    };
    // The largest threshold at or above which there is enough (there is in all), at most the largest key: 32 bits of order, 18 of id.
    auto threshold = [&](bool masses, auto enough) {
        constexpr int DIGITS = 1024, RUN = DIGITS / THREADS;
        u64 c = 0, over = 0;                          // the digits so far; what lies above all keys that have them
        for (int shift = 40; shift >= 0; shift -= 10) {
            __syncthreads();
            for (int i = t; i < DIGITS; i += THREADS) room.mass[i] = 0;
            __syncthreads();
            for (int i = t; i < V; i += THREADS) {
                const float v = (float)z[i];
                const unsigned o = order_of(v);
                const u64 key = (u64)o << 18 | (~i & 0x3ffff);
                if (o && key >> (shift + 10) == c) atomicAdd(&room.mass[(key >> shift) & (DIGITS - 1)], masses ? units(v) : 1ull);
            }
            if (t == 0) { room.found = enough(over) ? DIGITS - 1 : 0; room.found_before = over; }
            __syncthreads();
            u64 mine[RUN], sum = 0;                   // from the highest digit down
#pragma unroll
            for (int e = 0; e < RUN; e++) sum += mine[e] = room.mass[DIGITS - 1 - (t * RUN + e)];
            u64 run = over + block.before(sum);
#pragma unroll
            for (int e = 0; e < RUN; e++) {
                if (enough(run + mine[e]) && !enough(run)) { room.found = DIGITS - 1 - (t * RUN + e); room.found_before = run; }
                run += mine[e];
            }
            __syncthreads();
            c = c << 10 | (unsigned)room.found;
            over = room.found_before;
        }
        const u64 key = (c >> 18) << 32 | 0xfffc0000u | (c & 0x3ffff);
        return key < first ? key : first;
    };
    const Both all = above(1);
    u64 cut = 1, leading = all.mass;
    if (infinite) cut = (u64)order_of(INFINITY) << 32;
    const int k = a.top_k ? a.top_k[row] : 0;
    if (k > 0 && (u64)k < all.count) {
        const u64 c = threshold(false, [&](u64 count) { return count >= (u64)k; });
        cut = c > cut ? c : cut;
        leading = above(cut).mass;
    }
    const float p = a.top_p ? a.top_p[row] : 1.f;
    if (p < 1.f) {
        const double want = (double)(p > 0.f ? p : 0.f) * (double)leading;
        const u64 c = threshold(true, [&](u64 mass) { return (double)mass >= want; });
        cut = c > cut ? c : cut;
    }
    const float least = fminf(a.min_p ? a.min_p[row] : 0.f, 1.f);
    auto kept = [&](float v, int i) {
        const unsigned o = order_of(v);
        if (!o) return false;
        const u64 key = rank_key(o, i);
        return key >= cut && weight(v) >= (double)least;
    };
    // ids in runs of consecutive ones per thread: running masses in id order
    const int per = (V + THREADS - 1) / THREADS, i0 = t * per, i1 = min(V, i0 + per);
    Both mine{0, 0};
    for (int i = i0; i < i1; i++) {
        const float v = (float)z[i];
        if (kept(v, i)) { mine.count++; mine.mass += units(v); }
    }
    const Both total = block.both(mine);
    scan[t] = mine.mass;
    __syncthreads();
    if (t == 0) {
        u64 run = 0;
        for (int i = 0; i < THREADS; i++) { const u64 x = scan[i]; scan[i] = run; run += x; }
    }
    __syncthreads();
    int token = id_of(first);
    if (!greedy) {
        const float u = a.u[row];
        const double want = (double)u * (double)total.mass;
        Both pick{0, 0};
        u64 run = scan[t];
        for (int i = i0; i < i1; i++) {
            const float v = (float)z[i];
            if (!kept(v, i)) continue;
            const u64 w = units(v);
            if (falls_in(run, w, want, total.mass)) pick.count = (unsigned)i + 1ull;
            run += w;
        }
        token = (int)block.both(pick, true).count - 1;
    }
    if (t == 0) {
        const float v = (float)z[token];
        const double y = infinite ? 0.0 : ((double)v - sc.zmax) * sc.rate * (0.69314718055994530942 / TABLE);
        a.token[row] = token;
        if (a.logp) a.logp[row] = (float)(y - log((double)all.mass / UNIT));
        if (a.logp_kept) a.logp_kept[row] = (float)(y - log((double)total.mass / UNIT));
        if (a.n_kept) a.n_kept[row] = (int)total.count;
    }
}


// WHOLE: the row itself is the list.
template <int THREADS, int SEGMENT, bool WHOLE, typename T> __global__ void __launch_bounds__(THREADS) sample_rows_kernel(SampleArgs a) {
    __shared__ Room<THREADS> room;
    Block<THREADS> &block = room.block;
    const int row = blockIdx.x, t = threadIdx.x, V = a.vocab;
    const T *z = (const T *)a.logits + row * a.stride;
    typedef Segment<SEGMENT, T> Seg;
    // (asked for together with the row: each alone is a memory latency)
    const float T0 = a.temperature ? a.temperature[row] : 1.f, p = a.top_p ? a.top_p[row] : 1.f, least = fminf(a.min_p ? a.min_p[row] : 0.f, 1.f), u = a.u ? a.u[row] : 0.f;
    int k = a.top_k ? a.top_k[row] : 0;
    fill_table(room.table);                // (there for all once the largest is known)
    // ---- the largest, and how many there are
    Both top{0, 0};
    int P = 2;                             // places of the list, a power of two
    if constexpr (WHOLE) {
        while (P < V) P <<= 1;
        for (int i = t; i < P; i += THREADS) {
            const unsigned o = i < V ? order_of((float)z[i]) : 0u;
            const u64 key = o ? rank_key(o, i) : 0;
            room.keys[i] = key;
            top.count = key > top.count ? key : top.count;
            top.mass += o != 0;
        }
    } else {
        float best = -INFINITY;
        int at = 0, in = 0, is = 0;
        each_token<THREADS, SEGMENT>(z, V, [&](float v, int n, int s) {
            if (v > best) { best = v; at = n; in = s; }      // (a lane's ids ascend: the lowest of equals stays)
            is += v > -INFINITY;
        });
        const unsigned o = order_of(best);
        top.count = o ? rank_key(o, Seg::id_at(in, at)) : 0;
        top.mass = is;
    }
    top = block.both(top, true);
    const u64 first = top.count;
    const int valid = (int)top.mass;
    if (first == 0) {
        if (t == 0) {
            a.token[row] = -1;
            if (a.logp) a.logp[row] = -INFINITY;
            if (a.logp_kept) a.logp_kept[row] = -INFINITY;
            if (a.n_kept) a.n_kept[row] = 0;
        }
        return;
    }
    const float zmax = value_at(first);
    if (zmax == INFINITY) { sample_by_digits<THREADS>(a, z, row, first, room); return; }
    const bool greedy = !(T0 > 0.f) || !a.u;
    const Scale sc{(double)zmax, 1.4426950408889634074 * TABLE / (T0 > 0.f ? (double)T0 : 1.0), room.table};
    if (k <= 0 || k >= valid) k = valid;
    const bool cut_k = k < valid, cut_p = p < 1.f;
    const double share = p > 0.f ? (double)p : 0.0;
    const bool ranked = WHOLE || cut_k;    // the list holds all leading tokens (else: those of the bin in which the cut of top-p falls)

    u64 all_mass = 0, kept_mass = 0, above = 0;      // of the row; of the kept tokens; of the bins before the border
    int n_kept = 0, border = BINS;
    double limit = 0.0;                              // mass before a token at which top-p ends
    if constexpr (!WHOLE) {
        // ---- bins: where the cut falls
        if (cut_k || cut_p) {
            for (int i = t; i < BINS; i += THREADS) room.mass[i] = 0;
            __syncthreads();
            if (cut_k) {
                u64 all = 0;                         // (of the row, for logp: the same whole numbers whatever the cuts are)
                each_token<THREADS, SEGMENT>(z, V, [&](float v, int, int) {
                    const auto y = sc.steps(v);
                    all += units_of(sc.weight_of(y));
                    atomicAdd(&room.count[sc.bin_of(y)], v > -INFINITY ? 1u : 0u);
                });
                all_mass = block.both(Both{0, all}).mass;
            } else
                each_token<THREADS, SEGMENT>(z, V, [&](float v, int, int) {
                    const auto y = sc.steps(v);
                    atomicAdd(&room.mass[sc.bin_of(y)], units_of(sc.weight_of(y)));
                });
            __syncthreads();
            constexpr int RUN = BINS / THREADS;
            u64 mine[RUN], sum = 0;
#pragma unroll
            for (int e = 0; e < RUN; e++) { mine[e] = cut_k ? room.count[t * RUN + e] : room.mass[t * RUN + e]; sum += mine[e]; }
            u64 run = block.before(sum);
            if (!cut_k) {
                all_mass = block.both(Both{0, sum}).mass;
                limit = share * (double)all_mass;
            }
            auto reached = [&](u64 x) { return cut_k ? x >= (u64)k : (double)x >= limit; };
#pragma unroll
            for (int e = 0; e < RUN; e++) {          // (top-p of nothing: the first bin)
                if (reached(run + mine[e]) && (!reached(run) || t + e == 0)) { room.found = t * RUN + e; room.found_before = run; }
                run += mine[e];
            }
            __syncthreads();
            border = room.found;
            above = cut_k ? 0 : room.found_before;
        }
        // ---- the list; without top-k also the mass of the other kept tokens, by segment
        if (t == 0) room.n = 0;
        __syncthreads();
        auto enlist = [&](int segment, unsigned &listed) {
            for (; listed; listed &= listed - 1) {
                const int i = Seg::id_at(segment, __builtin_ctz(listed)), at = atomicAdd(&room.n, 1);
                if (at < LIST) room.keys[at] = rank_key(order_of((float)z[i]), i);
            }
        };
        if (cut_k) {
            unsigned listed = 0;                     // of a segment's numbers
            each_token<THREADS, SEGMENT>(z, V, [&](float v, int n, int) {
                listed |= (unsigned)(v > -INFINITY && sc.bin_of(sc.steps(v)) <= border) << n;
            }, [&](int s) { enlist(s, listed); });
        } else {
            u64 m = 0, all = 0;
            unsigned listed = 0;
            each_token<THREADS, SEGMENT>(z, V, [&](float v, int n, int) {
                const auto y = sc.steps(v);
                const int b = sc.bin_of(y);
                const bool is = v > -INFINITY;
                listed |= (unsigned)(b == border && is) << n;          // (border: BINS without a cut)
                const double w = sc.weight_of(y);
                const u64 x = units_of(w);
                const bool in = b < border && is && w >= (double)least;
                m += in ? x : 0;
                n_kept += in;
                all += x;
            }, [&](int s) {
                enlist(s, listed);
                m = wave_sum(m);
                if ((t & 63) == 0) room.segment[s] = m;
                m = 0;
            });
            if (!cut_p) all_mass = block.both(Both{0, all}).mass;
        }
        __syncthreads();
        const int m = room.n;
        if (m > LIST) { sample_by_digits<THREADS>(a, z, row, first, room); return; }
        while (P < m) P <<= 1;
        for (int i = m + t; i < P; i += THREADS) room.keys[i] = 0;
    }
    // ---- sorted, the cuts are places in the running sum
    int kept = 0;                          // of the list
    if (ranked || cut_p) {
        sort_keys<THREADS>(room.keys, P);
        const int per = (P + THREADS - 1) / THREADS, i0 = t * per, i1 = min(P, i0 + per), leading = ranked ? k : P;
        u64 all = 0, sum = 0;
        for (int i = i0; i < i1; i++) {
            const u64 key = room.keys[i], w = key ? sc.units(value_at(key)) : 0;
            all += w;
            if (i < leading) sum += w;
        }
        u64 run = above + block.before(sum);
        const Both sums = block.both(Both{all, sum});
        if (WHOLE) all_mass = sums.count;
        if (ranked) limit = share * (double)sums.mass;
        Both c{0, 0};
        for (int i = i0; i < min(i1, leading); i++) {
            const u64 key = room.keys[i];
            if (!key) break;
            const double x = sc.weight(value_at(key));
            const u64 w = units_of(x);
            if (key == first || ((!cut_p || (double)run < limit) && x >= (double)least)) { c.count++; c.mass += w; }
            run += w;
        }
        c = block.both(c);
        kept = (int)c.count;
        kept_mass = c.mass;
    }
    int token = id_of(first);
    if (ranked) {
        n_kept = kept;
        // ---- in id order: masses of buckets of ids, then the ids of the bucket in which u falls
        if (!greedy) {
            int shift = 0;
            while (((V - 1) >> shift) >= BINS) shift++;
            const int buckets = ((V - 1) >> shift) + 1, per = (buckets + THREADS - 1) / THREADS, b0 = t * per;
            for (int i = t; i < buckets; i += THREADS) room.bucket[i] = 0;
            if (t == 0) room.n = 0;
            __syncthreads();
            for (int i = t; i < kept; i += THREADS) atomicAdd(&room.bucket[id_of(room.keys[i]) >> shift], sc.units(value_at(room.keys[i])));
            __syncthreads();
            const double want = (double)u * (double)kept_mass;
            u64 sum = 0;
            for (int e = b0; e < min(b0 + per, buckets); e++) sum += room.bucket[e];
            u64 run = block.before(sum);
            for (int e = b0; e < min(b0 + per, buckets); e++) {
                if (falls_in(run, room.bucket[e], want, kept_mass)) { room.found = e; room.found_before = run; }
                run += room.bucket[e];
            }
            __syncthreads();
            token = room.found;                      // (shift 0: a bucket is an id)
            if (shift) {
                const int bucket = token;
                // its tokens, at most 2^shift <= 128, take the buckets' place
                for (int i = t; i < kept; i += THREADS)
                    if (id_of(room.keys[i]) >> shift == bucket) room.bucket[atomicAdd(&room.n, 1)] = room.keys[i];
                __syncthreads();
                const int m = room.n;
                Both pick{0, 0};
                if (t < m) {
                    const u64 key = room.bucket[t];
                    u64 r = room.found_before;
                    for (int j = 0; j < m; j++)
                        if (id_of(room.bucket[j]) < id_of(key)) r += sc.units(value_at(room.bucket[j]));
                    if (falls_in(r, sc.units(value_at(key)), want, kept_mass)) pick.count = (u64)id_of(key) + 1;
                }
                token = (int)block.both(pick, true).count - 1;
            }
        }
    } else {
        // ---- the list's kept tokens join their segments; the segment in which u falls is read once more
        const u64 last = kept > 0 ? room.keys[kept - 1] : ~0ull;
        for (int i = t; i < kept; i += THREADS) atomicAdd(&room.segment[id_of(room.keys[i]) / SEGMENT], sc.units(value_at(room.keys[i])));
        __syncthreads();
        const u64 mine = t * SEGMENT < V ? room.segment[t] : 0;
        const u64 run = block.before(mine);
        const Both sums = block.both(Both{(u64)n_kept, mine});
        n_kept = (int)sums.count + kept;
        kept_mass = sums.mass;
        if (!greedy) {
            const double want = (double)u * (double)kept_mass;
            if (falls_in(run, mine, want, kept_mass)) { room.found = t; room.found_before = run; }
            __syncthreads();
            const int i0 = room.found * SEGMENT;
            constexpr int RUN = (SEGMENT + THREADS - 1) / THREADS;
            u64 w[RUN], sum = 0;
#pragma unroll
            for (int e = 0; e < RUN; e++) {
                const int i = i0 + t * RUN + e;
                const float v = i < min(V, i0 + SEGMENT) ? (float)z[i] : -INFINITY;
                w[e] = 0;
                if (v > -INFINITY) {
                    const u64 key = rank_key(order_of(v), i);
                    const auto y = sc.steps(v);
                    const double x = sc.weight_of(y);
                    const int b = cut_p ? sc.bin_of(y) : 0;
                    if ((b < border || (b == border && key >= last)) && x >= (double)least) w[e] = units_of(x);
                }
                sum += w[e];
            }
            u64 r = room.found_before + block.before(sum);
            Both pick{0, 0};
#pragma unroll
            for (int e = 0; e < RUN; e++) {
                if (falls_in(r, w[e], want, kept_mass)) pick.count = (u64)(i0 + t * RUN + e) + 1;
                r += w[e];
            }
            token = (int)block.both(pick, true).count - 1;
        }
    }
    if (t == 0) {
        const double y = ((double)(float)z[token] - sc.zmax) * sc.rate * (0.69314718055994530942 / TABLE);
        a.token[row] = token;
        if (a.logp) a.logp[row] = (float)(y - log((double)all_mass / UNIT));
        if (a.logp_kept) a.logp_kept[row] = (float)(y - log((double)kept_mass / UNIT));
        if (a.n_kept) a.n_kept[row] = n_kept;
    }
}

}  // namespace

extern "C" {

size_t vla_sample_logits_workspace_bytes(int n, int vocab) {
    if (n <= 0 || vocab <= 0 || vocab > 262144) { vla_set_error("sample_logits: n must be positive, vocab 1 .. 262,144"); return 0; }
    return 256;          // (room that the call's form leaves: nothing is kept there)
}

int vla_sample_logits(const void *logits, int dtype, int64_t row_stride, int n, int vocab, const float *temperature, const int32_t *top_k,
                      const float *top_p, const float *min_p, const float *u, int32_t *token, float *logp, float *logp_kept, int32_t *n_kept,
                      void *ws, size_t ws_bytes, void *stream) {
    if (!logits || !token || !ws) { vla_set_error("sample_logits: logits, token or ws is NULL"); return VLA_EINVAL; }
    if (dtype != VLA_DTYPE_F32 && dtype != VLA_DTYPE_BF16) { vla_set_error("sample_logits: unknown dtype %d", dtype); return VLA_EDTYPE; }
    if (n <= 0 || vocab <= 0) { vla_set_error("sample_logits: n and vocab must be positive"); return VLA_EINVAL; }
    if (vocab > 262144) { vla_set_error("sample_logits: vocab %d unsupported (at most 262,144)", vocab); return VLA_ESHAPE; }
    if (row_stride < vocab) { vla_set_error("sample_logits: row stride shorter than vocab"); return VLA_ESHAPE; }
    const size_t need = vla_sample_logits_workspace_bytes(n, vocab);
    if (ws_bytes < need) { vla_set_error("sample_logits: workspace %zu bytes, need %zu", ws_bytes, need); return VLA_EWORKSPACE; }
    const SampleArgs a{(const char *)logits, (long)row_stride, n, vocab, temperature, top_k, top_p, min_p, u, token, logp, logp_kept, n_kept};
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps("sample_logits", (double)n * vocab * (dtype == VLA_DTYPE_F32 ? 4.0 : 2.0), st);
    // A row of up to SHORT tokens is sorted whole, by few waves; longer ones go by bins (256 rows of 1024 tokens, 4096: sorted whole 28 and 63 us,
    // by bins 20 and 24).  Up to 8192 by eight waves, whose barriers cost less than sixteen's (1000: 20 us for 23, 8000: 26 for 27; 16,000: 31 both ways, 32,000: 45
    // for 40).  Segments of 512 ids have two loads of 16 bytes a lane on their way, and 512 of them are the longest row; shorter rows
    // take 256, so that each of the waves has some.  (1024 ids do not fit the registers: 128,000 logits 160 us for 112.)
    auto go = [&](auto type) {
        typedef decltype(type) T;
        if (vocab <= SHORT) sample_rows_kernel<256, 256, true, T><<<n, 256, 0, st>>>(a);
        else if (vocab <= 8192) sample_rows_kernel<512, 256, false, T><<<n, 512, 0, st>>>(a);
        else if (vocab <= 32768) sample_rows_kernel<1024, 256, false, T><<<n, 1024, 0, st>>>(a);
        else sample_rows_kernel<1024, 512, false, T><<<n, 1024, 0, st>>>(a);
    };
    if (dtype == VLA_DTYPE_F32) go(0.f);
    else go((bf16_t)0.f);
    return vla_check_launch("sample_logits");
}

}  // extern "C"
