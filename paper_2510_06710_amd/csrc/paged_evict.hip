// Eviction from a paged KV cache by accumulated attention weight: the weights of a call's rows summed per position, and a cache cut to the
// heaviest positions.
#include "paged_rows.h"
#include "paged_select.h"

namespace {

// ---- weights -----------------------------------------------------------------------------------------------------------------
// One product, S = Q K^T (rows queries, columns keys, on 32 x 32 matrix instructions), so a lane owns a key: its weights' sum over the queries is a
// sum over the lane's registers (and lane ^ 32).  The packed rows are those of paged_attention.hip: query r / group, head r % group of a key head's
// group.  Two forms: few packed rows stay in registers and the keys stream by (paged_weights_step_kernel); of many, the keys stay and the
// rows stream (paged_weights_rows_kernel), in parts that paged_weights_join_kernel adds up in order.
struct WeightArgs {
    AttnArgs a;
    const float *lse_in;
    float *mass, *part;      // part: [parts][n_seq][n_kv][max_len]
    long mass_stride;
    int chunk;               // tiles of keys (step) or of packed rows (rows) of one workgroup
    int parts;
    int waves;               // step: among which a key head's tiles are divided (0: by chunks)
};

// The packed rows of a sequence, as tiles of 32, that may see one of the keys key0 .. key0 + n - 1: positions key0 on, below key0 + n - 1 + window; all where the prefix reaches.
struct RowTiles { int t0, t1; };
__device__ __forceinline__ int prefix_of(const AttnArgs &a, int s, const PagedSeq &sq) { return a.prefix_len ? min(max(paged_int(a.prefix_len, s), 0), sq.keys) : 0; }
__device__ __forceinline__ RowTiles row_tiles(const AttnArgs &a, const PagedSeq &sq, int prefix, int key0, int n) {
    const int base = sq.len - sq.n;
    int i0 = max(0, key0 - base), i1 = sq.rows;
    if (a.window) i1 = (int)min((long)i1, max(0L, (long)key0 + n - 1 + a.window - base));
    if (key0 < prefix) { i0 = 0; i1 = sq.rows; }
    if (i0 >= i1) return {0, 0};
    return {i0 * a.group / 32, (i1 * a.group + 31) / 32};
}

// A capped score, in the units of Rows::shaped.
template <typename T> __device__ __forceinline__ float capped(const AttnArgs &a, float z) {
    return sizeof(T) == 4 ? tanhf(z * (a.scale / a.cap)) : -__builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * (2.f * LOG2E * a.scale / a.cap)));
}

// The weights of one tile, in a lane sixteen rows' for its key: register 4 g + e is packed row 8 g + 4 hh + e.  l: lse in log2 units less the scores' offset; p: positions; MASKED: not all
// of them may count.  Summed by fours first, so that a long sum has few steps of its own.
template <typename T, int DP, int MODE, bool MASKED>
__device__ __forceinline__ float tile_weight(const AttnArgs &a, const f32x16_t &x, const float (&l)[16], const int (&p)[16], const float (&slope)[16], int key, int keys, int prefix) {
    const float unit = Rows<T, DP, MODE, false>::unit_of(a);
    const int window = a.window ? a.window : 0x7fffffff;
    float sum[4];
#pragma unroll
    for (int i = 0; i < 16; i++) {
        float z = x[i];
        if (MODE & CAPPED) z = capped<T>(a, z);
        if (MODE & BIASED) {
            const float factor = MODE & CAPPED ? (sizeof(T) == 4 ? 1.f : 2.f) * a.cap * LOG2E : a.scale * LOG2E;
            z = __builtin_fmaf(-slope[i], fabsf((float)(p[i] - key)), z * factor);
        }
        float w = __builtin_amdgcn_exp2f(__builtin_fmaf(z, unit, -l[i]));
        if (MASKED) {                                         // (p - key below 0, or beyond the window: as one comparison without sign)
            const bool see = (((unsigned)(p[i] - key) < (unsigned)window) | (key < prefix)) & (key < keys) & (l[i] != INFINITY);
            w = see ? w : 0.f;
        }
        sum[i % 4] = i < 4 ? w : sum[i % 4] + w;
    }
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

// One wave a workgroup, as many as their rings fit the chip; each takes one key head's equal run of the key tiles of all sequences, whatever their lengths.  Up to 32 packed rows of a
// sequence are in registers, its tiles of 32 keys come through a ring of three in LDS (rows of 16 keys of a page, as in paged_attention.hip); their sums go to LDS and to memory eight tiles at a time.
// Of more than 2048 sequences a wave takes `chunk` tiles of one (every wave looks at all sequences' lengths to find its run).
// Bound by memory: 64 rows behind up to 4096 keys, 8 heads of 128, 248 MB in 56 us, 4.4 TB/s; in fp32 488 MB in 139 us, 3.5 TB/s.  (Chunks of one sequence's tiles a workgroup: 57 to 67.)  Scores, weights and sums are fp32.
constexpr int STEP_TILES = 8;
struct StepTiles { int from, n; };           // of a sequence: those that a row sees or that hold new positions (all behind the first row's window, and before the prefix's end)
__device__ __forceinline__ StepTiles step_tiles(const AttnArgs &a, int s) {
    const PagedSeq sq = paged_seq(a.pv, s);
    if (sq.rows == 0) return {0, 0};
    const int from = a.window && prefix_of(a, s, sq) == 0 ? max(0, sq.len - sq.n + 1 - a.window) / 32 : 0;
    return {from, max(0, (sq.keys + 31) / 32 - from)};
}
template <typename T, int DP, int MODE>
__global__ void __launch_bounds__(64) paged_weights_step_kernel(WeightArgs w) {
    typedef Tile<T, DP> TL;
    typedef Rows<T, DP, MODE, false> R;
    constexpr int KS = DP / 16, BYTES = 32 * TL::ROW, LOADS = 2 * 16 / TL::RPI;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ __attribute__((aligned(16))) float sums[STEP_TILES * 32], info[3][32];
    const unsigned ring0 = (unsigned)(size_t)(lds_void *)lds;
    const AttnArgs &a = w.a;
    const PagedView &pv = a.pv;
    const int lane = threadIdx.x, col = lane & 31, hh = lane >> 5;
    const unsigned id = blockIdx.x / (unsigned)pv.n_kv;
    const int kvh = blockIdx.x % (unsigned)pv.n_kv;
    int s = 0, skip = 0, left;                               // the sequence it is in; tiles of it that are not its own; tiles of its run that are left
    if (w.waves) {
        int all = 0, c = 0;
        for (int z = lane; z < pv.n_seq; z += 64) all += c = step_tiles(a, z).n;
        all = __builtin_amdgcn_readfirstlane(wave_sum(all));
        const int share = max(2, (int)((unsigned)(all + w.waves - 1) / (unsigned)w.waves));
        int rest = __builtin_amdgcn_readfirstlane(id * share);
        left = __builtin_amdgcn_readfirstlane(min(share, all - rest));
        if (left <= 0) return;
        for (int s0 = 0; s0 < pv.n_seq; s0 += 64) {
            if (pv.n_seq > 64) c = s0 + lane < pv.n_seq ? step_tiles(a, s0 + lane).n : 0;
            int in = c;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) { const int v = __shfl_up(in, o, 64); if (lane >= o) in += v; }
            const unsigned long long past = __ballot(in > rest);
            if (past) {
                const int l = __builtin_ctzll(past);
                s = __builtin_amdgcn_readfirstlane(s0 + l);
                skip = __builtin_amdgcn_readfirstlane(rest - __shfl(in - c, l, 64));
                break;
            }
            rest -= __builtin_amdgcn_readlane(in, 63);
        }
    } else {
        s = __builtin_amdgcn_readfirstlane(id % (unsigned)pv.n_seq);
        skip = __builtin_amdgcn_readfirstlane(id / (unsigned)pv.n_seq * w.chunk);
        left = min(w.chunk, step_tiles(a, s).n - skip);
        if (left <= 0) return;
    }
    typename TL::template Offsets<false, 16> off;
    off.start(pv, 0);
    const Place place(pv, kvh, sizeof(T));
    for (; left > 0 && s < pv.n_seq; s++, skip = 0) {
        const StepTiles its = step_tiles(a, s);
        const int take = min(its.n - skip, left), t0 = its.from + skip, t1 = t0 + take;
        if (take <= 0) continue;
        left -= take;
        const PagedSeq sq = paged_seq(pv, s);
        const int base = sq.len - sq.n, prefix = prefix_of(a, s, sq);
        const Span sp{0, sq.keys, 0, 0};
        const int32_t *table = pv.table + (size_t)s * pv.table_stride;
        int p0 = sp.page(table, pv.page_log, t0 * 32), p1 = sp.page(table, pv.page_log, t0 * 32 + 16);
        auto load = [&](int t, int stage) __attribute__((always_inline)) {
            const unsigned at = ring0 + stage * BYTES;
            if ((t + 1) * 32 <= sq.keys) {
                off.load(at, place.in(pv, pv.k, p0, place.at(pv, p0, t * 32)));
                off.load(at + 16 * TL::ROW, place.in(pv, pv.k, p1, place.at(pv, p1, t * 32 + 16)));
            } else {
                TL::template load<false, 16>(at, pv.k, pv, p0, kvh, t * 32, sp);
                TL::template load<false, 16>(at + 16 * TL::ROW, pv.k, pv, p1, kvh, t * 32 + 16, sp);
            }
            p0 = sp.page(table, pv.page_log, t * 32 + 32);
            p1 = sp.page(table, pv.page_log, t * 32 + 48);
        };
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");    // the reads of the last sequence's tiles are through
        load(t0, 0);
        if (t0 + 1 < t1) load(t0 + 1, 1);
        Query y{};
        const int i = col / a.group, hg = col - i * a.group;
        y.valid = i < sq.rows;
        y.row = sq.r0 + (y.valid ? i : 0);
        y.head = kvh * a.group + hg;
        if (hh == 0) {
            const float l = y.valid ? w.lse_in[(size_t)y.row * a.n_heads + y.head] : -INFINITY;
            info[0][col] = l == -INFINITY ? INFINITY : l * LOG2E - a.offset;          // (such a row's weights are exp2 of -inf)
            info[1][col] = __builtin_bit_cast(float, y.valid ? base + i : 0x7fffffff);
            info[2][col] = (MODE & BIASED) && y.valid ? a.slopes[y.head] * LOG2E : 0.f;
        }
        R rows;
        rows.start(a, y);
        float l[16], slope[16];
        int p[16], low = 0x7fffffff;                          // low: the first row's position
        bool odd = false;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
        for (int r = 0; r < 16; r++) {
            const int at = 8 * (r / 4) + 4 * hh + r % 4;
            l[r] = info[0][at];
            p[r] = __builtin_bit_cast(int, info[1][at]);
            slope[r] = info[2][at];
            low = min(low, p[r]);
            odd |= !(l[r] < INFINITY);
        }
        low = wave_min(low);
        odd = __any(odd);
        float *mass = w.mass + ((size_t)s * pv.n_kv + kvh) * w.mass_stride;
        int stage = 0, first = t0;                            // of the tiles whose sums are in LDS
        for (int t = t0; t < t1; t++) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // the reads of the stage that is loaded again are through
            if (t + 2 < t1) { load(t + 2, stage >= 1 ? stage - 1 : 2); vm_wait<2 * LOADS>(); }
            else if (t + 1 < t1) vm_wait<LOADS>();
            else vm_wait<0>();
            const char *kt = lds + stage * BYTES;
            f32x16_t x;
#pragma unroll
            for (int e = 0; e < 16; e++) x[e] = 0.f;
#pragma unroll
            for (int kk = 0; kk < KS; kk++) x = mma(rows.q[kk], R::key(kt, kk), x);
            const bool masked = odd || t * 32 + 31 > low || (t + 1) * 32 > sq.keys || a.window;
            float sum = masked ? tile_weight<T, DP, MODE, true>(a, x, l, p, slope, t * 32 + col, sq.keys, prefix) : tile_weight<T, DP, MODE, false>(a, x, l, p, slope, t * 32 + col, sq.keys, prefix);
            sum = vla_fold_step<32>(sum, VlaAdd());
            if (hh == 0) sums[(t - first) * 32 + col] = sum;
            stage = stage == 2 ? 0 : stage + 1;
            if (t + 1 == t1 || t + 1 - first == STEP_TILES) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                for (int key = first * 32 + lane; key < min((t + 1) * 32, sq.keys); key += 64) {
                    const float add = sums[key - first * 32];
                    mass[key] = key < base ? mass[key] + add : add;
                }
                first = t + 1;
            }
        }
    }
}

// (Tried: four tiles of keys a wave with the lse subtracted by a matrix instruction, which halves what is read of LDS, 130 us and more: one tile's products wait for each other.  Vector and matrix work
// share the time of a CU's units here: without the exponentials a call of 140 us took 122, without the products 106, without loads 127.)
// Four waves, each with KW tiles of 32 keys in registers; tiles of 32 packed rows of q come through a ring of four in LDS, a quarter loaded by each wave, with the rows' lse
// beside them (a copy for each wave: no register is loaded inside the loop).  A row of q may start anywhere: where rows are no multiples of 16 bytes they go through registers.
// The exponentials of one tile of rows are taken between the matrix instructions of the next.
// Bound by the matrix and the vector units together: 4096 causal rows of 32 heads of 128, 8 key heads: 118 us and 5 for the join, 580 TFLOP/s of scores, where a plain product of that
// size takes 49 us and the vector work of 268 million weights most of the rest; in fp32 680 us, 101 TFLOP/s of the card's 153.  (The simple kernel, rows kept and keys streamed: 1359 us.)
template <typename T, int DP> constexpr int KEY_TILES = sizeof(T) * DP <= 256 ? 2 : 1;
template <typename T, int DP, int MODE>
__global__ void __launch_bounds__(256, sizeof(T) * DP <= 256 ? 2 : 1) paged_weights_rows_kernel(WeightArgs w) {
    typedef Tile<T, DP> TL;
    typedef Rows<T, DP, MODE, false> R;
    typedef typename FragOf<T>::type frag;
    constexpr int KS = DP / 16, BYTES = 32 * TL::ROW, RG = 4, EACH = 8 / TL::RPI, LOADS = EACH + 1, KW = KEY_TILES<T, DP>, KEYS = 128 * KW;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    constexpr int GONE = -0x40000000;
    __shared__ __attribute__((aligned(16))) float lse_at[RG][4][64];
    __shared__ __attribute__((aligned(16))) int info[2][4][32];
    const unsigned lds0 = (unsigned)(size_t)(lds_void *)lds, lse0 = (unsigned)(size_t)(lds_void *)&lse_at[0][0][0];
    const AttnArgs &a = w.a;
    const PagedView &pv = a.pv;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 31, hh = lane >> 5;
    const unsigned id = blockIdx.x / (unsigned)pv.n_kv;
    const int kvh = blockIdx.x % (unsigned)pv.n_kv, s = id % (unsigned)pv.n_seq, block0 = __builtin_amdgcn_readfirstlane(id / (unsigned)pv.n_seq * KEYS);
    const PagedSeq sq = paged_seq(pv, s);
    if (block0 >= sq.keys) return;
    const int base = sq.len - sq.n, prefix = prefix_of(a, s, sq), rows = sq.rows * a.group;
    const RowTiles all = row_tiles(a, sq, prefix, block0, KEYS);
    const int t0 = __builtin_amdgcn_readfirstlane(max(all.t0, (int)blockIdx.y * w.chunk)), t1 = __builtin_amdgcn_readfirstlane(min(all.t1, ((int)blockIdx.y + 1) * w.chunk));
    const int key0 = block0 + wave * 32 * KW;
    if (w.parts > 1 ? t0 >= t1 : sq.rows == 0 || (all.t0 == all.t1 && base >= block0 + KEYS)) return;
    // a lane's part of a tile of rows: the head of each of its loads, and its offset from the tile's first row's first head (of q in bytes, of lse in words)
    const int step_i = 32 / a.group, step_h = 32 % a.group;
    int head[EACH + 1];
    unsigned off[EACH + 1];
    int i0 = 0, h0 = 0;                                       // the first row and its head of the next tile to load
    auto offsets = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e <= EACH; e++) {
            const unsigned r = h0 + (e < EACH ? wave * 8 + e * TL::RPI + lane / TL::CPR : col), i = r / (unsigned)a.group;
            head[e] = r - i * a.group;
            // (rows behind the last: the last's, which count for nothing)
            const unsigned at = min((int)i, sq.rows - 1 - i0);
            if (e == EACH) off[e] = (at * a.n_heads + head[e]) * 4;
            else {
                const int z = wave * 8 + e * TL::RPI + lane / TL::CPR, c = min((lane % TL::CPR) ^ TL::fk(z), pv.d * (int)sizeof(T) / 16 - 1);
                off[e] = (unsigned)(at * a.q_stride + head[e] * pv.d) * (unsigned)sizeof(T) + c * 16;
            }
        }
    };
    {
        const unsigned r = t0 * 32, i = r / (unsigned)a.group;
        i0 = __builtin_amdgcn_readfirstlane(i);
        h0 = __builtin_amdgcn_readfirstlane(r - i * a.group);
    }
    if (t0 < t1) offsets();
    const T *q_at = (const T *)a.q + (size_t)(sq.r0 + i0) * a.q_stride + (size_t)kvh * a.group * pv.d;
    const float *l_at = w.lse_in + (size_t)(sq.r0 + i0) * a.n_heads + kvh * a.group;
    const size_t q_step = step_i * a.q_stride, l_step = (size_t)step_i * a.n_heads;
    auto load = [&](int t, int stage) __attribute__((always_inline)) {
        if (t >= t1) return;
        // (the offsets are the last tile's, unless a tile is no whole number of rows, or this is the end of the rows)
        if (step_h || (t + 1) * 32 > rows) offsets();
        const unsigned at = lds0 + stage * BYTES + wave * 8 * TL::ROW;
        if (a.aligned) {
#pragma unroll
            for (int e = 0; e < EACH; e++) dma16(at + e * 1024, off[e], (const char *)q_at);
        } else {
#pragma unroll
            for (int e = 0; e < EACH; e++) {
                const int z = wave * 8 + e * TL::RPI + lane / TL::CPR, c = min((lane % TL::CPR) ^ TL::fk(z), pv.d * (int)sizeof(T) / 16 - 1);
                const unsigned i = (unsigned)(h0 + z) / (unsigned)a.group;
                const T *src = q_at + (size_t)min((int)i, sq.rows - 1 - i0) * a.q_stride + head[e] * pv.d + c * (16 / (int)sizeof(T));
                T x[16 / sizeof(T)];
#pragma unroll
                for (int y = 0; y < 16 / (int)sizeof(T); y++) x[y] = src[y];
                __builtin_memcpy(lds + stage * BYTES + wave * 8 * TL::ROW + e * 1024 + lane * 16, x, 16);
            }
        }
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lse0 + (stage * 4 + wave) * 256), "v"(off[EACH]), "s"(l_at) : "memory");
        i0 += step_i;
        q_at += q_step;
        l_at += l_step;
        if (step_h) {
            h0 += step_h;
            if (h0 >= a.group) { h0 -= a.group; i0++; q_at += a.q_stride; l_at += a.n_heads; }
        }
    };
#pragma unroll
    for (int t = 0; t < RG; t++) load(t0 + t, t);
    // the keys; zeros in dims that are not there (LDS holds repeated values of q in their place)
    frag k[KW][KS];
    {
        const Span sp{0, sq.keys, 0, 0};
        const int32_t *table = pv.table + (size_t)s * pv.table_stride;
#pragma unroll
        for (int b = 0; b < KW; b++) {
            const int at = key0 + b * 32, p0 = sp.page(table, pv.page_log, at), p1 = sp.page(table, pv.page_log, at + 16), page = col < 16 ? p0 : p1;
            const bool ok = (unsigned)page < (unsigned)pv.n_pages;
            const T *src = ok ? (const T *)pv.k + ((((size_t)page * pv.n_kv + kvh) << pv.page_log) + (min(at + col, sq.keys - 1) & ((1 << pv.page_log) - 1))) * pv.d : (const T *)zero_rows;
#pragma unroll
            for (int kk = 0; kk < KS; kk++) {
                if (kk * 16 < pv.d) k[b][kk] = *(const frag *)(src + kk * 16 + hh * 8);
                else
#pragma unroll
                    for (int e = 0; e < 8; e++) k[b][kk][e] = (T)0.f;
            }
        }
    }
    const float unit = R::unit_of(a);
    const int window = a.window ? a.window : 0x7fffffff;
    float sum[KW], l[16];
#pragma unroll
    for (int b = 0; b < KW; b++) sum[b] = 0.f;
    // Of a tile that has arrived: lse in log2 units less the scores' offset, by the lane that has the row; whether every row is there, its lse finite, and all of the wave's keys before it.
    const int whole0 = key0 + 32 * KW > sq.keys || a.window ? 0x7fffffff : (max(0, key0 + 32 * KW - 1 - base) * a.group + 31) / 32;
    const int hidden = key0 < prefix ? 0 : max(0, key0 - base) * a.group / 32;
    bool masked;
    float mine;
    auto arrive = [&](int t, int stage) __attribute__((always_inline)) {
        const float v = lse_at[stage][wave][lane];
        mine = MODE & CAPPED ? __builtin_fmaf(v, LOG2E, -a.offset) : v * LOG2E;
        masked = t < whole0 || t * 32 + 32 > rows || __any(!(fabsf(v) < INFINITY));
        lse_at[stage][wave][lane] = mine;
    };
    // The tile's scores as they enter the exponentials (-inf where the key is not seen), and its lse.
    auto shape = [&](int t, int stage, f32x16_t (&x)[KW]) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < 4; g++) {
            const f32x4_t v = *(const f32x4_t *)&lse_at[stage][wave][8 * g + 4 * hh];
#pragma unroll
            for (int e = 0; e < 4; e++) l[4 * g + e] = v[e];
        }
        if (MODE & CAPPED)
#pragma unroll
            for (int b = 0; b < KW; b++)
#pragma unroll
                for (int r = 0; r < 16; r++) x[b][r] = capped<T>(a, x[b][r]);
        if (t < hidden) {                                     // none of the rows sees any of the wave's keys
#pragma unroll
            for (int r = 0; r < 16; r++) {
                l[r] = 0.f;
#pragma unroll
                for (int b = 0; b < KW; b++) x[b][r] = -INFINITY;
            }
            return;
        }
        if (masked || (MODE & BIASED)) {
            // a lane's own row of the tile, for the others: lse as it is used, position (GONE: of a row that counts for nothing), slope
            const int at = t * 32 + col, i = (unsigned)at / (unsigned)a.group;
            const bool there = (at < rows) & (mine != -INFINITY);
            if (hh == 0) {
                lse_at[stage][wave][col] = there ? mine : 0.f;
                info[0][wave][col] = there ? base + i : GONE;
                if (MODE & BIASED) info[1][wave][col] = there ? __builtin_bit_cast(int, a.slopes[kvh * a.group + at - i * a.group] * LOG2E) : 0;
            }
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
            for (int g = 0; g < 4; g++) {
                __builtin_amdgcn_sched_barrier(0);            // (few values alive at a time)
                const i32x4_v p = *(const i32x4_v *)&info[0][wave][8 * g + 4 * hh];
                const f32x4_t v = *(const f32x4_t *)&lse_at[stage][wave][8 * g + 4 * hh];
#pragma unroll
                for (int e = 0; e < 4; e++) {
                    const int r = 4 * g + e;
                    l[r] = v[e];
#pragma unroll
                    for (int b = 0; b < KW; b++) {
                        const int key = key0 + b * 32 + col;
                        if (MODE & BIASED) {
                            const float factor = MODE & CAPPED ? (sizeof(T) == 4 ? 1.f : 2.f) * a.cap * LOG2E : a.scale * LOG2E;
                            x[b][r] = __builtin_fmaf(-__builtin_bit_cast(float, info[1][wave][8 * g + 4 * hh + e]), fabsf((float)(p[e] - key)), x[b][r] * factor);
                        }
                        // (p - key below 0, or beyond the window: as one comparison without sign)
                        const bool see = (((unsigned)(p[e] - key) < (unsigned)window) | ((key < prefix) & (p[e] != GONE))) & (key < sq.keys);
                        x[b][r] = see ? x[b][r] : -INFINITY;
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // the scores of the tile in stage `next_at`, and the weights of x between them
    constexpr int N = 16 * KW, AHEAD = KS < 3 ? KS : 3;
    auto weights = [&](f32x16_t (&x)[KW], float (&part)[KW][4], int from, int to) __attribute__((always_inline)) {
#pragma unroll
        for (int n = from; n < to; n++) {
            const int b = n / 16, i = n % 16;
            const float v = __builtin_amdgcn_exp2f(__builtin_fmaf(x[b][i], unit, -l[i]));
            part[b][i % 4] = i < 4 ? v : part[b][i % 4] + v;
        }
    };
    auto scores = [&](int stage, f32x16_t (&next)[KW], f32x16_t (&x)[KW], bool between) __attribute__((always_inline)) {
        const char *qt = lds + stage * BYTES;
        float part[KW][4];
        frag q[AHEAD];
#pragma unroll
        for (int kk = 0; kk < AHEAD; kk++) q[kk] = R::key(qt, kk);
#pragma unroll
        for (int b = 0; b < KW; b++)
#pragma unroll
            for (int e = 0; e < 16; e++) next[b][e] = 0.f;
#pragma unroll
        for (int kk = 0; kk < KS; kk++) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int b = 0; b < KW; b++) next[b] = mma(q[kk % AHEAD], k[b][kk], next[b]);
            if (kk + AHEAD < KS) q[kk % AHEAD] = R::key(qt, kk + AHEAD);
            if (between) weights(x, part, kk * N / KS, (kk + 1) * N / KS);
        }
        __builtin_amdgcn_sched_barrier(0);
        if (between)
#pragma unroll
            for (int b = 0; b < KW; b++) {
                sum[b] += (part[b][0] + part[b][1]) + (part[b][2] + part[b][3]);
                asm volatile("" : "+v"(sum[b]));              // (here, and not where the compiler would move it, behind the next tile's masks)
            }
    };
    // Tile t lies in stage (t - t0) % RG.  At step t its scores are there; everyone is through with its place, which tile t + RG takes.
    auto arrived = [&](int t) __attribute__((always_inline)) {          // tile t, t + 1 and t + 2 perhaps not
        if (a.aligned && t + 2 < t1) vm_wait<2 * LOADS>();
        else vm_wait<0>();
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    };
    f32x16_t x0[KW], x1[KW];
    if (t0 < t1) {
        if (a.aligned && t0 + 3 < t1) vm_wait<3 * LOADS>();
        else vm_wait<0>();
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        arrive(t0, 0);
        scores(0, x0, x1, false);
        shape(t0, 0, x0);
        int t = t0;
        auto step = [&](int stage, f32x16_t (&x)[KW], f32x16_t (&next)[KW]) __attribute__((always_inline)) {
            const int after = stage == RG - 1 ? 0 : stage + 1;
            if (t + 1 < t1) {
                arrived(t + 1);
                load(t + RG, stage);
                arrive(t + 1, after);
            }
            scores(after, next, x, true);                     // (behind the last tile: of what lies there, for no one)
            if (t + 1 < t1) shape(t + 1, after, next);
            return ++t < t1;
        };
        while (step(0, x0, x1) && step(1, x1, x0) && step(2, x0, x1) && step(3, x1, x0)) {}
    }
#pragma unroll
    for (int b = 0; b < KW; b++) {
        const float all_of = vla_fold_step<32>(sum[b], VlaAdd());
        const int key = key0 + b * 32 + col;
        if (hh || key >= sq.keys) continue;
        if (w.parts > 1) w.part[(((size_t)blockIdx.y * pv.n_seq + s) * pv.n_kv + kvh) * pv.max_len + key] = all_of;
        else {
            float *m = w.mass + ((size_t)s * pv.n_kv + kvh) * w.mass_stride + key;
            *m = key < base ? *m + all_of : all_of;
        }
    }
}

// The parts of each position, in order.  keys: of a block of paged_weights_rows_kernel.  5 us for 24 parts of 8 x 4096 positions: its look-ups and one round of loads.
__global__ void __launch_bounds__(256) paged_weights_join_kernel(WeightArgs w, int keys) {
    const AttnArgs &a = w.a;
    const PagedView &pv = a.pv;
    const unsigned id = blockIdx.x / (unsigned)pv.n_kv;
    const int kvh = blockIdx.x % (unsigned)pv.n_kv, s = id % (unsigned)pv.n_seq, key = (int)(id / (unsigned)pv.n_seq) * 256 + threadIdx.x;
    const PagedSeq sq = paged_seq(pv, s);
    if (key >= sq.keys || sq.rows == 0) return;
    const int base = sq.len - sq.n;
    const RowTiles all = row_tiles(a, sq, prefix_of(a, s, sq), key / keys * keys, keys);
    float sum = 0.f;
    const size_t step = (size_t)pv.n_seq * pv.n_kv * pv.max_len;
    const float *part = w.part + ((size_t)s * pv.n_kv + kvh) * pv.max_len + key;
    if (all.t0 < all.t1)
#pragma unroll 8
        for (int z = all.t0 / w.chunk; z <= (all.t1 - 1) / w.chunk; z++) sum += part[z * step];
    float *m = w.mass + ((size_t)s * pv.n_kv + kvh) * w.mass_stride + key;
    if (key >= base) *m = sum;
    else if (all.t0 < all.t1) *m += sum;
}

// How a call is divided.
struct WeightPlan {
    bool step;
    int chunk, parts, waves;
    long items;              // workgroups of a part
};
int weight_keys(int d, bool f32) { return 128 * (padded_dim(d) * (f32 ? 4 : 2) <= 256 ? 2 : 1); }
WeightPlan plan_weights(const AttnArgs &a, bool f32) {
    WeightPlan p{};
    const PagedView &pv = a.pv;
    const long pairs = (long)pv.n_kv * pv.n_seq, packed = (long)(pv.max_rows < pv.n_rows ? pv.max_rows : pv.n_rows) * a.group;
    p.step = packed <= 32;
    p.parts = 1;
    if (p.step) {
        const long tiles = (pv.max_len + 31) / 32, all = pairs * tiles;
        // (LDS is handed out in units of 1280 bytes)
        const int units = (3 * 32 * padded_dim(pv.d) * (f32 ? 4 : 2) + (STEP_TILES + 3) * 128 + 1279) / 1280, fit = 128 / units;
        p.waves = pv.n_seq <= 2048 && all < 1L << 30 ? 256 * (fit > 8 ? 8 : fit) / pv.n_kv : 0;
        if (p.waves == 0 && pv.n_seq <= 2048 && all < 1L << 30) p.waves = 1;
        if (p.waves > all / pv.n_kv) p.waves = all / pv.n_kv > 0 ? (int)(all / pv.n_kv) : 1;
        p.chunk = STEP_TILES;
        p.items = pv.n_seq <= 2048 && all < 1L << 30 ? (long)p.waves * pv.n_kv : pairs * ((tiles + p.chunk - 1) / p.chunk);
        return p;
    }
    // Workgroups for six rounds of two a CU, with eight tiles of rows at least (4096 causal rows, 8 key heads: one round 141 us, from three to ten 120 to 128).
    const int keys = weight_keys(pv.d, f32);
    const long tiles = (packed + 31) / 32, blocks = pairs * ((pv.max_len + keys - 1) / keys);
    long parts = blocks > 0 ? (6 * 512 + blocks - 1) / blocks : 1;
    if (parts > tiles / 8) parts = tiles / 8;
    if (parts > 256) parts = 256;
    if (parts < 1) parts = 1;
    p.chunk = (int)((tiles + parts - 1) / parts);
    p.parts = (int)((tiles + p.chunk - 1) / p.chunk);
    p.items = blocks;
    return p;
}
size_t weight_bytes(const AttnArgs &a, const WeightPlan &p) {
    return p.parts > 1 ? round_up((size_t)p.parts * a.pv.n_seq * a.pv.n_kv * a.pv.max_len * sizeof(float)) : 256;
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
    a->scale = mask->scale; a->cap = mask->softcap; a->slopes = mask->slopes; a->prefix_len = mask->prefix_len; a->window = mask_window(*mask);
    const long items = plan_weights(*a, cache->dtype == VLA_DTYPE_F32).items, joins = (long)cache->n_kv_heads * batch->n_seq * ((batch->max_len + 255) / 256);
    if (items > 0x7fffffffL / 256 || joins > 0x7fffffffL / 256) { vla_set_error("%s: %ld tiles of positions are too many: split the batch", what, items); return VLA_ESHAPE; }
    return VLA_OK;
}

template <typename T, int DP, int MODE>
int launch_weights(WeightArgs w, const WeightPlan &p, hipStream_t st) {
    const PagedView &pv = w.a.pv;
    w.chunk = p.chunk;
    w.parts = p.parts;
    w.waves = p.waves;
    if (p.step) {
        constexpr size_t bytes = 3 * 32 * Tile<T, DP>::ROW;
        if (int rc = vla_allow_lds((const void *)paged_weights_step_kernel<T, DP, MODE>, bytes)) return rc;
        paged_weights_step_kernel<T, DP, MODE><<<(unsigned)p.items, 64, bytes, st>>>(w);
        return vla_check_launch("paged_weights");
    }
    constexpr size_t bytes = 4 * 32 * Tile<T, DP>::ROW;
    if (int rc = vla_allow_lds((const void *)paged_weights_rows_kernel<T, DP, MODE>, bytes)) return rc;
    paged_weights_rows_kernel<T, DP, MODE><<<dim3((unsigned)p.items, p.parts), 256, bytes, st>>>(w);
    if (int rc = vla_check_launch("paged_weights")) return rc;
    if (p.parts == 1) return VLA_OK;
    paged_weights_join_kernel<<<(unsigned)(pv.n_kv * pv.n_seq * ((pv.max_len + 255) / 256)), 256, 0, st>>>(w, 128 * KEY_TILES<T, DP>);
    return vla_check_launch("paged_weights join");
}
template <typename T, int DP>
int launch_weights_masked(const WeightArgs &w, const WeightPlan &p, hipStream_t st) {
    switch ((w.a.cap > 0.f ? CAPPED : 0) | (w.a.slopes ? BIASED : 0)) {
        case 0: return launch_weights<T, DP, 0>(w, p, st);
        case CAPPED: return launch_weights<T, DP, CAPPED>(w, p, st);
        case BIASED: return launch_weights<T, DP, BIASED>(w, p, st);
        default: return launch_weights<T, DP, CAPPED | BIASED>(w, p, st);
    }
}
template <typename T>
int launch_weights_sized(const WeightArgs &w, const WeightPlan &p, hipStream_t st) {
    switch (padded_dim(w.a.pv.d)) {
        case 64: return launch_weights_masked<T, 64>(w, p, st);
        case 128: return launch_weights_masked<T, 128>(w, p, st);
        default: return launch_weights_masked<T, 256>(w, p, st);
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

// A workgroup for each (sequence, key head): the least mass that stays, then the positions of what is above it and of the first that equal it, in order, then their masses, 8192 at a time, read
// before they are written: none lands behind its place, so mass_out may be mass.  Up to 32,768 positions' masses are held in LDS as the numbers they are ordered by (HELD); of more every pass reads
// them again.  The first and last that stay anyway have the largest number.  Positions without weight, many of a kind, are counted by ballot: as one bin they would be added to one after the other.
// Bound by the vector instructions of one CU, some fifteen a position and pass: 128 lists of up to 32,768 cut to 4096 take 32 us, of which the masses and the first digit 9.7, the other digits 7 to 10, the
// positions 8, their masses 3; one of 64,106 cut to 24,377 67 us; one of 1003, 8 us, where every step waits for the one before it.  (Eight loads of a lane on their way, two more comparisons a position and the
// first digit counted by a pass of its own: 38 us.)
constexpr int EVICT_THREADS = 1024, EVICT_HELD = 32 * 1024;
template <bool HELD>
__global__ void __launch_bounds__(EVICT_THREADS) paged_evict_select_kernel(EvictArgs a) {
    extern __shared__ __attribute__((aligned(16))) unsigned held[];
    __shared__ CutLds cut;
    const PagedView &pv = a.pv;
    const int h = blockIdx.x % (unsigned)pv.n_kv, s = blockIdx.x / (unsigned)pv.n_kv, t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
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
    const int lo = a.first, hi = n - a.recent, want = a.keep - a.first - a.recent;
    constexpr unsigned STAYS = ~0u;                          // (no mass is that)
    const unsigned zero = order_of(0.f);
    auto number = [&](int i, float m) { return i >= lo && i < hi ? order_of(m) : STAYS; };
    constexpr int U = 16;                                    // of a lane, on their way at once
    auto counted = [&](const auto &key, auto f) {
        int zeros = 0;
        for (const unsigned k : key) {
            zeros += __popcll(__ballot(k == zero));
            if (k != zero && k != STAYS) f(k, 1);
        }
        if (lane == 0 && zeros) f(zero, zeros);
    };
    auto from_memory = [&](auto f) {
        int i0 = wave * 64 + lane;
        auto some = [&](auto each) {
            constexpr int N = decltype(each)::value;
            float m[N];
            unsigned key[N];
#pragma unroll
            for (int u = 0; u < N; u++) m[u] = mass[min(i0 + u * EVICT_THREADS, n - 1)];
#pragma unroll
            for (int u = 0; u < N; u++) {
                const int i = i0 + u * EVICT_THREADS;
                key[u] = number(i, m[u]);                     // (hi <= n: STAYS behind the last)
                if (HELD && i < n) held[i] = key[u];
            }
            counted(key, f);
            i0 += N * EVICT_THREADS;
        };
        while (i0 - lane + (U - 4) * EVICT_THREADS < n) some(std::integral_constant<int, U>());
        while (i0 - lane < n) some(std::integral_constant<int, 4>());
    };
    Cut<unsigned> c{STAYS - 1, ~0u, 0};
    for (int i = t; i < CUT_BINS; i += EVICT_THREADS) cut.bins[i] = 0;
    __syncthreads();
    from_memory([&](unsigned key, int times) { atomicAdd(&cut.bins[cut_bin(key >> (32 - CUT_BITS))], times); });
    __syncthreads();
    if (want > 0)
        c = cut_keys<EVICT_THREADS, true, unsigned>([&](auto f) {
            if constexpr (!HELD) from_memory(f);
            else
                for (int i0 = wave * 64 + lane; i0 - lane < n; i0 += 4 * EVICT_THREADS) {
                    unsigned key[4];
#pragma unroll
                    for (int u = 0; u < 4; u++) key[u] = i0 + u * EVICT_THREADS < n ? held[i0 + u * EVICT_THREADS] : STAYS;
                    counted(key, f);
                }
        }, want, 32, 0u, cut);
    auto put = [&](int place, int i) { kept[place] = i; };
    if constexpr (HELD) cut_numbers<EVICT_THREADS, 8>(n, c, [&](int i) { return held[i]; }, [](int, unsigned key) { return key; }, put, cut);
    else cut_numbers<EVICT_THREADS, U>(n, c, [&](int i) { return mass[i]; }, number, put, cut);
    for (int i0 = 0; i0 < a.keep; i0 += 8 * EVICT_THREADS) {
        __syncthreads();
        float m[8];
#pragma unroll
        for (int u = 0; u < 8; u++) {
            const int i = i0 + u * EVICT_THREADS + t;
            m[u] = i < a.keep ? mass[kept[i]] : 0.f;
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < 8; u++)
            if (i0 + u * EVICT_THREADS + t < a.keep) out[i0 + u * EVICT_THREADS + t] = m[u];
    }
}

// K and V of the kept positions to their places: 16 bytes a lane, four rows of one key head on their way at once.  Bound by memory: 16 x 8 x 4096 rows of 256 bytes (475 MB read and written, rows in any order) in 100 us,
// the rate of a large copy; in fp32 (931 MB) 201 us.
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
    return check_weights(cache, batch, mask, n_heads, &a) ? 0 : weight_bytes(a, plan_weights(a, cache->dtype == VLA_DTYPE_F32));
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
    const bool f32 = cache->dtype == VLA_DTYPE_F32;
    const WeightPlan p = plan_weights(a, f32);
    if (batch->n_rows > 0 && ws_bytes < weight_bytes(a, p)) { vla_set_error("paged_weights: workspace %zu bytes, need %zu", ws_bytes, weight_bytes(a, p)); return VLA_EWORKSPACE; }
    if (batch->n_rows == 0 || batch->max_rows == 0 || batch->max_len == 0) return VLA_OK;
    a.q = (const char *)q; a.q_stride = q_stride;
    a.aligned = ((uintptr_t)q | (size_t)q_stride * (f32 ? 4 : 2)) % 16 == 0 && q_stride < 1 << 24;          // (a tile's rows at 32-bit offsets from its first)
    a.offset = !f32 ? a.cap * LOG2E : 0.f;
    w.lse_in = lse; w.mass = mass; w.mass_stride = mass_stride; w.part = (float *)ws;
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps("paged_weights", 0.0, st);
    return f32 ? launch_weights_sized<float>(w, p, st) : launch_weights_sized<bf16_t>(w, p, st);
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
    const int row_bytes = cache->head_dim * (cache->dtype == VLA_DTYPE_F32 ? 4 : 2), chunks = row_bytes / 16, per = 256 / chunks * 4;
    if ((least + per - 1) / per > 0x7fffffff / 256) { vla_set_error("paged_evict: keep %d is too many", keep); return VLA_ESHAPE; }
    // every workgroup of a sequence reads kv_len while the first writes new_len
    if (paged_overlap(new_len, (size_t)batch->n_seq * 4, batch->kv_len, (size_t)batch->n_seq * 4) ||
        (mass != mass_out && paged_overlap(mass, pairs * mass_stride * 4, mass_out, pairs * mass_out_stride * 4))) {
        vla_set_error("paged_evict: new_len overlaps kv_len, or mass_out a part of mass");
        return VLA_EINVAL;
    }
    a.mass = mass; a.mass_out = mass_out; a.mass_stride = mass_stride; a.out_stride = mass_out_stride;
    a.keep = keep; a.first = first; a.recent = recent; a.to_table = to_table; a.to_stride = to_stride; a.kept = kept; a.new_len = new_len;
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps("paged_evict", 0.0, st);
    if (batch->max_len <= EVICT_HELD) {
        if (int rc = vla_allow_lds((const void *)paged_evict_select_kernel<true>, EVICT_HELD * sizeof(float))) return rc;
        paged_evict_select_kernel<true><<<(unsigned)pairs, EVICT_THREADS, batch->max_len * sizeof(float), st>>>(a);
    } else paged_evict_select_kernel<false><<<(unsigned)pairs, EVICT_THREADS, 0, st>>>(a);
    if (int rc = vla_check_launch("paged_evict")) return rc;
    if (least == 0) return VLA_OK;
    paged_evict_move_kernel<4><<<dim3((least + per - 1) / per, (unsigned)pairs), 256, 0, st>>>(a, chunks, row_bytes);
    return vla_check_launch("paged_evict move");
}

}  // extern "C"
