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
//
// Drafted trees (TREE) differ in what is seen alone: all below the sequence's new rows, and of these the ones whose bits are set, a word or two of them for a tile of 32 keys.  Their weights keep
// the tail in both forms.  8 nodes behind 700 positions, 32 heads, 11.5 us and 4.3 for the join; 61 behind 32,768, 16 heads, capped, 44 and 8.5; 32 sequences of up to 24 nodes behind up to 4096,
// 280 MB, 91 and 7, where the longest sequence's workgroups end 45 us behind the average.  The same in fp32: 17.7 and 4.3, 191 and 6.7, 560 (25 TFLOP/s of the card's 153, in tiles of 128 packed rows
// of which 4 to 96 are there).
#include "paged_rows.h"

namespace {

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
    it->hi = a.seen ? it->sq.keys : min(it->sq.keys, max(p0 + i1 + 1, prefix));          // (a tree's nodes are seen in any order)
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
    if constexpr (MODE & TREE) q.words = 0;                  // (no new row lies there: what a tile of 32 holds behind an odd multiple of 16 is the prefix's last key again)
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
        // (a tree's packed rows may be few: a wave without any loads its share of the tiles, and leaves the matrix pipe to the others)
        const bool idle = (MODE & TREE) && !__any(y.valid);
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
            if (idle) return ++t < t1;
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
    a->window = mask_window(*mask); a->shared_len = mask->shared_len;
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
    constexpr bool BF16 = sizeof(T) == 2, TAILS = BF16 && (MODE & TREE) != 0;          // (trees are few rows that wait for memory, like single tokens)
    if (a.shared_len > 0 && (rc = p.decode ? launch_prompt<T, DP, MODE, BF16>(a, p.whole, true, 1, st) : launch_prompt<T, DP, MODE, TAILS>(a, p.whole, true, p.own.parts, st))) return rc;
    if (p.decode) {
        constexpr size_t bytes = 2 * 2 * 32 * Tile<T, DP>::ROW;
        if ((rc = vla_allow_lds((const void *)paged_decode_kernel<T, DP, MODE>, bytes))) return rc;
        paged_decode_kernel<T, DP, MODE><<<(p.waves ? p.waves : a.pv.n_seq) * a.pv.n_kv, 64, bytes, st>>>(a);
        rc = vla_check_launch("paged_attention");
    } else rc = launch_prompt<T, DP, MODE, TAILS>(a, p.own, false, 0, st);
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
    if (a.seen) return a.cap > 0.f ? launch_sized<T, CAPPED | TREE>(a, p, st) : launch_sized<T, TREE>(a, p, st);
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

// The call itself; `seen`: drafted trees (a->seen and a->words are there already).
static int attend(AttnArgs &a, const vla_paged_cache *cache, const vla_paged_batch *batch, const void *q, int n_heads, int64_t q_stride, void *out,
                  int64_t out_stride, float *lse, void *ws, size_t ws_bytes, void *stream) {
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
    ProfScope ps(a.seen ? "paged_tree_attention" : "paged_attention", 0.0, st);               // (how much there is to do stands in arrays of the device)
    return f32 ? launch_typed<float>(a, p, st) : launch_typed<bf16_t>(a, p, st);
}

int vla_paged_attention(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_paged_mask *mask, const void *q, int n_heads,
                        int64_t q_stride, void *out, int64_t out_stride, float *lse, void *ws, size_t ws_bytes, void *stream) {
    AttnArgs a{};
    if (int rc = check(cache, batch, mask, n_heads, &a)) return rc;
    return attend(a, cache, batch, q, n_heads, q_stride, out, out_stride, lse, ws, ws_bytes, stream);
}

int vla_paged_tree_attention(const vla_paged_cache *cache, const vla_paged_batch *batch, const vla_paged_mask *mask, const int32_t *seen, int words,
                             const void *q, int n_heads, int64_t q_stride, void *out, int64_t out_stride, float *lse, void *ws, size_t ws_bytes, void *stream) {
    AttnArgs a{};
    if (int rc = check(cache, batch, mask, n_heads, &a)) return rc;
    if (mask->slopes || mask->prefix_len || mask->window) {
        vla_set_error("paged_tree_attention: a tree takes no slopes, prefix_len or window (its rows' distances are not those of their places)");
        return VLA_EINVAL;
    }
    if (batch->n_rows > 0 && !seen) { vla_set_error("paged_tree_attention: seen is NULL"); return VLA_EINVAL; }
    if (batch->max_rows > VLA_TREE_ROWS || words < 1 || words > VLA_TREE_ROWS / 32 || words * 32 < batch->max_rows) {
        vla_set_error("paged_tree_attention: trees of up to %d rows in %d words (at most %d rows, 32 to a word)", batch->max_rows, words, VLA_TREE_ROWS);
        return VLA_ESHAPE;
    }
    a.seen = seen; a.words = words;
    return attend(a, cache, batch, q, n_heads, q_stride, out, out_stride, lse, ws, ws_bytes, stream);
}

}  // extern "C"
