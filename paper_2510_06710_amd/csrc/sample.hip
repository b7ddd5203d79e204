// Sampling from rows of logits with temperature, top-k, top-p and min-p, from given random numbers.
//
// A token's place in the order "largest first, lowest id first among equals" is its rank; 64 bits hold (value, id) so that a
// larger number comes earlier.  Every cut keeps a leading run of that order, so the kept set is one threshold on that
// number.  Masses are w = exp((z - max) / T) in fp64, rounded to multiples of 2^-44 and summed as whole numbers: the sums are exact,
// in any order, and the border cases of top-p and of u fall alike every time (2^18 tokens of mass 1 stay below 2^63).
#include "vla_internal.h"

namespace {

constexpr int THREADS = 1024;
constexpr double UNIT = 17592186044416.0;      // 2^44

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
__device__ __forceinline__ unsigned long long rank_key(unsigned order, int id) { return (unsigned long long)order << 32 | (unsigned)~id; }

__device__ __forceinline__ unsigned long long wave_sum(unsigned long long v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ __forceinline__ unsigned long long wave_max(unsigned long long v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) { const unsigned long long w = __shfl_xor(v, o, 64); v = w > v ? w : v; }
    return v;
}
struct Both { unsigned long long count, mass; };
// Sums (or the maximum of `count`) over the workgroup, to all threads.
__device__ __forceinline__ Both block_both(Both v, bool largest, unsigned long long (*red)[THREADS / 64]) {
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

// One workgroup per row; each cut by bisection of the order's 50 bits, a pass over the row a bit.
template <typename T>
__global__ void __launch_bounds__(THREADS) sample_rows_kernel(SampleArgs a) {
    __shared__ unsigned long long red[2][THREADS / 64];
    __shared__ unsigned long long scan[THREADS];
    const int row = blockIdx.x, t = threadIdx.x, V = a.vocab;
    const T *z = (const T *)a.logits + row * a.stride;
    Both top{0, 0};
    for (int i = t; i < V; i += THREADS) {
        const unsigned o = order_of((float)z[i]);
        if (o) { const unsigned long long k = rank_key(o, i); top.count = k > top.count ? k : top.count; }
    }
    const unsigned long long first = block_both(top, true, red).count;
    if (first == 0) {
        if (t == 0) {
            a.token[row] = -1;
            if (a.logp) a.logp[row] = -INFINITY;
            if (a.logp_kept) a.logp_kept[row] = -INFINITY;
            if (a.n_kept) a.n_kept[row] = 0;
        }
        return;
    }
    const float zmax = value_of((unsigned)(first >> 32));
    const float T0 = a.temperature ? a.temperature[row] : 1.f;
    const bool greedy = !(T0 > 0.f) || !a.u;
    const double inv_t = T0 > 0.f ? (double)T0 : 1.0;
    const bool infinite = zmax == INFINITY;
    auto weight = [&](float v) { return infinite ? (v == INFINITY ? 1.0 : 0.0) : exp(((double)v - (double)zmax) / inv_t); };
    auto units = [&](float v) { return (unsigned long long)(weight(v) * UNIT + 0.5); };
    // count and mass of what lies at or above a threshold
    auto above = [&](unsigned long long least) {
        Both b{0, 0};
        for (int i = t; i < V; i += THREADS) {
            const float v = (float)z[i];
            const unsigned o = order_of(v);
            if (o && rank_key(o, i) >= least) { b.count++; b.mass += units(v); }
        }
        return block_both(b, false, red);
    };
    // the largest threshold that holds at least what `enough` asks for; below it nothing changes what was asked
    auto bisect = [&](auto enough) {
        unsigned long long lo = 1ull, hi = first;                    // enough(lo) by assumption
        while (lo < hi) {
            const unsigned long long mid = lo + (hi - lo + 1) / 2;
            if (enough(above(mid))) lo = mid; else hi = mid - 1;
        }
        return lo;
    };
    const Both all = above(1);
    unsigned long long cut = 1, leading = all.mass;
    if (infinite) cut = (unsigned long long)order_of(INFINITY) << 32;
    const int k = a.top_k ? a.top_k[row] : 0;
    if (k > 0 && (unsigned long long)k < all.count) {
        const unsigned long long c = bisect([&](Both b) { return b.count >= (unsigned long long)k; });
        cut = c > cut ? c : cut;
        leading = above(cut).mass;
    }
    const float p = a.top_p ? a.top_p[row] : 1.f;
    if (p < 1.f) {
        const double want = (double)(p > 0.f ? p : 0.f) * (double)leading;
        const unsigned long long c = bisect([&](Both b) { return (double)b.mass >= want; });
        cut = c > cut ? c : cut;
    }
    const float least = a.min_p ? a.min_p[row] : 0.f;
    auto kept = [&](float v, int i) {
        const unsigned o = order_of(v);
        if (!o) return false;
        const unsigned long long key = rank_key(o, i);
        return key == first || (key >= cut && weight(v) >= (double)least);
    };
    // ids in runs of consecutive ones per thread: running masses in id order
    const int per = (V + THREADS - 1) / THREADS, i0 = t * per, i1 = min(V, i0 + per);
    Both mine{0, 0};
    for (int i = i0; i < i1; i++) {
        const float v = (float)z[i];
        if (kept(v, i)) { mine.count++; mine.mass += units(v); }
    }
    const Both total = block_both(mine, false, red);
    scan[t] = mine.mass;
    __syncthreads();
    if (t == 0) {
        unsigned long long run = 0;
        for (int i = 0; i < THREADS; i++) { const unsigned long long x = scan[i]; scan[i] = run; run += x; }
    }
    __syncthreads();
    int token = (int)~(unsigned)first;
    if (!greedy) {
        const float u = a.u[row];
        const double want = (double)u * (double)total.mass;
        // the first id whose running mass exceeds `want`; the last kept one with mass should rounding leave none
        Both pick{0, 0};
        unsigned long long run = scan[t];
        for (int i = i0; i < i1; i++) {
            const float v = (float)z[i];
            if (!kept(v, i)) continue;
            const unsigned long long w = units(v);
            const bool over = (double)(run + w) > want;
            if (w && ((over && !((double)run > want)) || (!over && run + w == total.mass))) pick.count = (unsigned)i + 1ull;
            run += w;
        }
        token = (int)block_both(pick, true, red).count - 1;
    }
    if (t == 0) {
        const float v = (float)z[token];
        const double y = infinite ? 0.0 : ((double)v - (double)zmax) / inv_t;
        a.token[row] = token;
        if (a.logp) a.logp[row] = (float)(y - log((double)all.mass / UNIT));
        if (a.logp_kept) a.logp_kept[row] = (float)(y - log((double)total.mass / UNIT));
        if (a.n_kept) a.n_kept[row] = (int)total.count;
    }
}

}  // namespace

extern "C" {

size_t vla_sample_logits_workspace_bytes(int n, int vocab) {
    if (n <= 0 || vocab <= 0 || vocab > 262144) { vla_set_error("sample_logits: n must be positive, vocab 1 .. 262,144"); return 0; }
    return 256;
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
    if (dtype == VLA_DTYPE_F32) sample_rows_kernel<float><<<n, THREADS, 0, st>>>(a);
    else sample_rows_kernel<bf16_t><<<n, THREADS, 0, st>>>(a);
    return vla_check_launch("sample_logits");
}

}  // extern "C"
