// The largest of many keys by one workgroup: where they are cut off, and their numbers in order.
//
// A key's digits of eleven bits are counted in LDS from the top until the keys that share the cut's digits are all taken or no digit is left; which of the last ones
// stay is decided by their order, lowest number first.  Numbers are written by waves that each hold a run of them: what a wave takes is counted first, and placed behind what the waves before it took.
#pragma once
#include "vla_internal.h"

constexpr int CUT_BITS = 11, CUT_BINS = 1 << CUT_BITS;
struct CutLds { int bins[CUT_BINS], wave[16], digit, want, count; };

// Sum over the threads before this one; *all: over all.
template <int THREADS> __device__ __forceinline__ int cut_scan(int v, int *all, int *wave_sums) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int in = v;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int x = __shfl_up(in, o, 64); if (lane >= o) in += x; }
    if (lane == 63) wave_sums[wave] = in;
    __syncthreads();
    int before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < THREADS / 64; w++) { if (w < wave) before += wave_sums[w]; total += wave_sums[w]; }
    *all = total;
    return before + in - v;
}

// Taken are keys with (key & mask) > prefix, and of those with (key & mask) == prefix the first `want`.
template <typename Key> struct Cut { Key prefix, mask; int want; };

// The bin of a digit: largest first.
__device__ __forceinline__ int cut_bin(int digit) { return CUT_BINS - 1 - digit; }

// The cut that leaves `want` (at least 1, at most as many as there are) of the keys that each(f) gives f, every thread its own, with how often they occur.  top: the bits above it are the same in all of them, those of `same`.
// COUNTED: the first digit's bins are filled already, behind a barrier.
template <int THREADS, bool COUNTED, typename Key, typename Each>
__device__ __forceinline__ Cut<Key> cut_keys(Each each, int want, int top, Key same, CutLds &s) {
    constexpr int EACH = CUT_BINS / THREADS;
    Cut<Key> c;
    c.mask = top >= (int)sizeof(Key) * 8 ? 0 : ~(Key)0 << top;
    c.prefix = same & c.mask;
    c.want = want;
    for (bool counted = COUNTED; top > 0; counted = false) {
        const int shift = top > CUT_BITS ? top - CUT_BITS : 0, bits = top - shift;
        if (!counted) {
            for (int i = threadIdx.x; i < CUT_BINS; i += THREADS) s.bins[i] = 0;
            __syncthreads();
            each([&](Key key, int times) {
                if ((key & c.mask) == c.prefix) atomicAdd(&s.bins[cut_bin((int)(key >> shift & (((Key)1 << bits) - 1)))], times);
            });
            __syncthreads();
        }
        // the digit at which the count from above reaches `want` (bins lie largest digit first)
        int here[EACH], sum = 0, all;
#pragma unroll
        for (int e = 0; e < EACH; e++) sum += here[e] = s.bins[threadIdx.x * EACH + e];
        int above = cut_scan<THREADS>(sum, &all, s.wave);
#pragma unroll
        for (int e = 0; e < EACH; e++) {
            if (above < c.want && above + here[e] >= c.want) {
                s.digit = CUT_BINS - 1 - ((int)threadIdx.x * EACH + e);
                s.want = c.want - above;
                s.count = here[e];
            }
            above += here[e];
        }
        __syncthreads();
        c.want = s.want;
        c.prefix |= (Key)s.digit << shift;
        c.mask |= (((Key)1 << bits) - 1) << shift;
        top = shift;
        if (s.count == c.want) break;                        // (all that share these digits are taken)
        __syncthreads();
    }
    return c;
}

// Of numbers 0 .. n - 1 those that the cut takes: put(place, i) for each, in order.  key(i, load(i)): their keys; ~0 is taken always.  U: of a lane at once.
// (Of every other key one of the highest CUT_BITS bits is zero.  A cut's mask has these at least, so its prefix is not all ones there, and ~0 lies above it.)
template <int THREADS, int U, typename Key, typename Load, typename KeyOf, typename Put>
__device__ __forceinline__ void cut_numbers(int n, const Cut<Key> &c, Load load, KeyOf key, Put put, CutLds &s) {
    constexpr int WAVES = THREADS / 64;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int run = (n + 64 * WAVES - 1) / (64 * WAVES) * 64, i0 = min(wave * run, n), i1 = min(i0 + run, n);
    // f(u, taken for sure, equal to the cut) of the 64 numbers from i + 64 u on
    auto block = [&](int i, auto f) {
        decltype(load(0)) x[U];
        if (i + 64 * U <= i1) {
#pragma unroll
            for (int u = 0; u < U; u++) x[u] = load(i + u * 64 + lane);
#pragma unroll
            for (int u = 0; u < U; u++) {
                const Key k = key(i + u * 64 + lane, x[u]) & c.mask;
                f(u, __ballot(k > c.prefix), __ballot(k == c.prefix));
            }
        } else {
#pragma unroll
            for (int u = 0; u < U; u++) x[u] = load(min(i + u * 64 + lane, n - 1));
#pragma unroll
            for (int u = 0; u < U; u++)
                if (i + u * 64 < i1) {
                    const int j = i + u * 64 + lane;
                    const Key k = key(j, x[u]) & c.mask;
                    f(u, __ballot((j < i1) & (k > c.prefix)), __ballot((j < i1) & (k == c.prefix)));
                }
        }
    };
    int sures = 0, ties = 0;
    for (int i = i0; i < i1; i += 64 * U)
        block(i, [&](int, unsigned long long a, unsigned long long b) { sures += __popcll(a); ties += __popcll(b); });
    __syncthreads();
    if (lane == 0) { s.bins[wave] = sures; s.bins[16 + wave] = ties; }
    __syncthreads();
    int place = 0, left = c.want;                            // of those equal to the cut, how many are taken from here on
    for (int w = 0; w < wave; w++) { place += s.bins[w]; left -= s.bins[16 + w]; }
    place = __builtin_amdgcn_readfirstlane(place + c.want - max(left, 0));
    left = __builtin_amdgcn_readfirstlane(max(left, 0));
    const unsigned long long below = (1ull << lane) - 1;
    for (int i = i0; i < i1; i += 64 * U)
        block(i, [&](int u, unsigned long long a, unsigned long long b) {
            if (left > 0 && b) {
                a |= __ballot((b >> lane & 1) & (__popcll(b & below) < left));
                left -= __popcll(b);
            }
            if (a) {
                if (a >> lane & 1) put(place + __popcll(a & below), i + u * 64 + lane);
                place += __popcll(a);
            }
        });
}
