// What the kernels of the paged KV cache (paged_*.hip) share: the cache and the ragged batch as
// they are handed to a kernel, and the checks of both on the host.
#pragma once
#include "vla_internal.h"

struct PagedView {
    char *k, *v;                 // [n_pages][n_kv][page][d]
    int n_pages, page_log, n_kv, d;
    int n_seq, n_rows, max_rows, max_len, table_stride;
    const int32_t *row_start, *kv_len, *table;
};

// Host: 0 or an error code with the message set.  `what` names the entry point.
int vla_check_paged(const char *what, const vla_paged_cache *cache, const vla_paged_batch *batch, PagedView *out);
// Whether two arrays share a byte (NULL: no).
inline bool paged_overlap(const void *a, size_t a_bytes, const void *b, size_t b_bytes) {
    return a && b && (uintptr_t)a < (uintptr_t)b + b_bytes && (uintptr_t)b < (uintptr_t)a + a_bytes;
}

// Rows of a ragged batch as the decoder takes and gives them (vla_forward_paged).
template <typename T>
int launch_paged_embed(float *X, const int32_t *ids, const T *patch, int n_patch, const T *embed, int n_rows, int H, int vocab, hipStream_t st);
int launch_paged_last_rows(float *out, const float *X, const int32_t *row_start, int n_seq, int n_rows, int H, hipStream_t st);
int launch_rotary_freq(double *freq, int d, float theta, hipStream_t st);

// The batch's arrays do not change while a kernel runs: read as constants, uniform indexes through the scalar cache (behind the
// kernels' assembler text the compiler would otherwise take vector loads, and wait for everything in flight).
typedef const __attribute__((address_space(4))) int32_t *const_ints;
__device__ __forceinline__ int paged_int(const int32_t *p, size_t i) { return ((const_ints)p)[i]; }

// A sequence's rows as the device arrays have them, within the batch's bounds whatever they hold.
struct PagedSeq {
    int r0, n;         // first row; rows, all of them
    int rows;          // ... that the call takes
    int len, keys;     // positions held; ... that it reads
};
__device__ __forceinline__ PagedSeq paged_seq(const PagedView &p, int s) {
    PagedSeq q;
    q.r0 = min(max(paged_int(p.row_start, s), 0), p.n_rows);
    q.n = min(max(paged_int(p.row_start, s + 1), q.r0), p.n_rows) - q.r0;
    q.rows = min(q.n, p.max_rows);
    q.len = max(paged_int(p.kv_len, s), 0);
    q.keys = min(q.len, p.max_len);
    return q;
}

// The sequence of a row (n_seq: padding), by all 64 lanes of a wave: how many of row_start[1 ..] lie at or before it.  Where sequences have one row each, as in a decode step, it is the row's
// own number: two words to look at.
__device__ __forceinline__ int paged_seq_of_row(const PagedView &p, int row) {
    const int guess = min(row, p.n_seq - 1);
    if (paged_int(p.row_start, guess) <= row && paged_int(p.row_start, guess + 1) > row) return guess;
    int n = 0;
    for (int s = threadIdx.x & 63; s < p.n_seq; s += 64) n += paged_int(p.row_start, s + 1) <= row;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) n += __shfl_xor(n, o, 64);
    return __builtin_amdgcn_readfirstlane(n);
}
