// Trees of drafted tokens behind a paged cache: what each node sees, and the path that the model's own tokens follow, with its K and V.
//
// A node's ancestors have smaller numbers, so a walk up from it meets them in descending order: the words of its row of bits are finished
// one after the other, last first, by one thread.  Both kernels are chains of dependent reads of a few hundred bytes; the parents of a
// sequence are read to LDS once, where a step of a walk costs a quarter of a microsecond at most and not a trip to memory.  Nothing is rounded: whole numbers and moved bits.
#include "paged.h"

namespace {

// The parent of node i: below 0 for none.
__device__ __forceinline__ int parent_of(const int32_t *parent, int i) { return parent[i] < i ? parent[i] : -1; }

// A thread a node.  In a captured graph 8 nodes take 1.8 us, 32 sequences of 24 2.7; of 1024 nodes whose paths are up to some 400 long 111 us, for one sequence as for 64 (8.9 MB, 2 us at the
// copy's rate): the longest walk, a quarter of a microsecond a node.
__global__ void __launch_bounds__(256) paged_tree_kernel(PagedView pv, const int32_t *parent, int32_t *seen, int words, int32_t *position) {
    __shared__ int32_t up[VLA_TREE_ROWS];
    const PagedSeq sq = paged_seq(pv, blockIdx.x);
    for (int i = threadIdx.x; i < sq.rows; i += 256) up[i] = parent[sq.r0 + i];
    __syncthreads();
    for (int i = threadIdx.x; i < sq.rows; i += 256) {
        int32_t *row = seen + (size_t)(sq.r0 + i) * words;
        int w = words - 1, depth = 0;
        unsigned bits = 0;
        for (int node = i; node >= 0; node = parent_of(up, node)) {
            for (; w > node >> 5; w--) { row[w] = (int32_t)bits; bits = 0; }
            bits |= 1u << (node & 31);
            depth++;
        }
        for (; w >= 0; w--) { row[w] = (int32_t)bits; bits = 0; }
        if (position) position[sq.r0 + i] = sq.len - sq.n + depth - 1;
    }
}

// A workgroup for each sequence and run of (layer, key head) pairs of K or V; all of them follow the path (one wave, 64 nodes at a time), the first
// writes it.  Of a path's rows only those move that leave their place.  A lane moves the same 16 bytes of every row, so what it writes
// (place i) it has read before: sources ascend and lie behind their targets.  Eight rows are on their way at once.  One sequence of 8 nodes in 32 layers of 8 heads: 4.8 us, the
// chain of the look-ups and the path; 64 sequences of up to 33 nodes, 16 layers of 32 heads: 44 us for 130 MB read and written, 2.9 TB/s (a copy: 4.75),
// where a lane stores the rows of one unit before it loads those of the next; in fp32 92 us for 259 MB, 2.8 TB/s.
struct AcceptArgs {
    PagedView pv;
    size_t layer_bytes;
    int units, per_block, es;          // pairs of a layer and a key head, of K and of V (2 layers n_kv); of one workgroup; bytes of an element
    const int32_t *parent, *ids, *chosen;
    int32_t *path, *n_accepted, *next, *new_len;
};
__global__ void __launch_bounds__(256) paged_accept_kernel(AcceptArgs a) {
    extern __shared__ long places[];                         // [max_rows] from, to; then up, id, want, path
    __shared__ int found;
    const PagedView &pv = a.pv;
    long *from = places, *to = from + pv.max_rows;
    int32_t *up = (int32_t *)(to + pv.max_rows), *id = up + pv.max_rows, *want = id + pv.max_rows, *path = want + pv.max_rows;
    const int s = blockIdx.x, t = threadIdx.x;
    const PagedSeq sq = paged_seq(pv, s);
    for (int i = t; i < sq.rows; i += 256) {
        up[i] = a.parent[sq.r0 + i];
        id[i] = a.ids[sq.r0 + i];
        want[i] = a.chosen[sq.r0 + i];
    }
    __syncthreads();
    if (t < 64) {
        int cur = sq.rows > 0 ? 0 : -1, n = 0;
        while (cur >= 0) {
            if (t == 0) path[n] = cur;
            n++;
            const int token = want[cur];
            int child = -1;
            for (int i0 = cur + 1; token >= 0 && child < 0 && i0 < sq.rows; i0 += 64) {
                const int i = i0 + t;
                const unsigned long long hit = __ballot(i < sq.rows && up[i] == cur && id[i] == token);
                if (hit) child = i0 + __builtin_ctzll(hit);
            }
            cur = child;
        }
        if (t == 0) found = n;
    }
    __syncthreads();
    const int n = found, base = sq.len - sq.n;
    if (blockIdx.y == 0) {
        for (int i = t; i < pv.max_rows; i += 256) a.path[(size_t)s * pv.max_rows + i] = i < n ? path[i] : -1;
        if (t == 0) {
            a.n_accepted[s] = n;
            if (a.next) a.next[s] = n > 0 ? want[path[n - 1]] : -1;
            if (a.new_len) a.new_len[s] = max(base + n, 0);
        }
    }
    int first = 0;                                            // rows before it stay where they are
    while (first < n && path[first] == first) first++;
    if (first == n) return;
    // where the rows that move are, and go: bytes within a key head's pages; below 0: nowhere
    const int32_t *table = pv.table + (size_t)s * pv.table_stride;
    const int row_bytes = pv.d * a.es, chunks = row_bytes / 16;
    auto at = [&](int pos) -> long {
        if (pos < 0 || pos >= pv.max_len) return -1;
        const int page = table[pos >> pv.page_log];
        if ((unsigned)page >= (unsigned)pv.n_pages) return -1;
        return (((long)page * pv.n_kv << pv.page_log) + (pos & ((1 << pv.page_log) - 1))) * row_bytes;
    };
    for (int i = first + t; i < n; i += 256) {
        from[i] = at(base + path[i]);
        to[i] = at(base + i);
    }
    __syncthreads();
    const int u0 = blockIdx.y * a.per_block, u1 = min(u0 + a.per_block, a.units);
    for (int x = u0 * chunks + t; x < u1 * chunks; x += 256) {
        const int unit = x / chunks, c = x - unit * chunks, pair = unit >> 1;
        char *rows = (unit & 1 ? pv.v : pv.k) + (size_t)(pair / pv.n_kv) * a.layer_bytes + ((size_t)(pair % pv.n_kv) << pv.page_log) * row_bytes + c * 16;
        for (int i0 = first; i0 < n; i0 += 8) {
            i32x4_v v[8];
#pragma unroll
            for (int j = 0; j < 8; j++) {
                const long src = i0 + j < n ? from[i0 + j] : -1;
                v[j] = src < 0 ? i32x4_v{0, 0, 0, 0} : *(const i32x4_v *)(rows + src);
            }
#pragma unroll
            for (int j = 0; j < 8; j++)
                if (i0 + j < n && to[i0 + j] >= 0) *(i32x4_v *)(rows + to[i0 + j]) = v[j];
        }
    }
}

int check_trees(const char *what, const PagedView &pv) {
    if (pv.max_rows > VLA_TREE_ROWS) { vla_set_error("%s: trees of up to %d rows (at most %d)", what, pv.max_rows, VLA_TREE_ROWS); return VLA_ESHAPE; }
    return VLA_OK;
}

}  // namespace

extern "C" {

int vla_paged_tree(const vla_paged_cache *cache, const vla_paged_batch *batch, const int32_t *parent, int32_t *seen, int words, int32_t *position,
                   void *stream) {
    PagedView pv;
    if (int rc = vla_check_paged("paged_tree", cache, batch, &pv)) return rc;
    if (int rc = check_trees("paged_tree", pv)) return rc;
    if (words < 1 || words > VLA_TREE_ROWS / 32 || words * 32 < pv.max_rows) {
        vla_set_error("paged_tree: %d words for trees of up to %d rows", words, pv.max_rows);
        return VLA_ESHAPE;
    }
    if (pv.n_rows > 0 && (!parent || !seen)) { vla_set_error("paged_tree: parent or seen is NULL"); return VLA_EINVAL; }
    if (pv.n_rows == 0 || pv.max_rows == 0) return VLA_OK;
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps("paged_tree", 4.0 * pv.n_rows * (words + 2), st);
    paged_tree_kernel<<<pv.n_seq, 256, 0, st>>>(pv, parent, seen, words, position);
    return vla_check_launch("paged_tree");
}

int vla_paged_accept(const vla_paged_cache *cache, int n_layers, size_t layer_stride, const vla_paged_batch *batch, const int32_t *parent,
                     const int32_t *ids, const int32_t *chosen, int32_t *path, int32_t *n_accepted, int32_t *next, int32_t *new_len,
                     void *stream) {
    AcceptArgs a{};
    if (int rc = vla_check_paged("paged_accept", cache, batch, &a.pv)) return rc;
    if (int rc = check_trees("paged_accept", a.pv)) return rc;
    const size_t layer = (size_t)cache->n_pages * cache->n_kv_heads * cache->page_size * cache->head_dim;
    a.es = cache->dtype == VLA_DTYPE_F32 ? 4 : 2;
    if (n_layers < 0 || n_layers > 65536) { vla_set_error("paged_accept: n_layers %d unsupported (0 .. 65,536)", n_layers); return VLA_EINVAL; }
    if ((long)n_layers * cache->n_kv_heads > 1 << 20) { vla_set_error("paged_accept: %d layers of %d key heads are too many", n_layers, cache->n_kv_heads); return VLA_ESHAPE; }
    if (n_layers > 1 && layer_stride < layer) { vla_set_error("paged_accept: layer stride of %zu elements, a layer has %zu", layer_stride, layer); return VLA_ESHAPE; }
    if (n_layers > 1 && layer_stride * a.es % 16) { vla_set_error("paged_accept: the layers are not 16-byte aligned"); return VLA_EINVAL; }
    if (!n_accepted || (batch->max_rows > 0 && !path)) { vla_set_error("paged_accept: path or n_accepted is NULL"); return VLA_EINVAL; }
    if (batch->n_rows > 0 && (!parent || !ids || !chosen)) { vla_set_error("paged_accept: parent, ids or chosen is NULL"); return VLA_EINVAL; }
    // every workgroup of a sequence reads these while the first writes
    const size_t rows = (size_t)batch->n_rows * 4, seqs = (size_t)batch->n_seq * 4;
    const struct { const void *at; size_t bytes; } in[] = {{parent, rows}, {ids, rows}, {chosen, rows}, {batch->kv_len, seqs}, {batch->row_start, seqs + 4}},
                                                   out[] = {{path, seqs * batch->max_rows}, {n_accepted, seqs}, {next, seqs}, {new_len, seqs}};
    for (auto &x : in)
        for (auto &y : out)
            if (paged_overlap(x.at, x.bytes, y.at, y.bytes)) { vla_set_error("paged_accept: an output overlaps an input"); return VLA_EINVAL; }
    a.layer_bytes = layer_stride * a.es;
    a.parent = parent; a.ids = ids; a.chosen = chosen; a.path = path; a.n_accepted = n_accepted; a.next = next; a.new_len = new_len;
    a.units = 2 * n_layers * a.pv.n_kv;
    // a workgroup's lanes each have 16 bytes of a row at a time; as many workgroups as stay on the chip at once (each walks the path again)
    const int chunks = a.pv.d * a.es / 16;
    const long all = (long)a.units * a.pv.n_seq;
    a.per_block = chunks < 256 ? 256 / chunks : 1;
    while (all > 2048L * a.per_block || a.units > 65535L * a.per_block) a.per_block *= 2;
    hipStream_t st = (hipStream_t)stream;
    ProfScope ps("paged_accept", 0.0, st);
    paged_accept_kernel<<<dim3(a.pv.n_seq, a.units > 0 ? (a.units + a.per_block - 1) / a.per_block : 1), 256, a.pv.max_rows * 32, st>>>(a);
    return vla_check_launch("paged_accept");
}

}  // extern "C"
