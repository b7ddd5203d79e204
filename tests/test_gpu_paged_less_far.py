"""Pages that begin beyond 2^32 bytes of their pool: the operators that read less per token give there what they give on the first pages, bit for bit."""
import pytest
import torch

from paged_ref import DEV
from paper_2510_06710_amd import binding as vb

pytestmark = pytest.mark.gpu
KV, PAGE, D, HEADS, NEAR = 8, 64, 128, 16, 12
FAR = 2 ** 32 // (KV * PAGE * D * 2) + 5                      # the first of the far pages


@pytest.mark.parametrize("rows", [1, 20])
def test_far_pages(rows):
    g, I = torch.Generator().manual_seed(1), torch.int32
    content = [torch.randn(NEAR, KV, PAGE, D, generator=g).bfloat16().to(DEV) for _ in range(2)]
    q = torch.randn(2 * rows, HEADS, D, generator=g).bfloat16().to(DEV)
    i32 = lambda x: torch.tensor(x, dtype=I, device=DEV)
    start, lens = i32([0, rows, 2 * rows]), i32([230, 170])
    parent, ids, chosen = i32([-1] + list(range(rows - 1)) + [-1] + [0] * (rows - 1)), i32([x % 3 for x in range(2 * rows)]), i32([(x + 1) % 3 for x in range(2 * rows)])
    results = []
    for first in (0, FAR):
        pools = [torch.zeros(first + NEAR, KV, PAGE, D, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
        for p, c in zip(pools, content):
            p[first:] = c
        cache, table, to = vb.make_paged_cache(*pools), i32([[3, 1, 5, 0], [4, 2, 7, -1]]), i32([[6, 8], [9, 10]])
        table, to = torch.where(table < 0, -1, table + first), to + first
        batch, mask = vb.make_paged_batch(start, lens, table, 2 * rows, rows, 240), vb.make_paged_mask(D ** -0.5)
        empty = lambda n: torch.empty(n, dtype=torch.uint8, device=DEV)
        z = lambda *shape, dtype=I: torch.zeros(*shape, dtype=dtype, device=DEV)
        bounds, selected, some, tree, lse = z(first + NEAR, KV, 2, D, dtype=torch.bfloat16), z(2 * rows, KV, 3), torch.zeros_like(q), torch.zeros_like(q), z(2 * rows, HEADS, dtype=torch.float32)
        seen, mass, kept, mass_out, path, count = z(2 * rows, 1), z(2, KV, 240, dtype=torch.float32), z(2, KV, 100), z(2, KV, 100, dtype=torch.float32), z(2, rows), z(2)
        whole = vb.make_paged_batch(i32([0, 230, 400]), lens, table, 400, 230, 240)
        vb.vla_paged_bounds(cache, whole, bounds)
        vb.vla_paged_select(cache, batch, bounds, q, selected, 1, 1, empty(vb.vla_paged_select_workspace_bytes(cache, batch)))
        vb.vla_paged_sparse_attention(cache, batch, mask, selected, q, some, None, empty(vb.vla_paged_sparse_attention_workspace_bytes(cache, batch, mask, HEADS, 3)))
        vb.vla_paged_tree(cache, batch, parent, seen)
        vb.vla_paged_tree_attention(cache, batch, mask, seen, q, tree, lse, empty(vb.vla_paged_attention_workspace_bytes(cache, batch, mask, HEADS)))
        vb.vla_paged_weights(cache, batch, mask, q, lse, mass, empty(vb.vla_paged_weights_workspace_bytes(cache, batch, mask, HEADS)))
        vb.vla_paged_evict(cache, batch, mass, 2, 9, to, kept, mass_out)
        vb.vla_paged_accept(cache, 1, 0, batch, parent, ids, chosen, path, count)
        torch.cuda.synchronize()
        results.append([x.clone() for x in (bounds[first:], selected, some, tree, seen, mass, kept, mass_out, path, count, pools[0][first:], pools[1][first:])])
        if first:
            assert not pools[0][:first].any() and not pools[1][:first].any() and not bounds[:first].any()
        del pools, bounds, cache, batch, whole
        torch.cuda.empty_cache()
    assert all(torch.equal(a, b) for a, b in zip(*results)) and results[0][9].min() >= 1 and not torch.equal(results[0][10], content[0])
