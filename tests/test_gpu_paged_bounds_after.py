"""Bounds of pages whose keys have moved: behind an accepted tree and behind an eviction, computed again as include/vla.h says.  Whole values of K: equal."""
import numpy as np
import pytest
import torch

from paged_less_ref import page_bounds, pools_of, random_tree, to_device
from paged_ref import DEV, TYPES, Batch
from paper_2510_06710_amd import binding as vb
from test_gpu_paged_sparse import selected_by

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("dtype", ["bf16", "f32"])
KV, D = 2, 64


def bounds_of(b, k):
    """Of all pages that hold positions; -77 elsewhere."""
    want = np.full((b.n_pages, KV, 2, D), -77.0)
    for s, (_, length) in enumerate(b.spec):
        for number in range(-(-length // b.page)):
            want[b.table[s, number]] = page_bounds(b, k, s, number).transpose(1, 0, 2)
    return want


@BOTH
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("spec", [[(40, 50)], [(33, 48), (1, 17), (0, 20), (70, 100), (64, 64), (9, 25)]])
def test_behind_an_accepted_tree(dtype, page, spec):
    b, rng, I = Batch(spec, page, padding=2), np.random.default_rng(page), torch.int32
    k, v = (p.to(DEV) for p in pools_of(b, dtype, KV, D, 1))
    cache, batch = vb.make_paged_cache(k, v), b.on_device()
    bounds = torch.full((b.n_pages, KV, 2, D), -77.0, dtype=TYPES[dtype], device=DEV)
    whole = Batch([(l, l) for _, l in spec], page)
    whole.table, whole.n_pages = b.table, b.n_pages
    vb.vla_paged_bounds(cache, whole.on_device(), bounds)
    # drafts that are all different, accepted down to the last node
    parents = [random_tree(n, rng) if n else [] for n, _ in spec]
    ids, chosen = np.arange(b.n_rows, dtype=np.int32), np.full(b.n_rows, -1, np.int32)
    for s, tree in enumerate(parents):
        node = len(tree) - 1
        while node > 0:
            chosen[b.start[s] + tree[node]] = ids[b.start[s] + node]
            node = tree[node]
    n = len(spec)
    path, count, new_len = (torch.zeros(*shape, dtype=I, device=DEV) for shape in ((n, b.max_rows), (n,), (n,)))
    parent = np.array([p for t in parents for p in t] + [0] * 2, np.int32)
    vb.vla_paged_accept(cache, 1, 0, batch, *map(to_device, (parent, ids, chosen)), path, count, None, new_len)
    # the accepted rows behind the new lengths: nothing of them is read on the host
    start = torch.cat([torch.zeros(1, dtype=I, device=DEV), count.cumsum(0).to(I)])
    vb.vla_paged_bounds(cache, vb.make_paged_batch(start, new_len, to_device(b.table), b.n_rows, b.max_rows, b.max_len), bounds)
    after = Batch([(1, int(l)) for l in new_len.tolist()], page)
    after.table, after.n_pages = b.table, b.n_pages
    assert any(l < old for (_, old), (_, l) in zip(spec, after.spec))
    want, got = bounds_of(after, k.double().cpu().numpy()), bounds.double().cpu().numpy()
    held = (want != -77).all((1, 2, 3))                       # (pages that only rejected drafts lie on keep what they had)
    assert np.array_equal(got[held], want[held])
    # and what the next tokens select by them
    q = torch.randn(n, 4, D, generator=torch.Generator().manual_seed(4)).to(TYPES[dtype])
    tokens = after.on_device()
    for most in (1, 2, 4):
        selected = torch.full((n, KV, most), -77, dtype=I, device=DEV)
        vb.vla_paged_select(cache, tokens, bounds, q.to(DEV), selected, 0, 1, torch.empty(vb.vla_paged_select_workspace_bytes(cache, tokens), dtype=torch.uint8, device=DEV))
        assert np.array_equal(selected.cpu().numpy(), selected_by(after, q.double().numpy(), want, most, 0, 1))


@BOTH
def test_behind_an_eviction(dtype):
    b, keep, n = Batch([(0, 200), (0, 20), (0, 97)], 16), 40, 3
    k, v = (p.to(DEV) for p in pools_of(b, dtype, KV, D, 2))
    extra = n * 3
    k, v = (torch.cat([p, torch.zeros(extra, *p.shape[1:], dtype=p.dtype, device=DEV)]) for p in (k, v))
    cache = vb.make_paged_cache(k, v)
    to_table = (b.n_pages + np.arange(extra)).reshape(n, 3).astype(np.int32)
    mass = torch.rand(n, KV, b.max_len, generator=torch.Generator().manual_seed(3)).to(DEV)
    kept, new_len = torch.zeros(n, KV, keep, dtype=torch.int32, device=DEV), torch.zeros(n, dtype=torch.int32, device=DEV)
    vb.vla_paged_evict(cache, b.on_device(), mass, 2, 5, to_device(to_table), kept, mass, new_len)
    # every position of the new pages as a row: numbers that the host knows bound them
    bounds = torch.full((b.n_pages + extra, KV, 2, D), -77.0, dtype=TYPES[dtype], device=DEV)
    start = torch.cat([torch.zeros(1, dtype=torch.int32, device=DEV), new_len.cumsum(0).to(torch.int32)])
    vb.vla_paged_bounds(cache, vb.make_paged_batch(start, new_len, to_device(to_table), n * keep, keep, keep), bounds)
    after = Batch([(0, int(l)) for l in new_len.tolist()], 16)
    after.table, after.n_pages = to_table, b.n_pages + extra
    assert np.array_equal(bounds.double().cpu().numpy(), bounds_of(after, k.double().cpu().numpy()))
