"""Bounds of pages, the pages that rows select by them, and the attention over lists of pages.

Bounds are values of K: equal.  Selections are whole numbers: equal to those of scores in fp64, whose ties and near ties are the same in any order of summation for bf16
(products of 16 bits, sums of a few hundred in 53) and do not occur among random fp32 ones.  The attention's tolerance is that of test_gpu_paged_attention.py with the weights' tail."""
import numpy as np
import pytest
import torch

from paged_less_ref import check_rows, choose, page_bounds, pools_of, rows_of, to_device
from paged_ref import DEV, TYPES, Batch
from paper_2510_06710_amd import binding as vb

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("dtype", ["bf16", "f32"])
SPEC = [(1, 1), (1, 16), (0, 9), (3, 40), (1, 200), (2, 17), (5, 5), (1, 333)]


@BOTH
@pytest.mark.parametrize("kv,d", [(1, 16), (2, 80), (8, 128), (3, 256)])
@pytest.mark.parametrize("page", [16, 64])
@pytest.mark.parametrize("whole", [False, True])
def test_bounds(dtype, kv, d, page, whole):
    b = Batch([(l if whole else n, l) for n, l in SPEC], page, padding=1)
    pools = pools_of(b, dtype, kv, d, 1)
    bounds = torch.full((b.n_pages, kv, 2, d), -77.0, dtype=TYPES[dtype], device=DEV)
    vb.vla_paged_bounds(vb.make_paged_cache(*[p.to(DEV) for p in pools]), b.on_device(), bounds)
    want = np.full((b.n_pages, kv, 2, d), -77.0)
    k = pools[0].double().numpy()
    for s, (n, length) in enumerate(b.spec):
        if n:
            for number in range((length - n) // page, -(-length // page)):
                want[b.table[s, number]] = page_bounds(b, k, s, number).transpose(1, 0, 2)
    assert np.array_equal(bounds.double().cpu().numpy(), want)


def selected_by(b, q, bounds, most, first, recent):
    n_heads, kv = q.shape[1], bounds.shape[1]
    group, want = n_heads // kv, np.full((b.n_rows, kv, most), -77)
    for row, s, p in b.rows():
        for h in range(kv):
            want[row, h] = -1
            if p >= 0:
                pages = bounds[b.table[s, :p // b.page + 1], h]
                x = q[row, h * group:(h + 1) * group, None]
                with np.errstate(invalid="ignore"):
                    score = np.maximum(x * pages[:, 0], x * pages[:, 1]).sum((0, 2))
                taken = choose(score, most, first, recent)
                want[row, h, :len(taken)] = taken
    return want


@BOTH
@pytest.mark.parametrize("heads,kv,d", [(1, 1, 16), (8, 2, 128), (7, 1, 80), (4, 4, 256)])
@pytest.mark.parametrize("most,first,recent", [(1, 0, 1), (3, 1, 2), (4, 0, 1), (9, 2, 3), (40, 1, 1)])
def test_select(dtype, heads, kv, d, most, first, recent):
    b = Batch(SPEC + [(2, 1), (1, 700)], 16, padding=2)
    g = torch.Generator().manual_seed(d)
    q = torch.randn(b.n_rows, heads, d, generator=g).to(TYPES[dtype])
    bounds = torch.randn(b.n_pages, kv, 2, d, generator=g).to(TYPES[dtype]).sort(2).values
    bounds[::3] = bounds[0]                                   # pages with equal scores
    qd = torch.zeros(b.n_rows, heads * d + 3, dtype=TYPES[dtype], device=DEV)[:, 1:1 + heads * d].unflatten(1, (heads, d))
    qd.copy_(q)
    selected = torch.full((b.n_rows, kv, most), -77, dtype=torch.int32, device=DEV)
    k = torch.zeros(b.n_pages, kv, 16, d, dtype=TYPES[dtype], device=DEV)
    cache, batch = vb.make_paged_cache(k, k), b.on_device()
    ws = torch.full((vb.vla_paged_select_workspace_bytes(cache, batch),), 255, dtype=torch.uint8, device=DEV)
    vb.vla_paged_select(cache, batch, bounds.to(DEV), qd, selected, first, recent, ws)
    assert np.array_equal(selected.cpu().numpy(), selected_by(b, q.double().numpy(), bounds.double().numpy(), most, first, recent))


def test_select_among_thousands_and_odd_scores():
    b = Batch([(1, 16 * 8192), (3, 50001)], 16)
    g = torch.Generator().manual_seed(1)
    q = torch.randn(b.n_rows, 2, 16, generator=g)
    bounds = torch.randn(b.n_pages, 1, 2, 16, generator=g).sort(2).values
    at = b.table[0, :8192]
    bounds[at[5]], bounds[at[7000]] = float("inf"), float("nan")
    bounds[at[100:3000]] = 0.0                                # thousands of equal ones
    k = torch.zeros(b.n_pages, 1, 16, 16, device=DEV)
    cache, batch = vb.make_paged_cache(k, k), b.on_device()
    ws = torch.empty(vb.vla_paged_select_workspace_bytes(cache, batch), dtype=torch.uint8, device=DEV)
    for most in (2, 64, 3000, 5500, 8191, 8192):
        selected = torch.full((b.n_rows, 1, most), -77, dtype=torch.int32, device=DEV)
        vb.vla_paged_select(cache, batch, bounds.to(DEV), q.to(DEV), selected, 1, 1, ws)
        assert np.array_equal(selected.cpu().numpy(), selected_by(b, q.double().numpy(), bounds.double().numpy(), most, 1, 1)), most


def lists_of(b, kv, most, rng):
    """Some ascending pages of each row, in lists of any length."""
    out = np.full((b.n_rows, kv, most), -1, np.int32)
    for row, _, p in b.rows():
        n = p // b.page + 1
        for h in range(kv):
            if p >= 0:
                some = np.sort(rng.permutation(n)[:rng.integers(0, min(n, most) + 1)])
                out[row, h, :len(some)] = some
    return out


def attend(b, dtype, heads, kv, d, lists, cap=0.0, layout="packed", seed=0, meant=None):
    pools = pools_of(b, dtype, kv, d, seed)
    q = torch.randn(b.n_rows, heads, d, generator=torch.Generator().manual_seed(seed + 1)).to(TYPES[dtype])
    qd, out = q.to(DEV), torch.full((b.n_rows, heads, d), -77.0, dtype=TYPES[dtype], device=DEV)
    if layout == "unaligned":
        qd = torch.zeros(b.n_rows, heads * d + 5, dtype=TYPES[dtype], device=DEV)[:, 3:3 + heads * d].unflatten(1, (heads, d))
        qd.copy_(q)
        out = torch.full((b.n_rows, heads * d + 7), -77.0, dtype=TYPES[dtype], device=DEV)[:, 1:1 + heads * d].unflatten(1, (heads, d))
    lse = torch.full((b.n_rows, heads), -77.0, device=DEV)
    cache, batch, mask = vb.make_paged_cache(*[p.to(DEV) for p in pools]), b.on_device(), vb.make_paged_mask(d ** -0.5, cap)
    ws = torch.full((vb.vla_paged_sparse_attention_workspace_bytes(cache, batch, mask, heads, lists.shape[2]),), 255, dtype=torch.uint8, device=DEV)
    vb.vla_paged_sparse_attention(cache, batch, mask, to_device(lists), qd, out, lse, ws)
    first = out.clone()
    vb.vla_paged_sparse_attention(cache, batch, mask, to_device(lists), qd, out, None, ws)
    assert torch.equal(first, out)
    meant = lists if meant is None else meant

    def seen_by(row, s, p, h):
        pages = [e for e in meant[row, h] if e >= 0]
        at = np.concatenate([np.arange(e * b.page, (e + 1) * b.page) for e in pages]) if pages else np.zeros(0, int)
        return at[(at <= p) & (at < b.spec[s][1])]

    want = rows_of(b, q.double().numpy(), *[p.double().numpy() for p in pools], d ** -0.5, cap, seen_by)
    check_rows(b, dtype, d, cap, out, lse, want, max(l for _, l in b.spec) or 1)
    return out


@BOTH
@pytest.mark.parametrize("heads,kv,d", [(4, 4, 64), (8, 1, 128), (6, 2, 80), (16, 8, 256), (40, 1, 32), (3, 3, 16)])
@pytest.mark.parametrize("page,most", [(16, 1), (16, 7), (64, 6), (128, 3)])
def test_attention(dtype, heads, kv, d, page, most):
    b = Batch(SPEC, page, padding=2)
    rng = np.random.default_rng(most)
    attend(b, dtype, heads, kv, d, lists_of(b, kv, most, rng))
    attend(b, dtype, heads, kv, d, lists_of(b, kv, most, rng), cap=3.0, layout="unaligned")


@BOTH
def test_long_lists_are_split(dtype):
    rng = np.random.default_rng(5)
    for spec, page, most in (([(1, 5000)], 16, 200), ([(2, 9000), (1, 130)], 64, 100), ([(1, 4000 + i) for i in range(5)], 32, 33)):
        b = Batch(spec, page)
        attend(b, dtype, 8, 2, 128, lists_of(b, 2, most, rng))


@BOTH
def test_odd_lists(dtype):
    b = Batch([(1, 100), (4, 3), (1, 61)], 16)                # (rows at negative positions: they see nothing)
    lists, meant = np.full((b.n_rows, 1, 6), -1, np.int32), np.full((b.n_rows, 1, 6), -1, np.int32)
    lists[0, 0], meant[0, 0] = [2, 2, 4, 1, 5, 6], [2, 4, 5, 6, -1, -1]           # given twice, or out of order: left out
    lists[1:5, 0] = [0, 1, 2, 3, 4, 5]
    meant[1:5, 0] = lists[1:5, 0]
    lists[5, 0], meant[5, 0] = [1, 3, 99, 2 ** 30, -5, 2], [1, 3, -1, -1, -1, -1]  # pages behind the row, and what comes after the end
    attend(b, dtype, 4, 1, 64, lists, meant=meant)


@BOTH
def test_all_pages_are_the_whole_attention(dtype):
    b = Batch(SPEC, 16)
    pools, q = pools_of(b, dtype, 2, 64, 3), torch.randn(b.n_rows, 4, 64, generator=torch.Generator().manual_seed(6)).to(TYPES[dtype]).to(DEV)
    cache, batch, mask = vb.make_paged_cache(*[p.to(DEV) for p in pools]), b.on_device(), vb.make_paged_mask(0.125)
    selected, bounds = torch.zeros(b.n_rows, 2, 21, dtype=torch.int32, device=DEV), torch.zeros(b.n_pages, 2, 2, 64, dtype=TYPES[dtype], device=DEV)
    empty = lambda n: torch.empty(n, dtype=torch.uint8, device=DEV)
    vb.vla_paged_bounds(cache, batch, bounds)
    vb.vla_paged_select(cache, batch, bounds, q, selected, 1, 1, empty(vb.vla_paged_select_workspace_bytes(cache, batch)))
    some, plain = torch.zeros_like(q), torch.zeros_like(q)
    vb.vla_paged_sparse_attention(cache, batch, mask, selected, q, some, None, empty(vb.vla_paged_sparse_attention_workspace_bytes(cache, batch, mask, 4, 21)))
    vb.vla_paged_attention(cache, batch, mask, q, plain, None, empty(vb.vla_paged_attention_workspace_bytes(cache, batch, mask, 4)))
    # both within half a step of the output (2^-8, |o| < 4.5) and the rest of the tolerance above
    assert (some.float() - plain.float()).abs().max().item() <= (2.5 * 2.0 ** -8 if dtype == "bf16" else 2.0 ** -18) * 4.5


@BOTH
def test_a_page_that_is_not_there_reads_as_zeros(dtype):
    b = Batch([(1, 100), (2, 90)], 16)
    pools, q = [p.to(DEV) for p in pools_of(b, dtype, 1, 64, 3)], torch.randn(b.n_rows, 2, 64, generator=torch.Generator().manual_seed(6)).to(TYPES[dtype]).to(DEV)
    lists, outs = to_device(np.tile(np.array([1, 3, 5], np.int32), (3, 1, 1))), []
    for bad in (False, True):
        for s, e in ((0, 3), (1, 5)):
            if bad:
                b.table[s, e] = -1 if s else b.n_pages
            else:
                for p in pools:
                    p[b.table[s, e]] = 0
        out = torch.zeros_like(q)
        cache, batch, mask = vb.make_paged_cache(*pools), b.on_device(), vb.make_paged_mask(0.125)
        vb.vla_paged_sparse_attention(cache, batch, mask, lists, q, out, None, torch.empty(vb.vla_paged_sparse_attention_workspace_bytes(cache, batch, mask, 2, 3), dtype=torch.uint8, device=DEV))
        outs.append(out)
    assert torch.equal(*outs)
