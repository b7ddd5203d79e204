"""Selections among infinite scores, in numbers below, equal to and above the places that are free: whole numbers, equal."""
import numpy as np
import pytest
import torch

from paged_ref import DEV, TYPES, Batch
from paper_2510_06710_amd import binding as vb
from test_gpu_paged_sparse import selected_by

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("dtype", ["bf16", "f32"])
INF = float("inf")


def select(b, dtype, q, bounds, most, first, recent):
    k = torch.zeros(b.n_pages, bounds.shape[1], 16, 16, dtype=TYPES[dtype], device=DEV)
    cache, batch = vb.make_paged_cache(k, k), b.on_device()
    selected = torch.full((b.n_rows, bounds.shape[1], most), -77, dtype=torch.int32, device=DEV)
    ws = torch.full((vb.vla_paged_select_workspace_bytes(cache, batch),), 255, dtype=torch.uint8, device=DEV)
    vb.vla_paged_select(cache, batch, bounds.to(DEV), q.to(DEV), selected, first, recent, ws)
    want = selected_by(b, q.double().numpy(), bounds.double().numpy(), most, first, recent)
    assert np.array_equal(selected.cpu().numpy(), want), (selected.tolist(), want.tolist())
    return want


def scored(b, dtype, scores):
    """q and bounds of one head of 16 dims, whose pages' scores are these: an infinite q times a key above, below or at zero (which gives NaN)."""
    q = torch.zeros(b.n_rows, 1, 16, dtype=TYPES[dtype])
    q[:, :, 0] = INF
    bounds = torch.zeros(b.n_pages, 1, 2, 16, dtype=TYPES[dtype])
    sign = np.nan_to_num(np.clip(scores, -1, 1), nan=0)
    bounds[torch.from_numpy(b.table[0, :len(scores)].astype(np.int64)), 0, :, 0] = torch.from_numpy(sign).to(TYPES[dtype])[:, None]
    return q, bounds


@BOTH
def test_as_many_as_there_are_places(dtype):
    b, nan = Batch([(1, 160)], 16), float("nan")
    want = select(b, dtype, *scored(b, dtype, [-INF, -INF, INF, nan, INF, -INF, INF, -INF, -INF, nan]), 6, 1, 2)
    assert want[0, 0].tolist() == [0, 2, 4, 6, 8, 9]


@BOTH
@pytest.mark.parametrize("n", [9, 64, 1000, 5000])
@pytest.mark.parametrize("first,recent", [(0, 1), (1, 2), (3, 1)])
def test_fewer_as_many_and_more(dtype, n, first, recent):
    b, rng = Batch([(1, 16 * n)], 16), np.random.default_rng(n)
    for places in (1, 2, 4, min(n - first - recent - 1, 300)):
        for infinite in {max(0, places - 1), places, places + 1, n}:
            for odd in (0.0, 0.3, 1.0):
                scores = np.where(rng.random(n) < odd, np.nan, -INF)
                scores[first + rng.permutation(n - first - recent)[:infinite]] = INF          # so many among the pages that are chosen from
                select(b, dtype, *scored(b, dtype, scores), first + places + recent, first, recent)
                scores[rng.permutation(n)[:infinite]] = INF
                select(b, dtype, *scored(b, dtype, scores), first + places + recent, first, recent)
                select(b, dtype, *scored(b, dtype, -scores), first + places + recent, first, recent)


@BOTH
def test_an_infinite_query(dtype):
    b, g = Batch([(1, 16 * 40), (2, 16 * 90 + 5)], 16), torch.Generator().manual_seed(2)
    for heads, kv in ((1, 1), (8, 2)):
        bounds = torch.randn(b.n_pages, kv, 2, 16, generator=g).to(TYPES[dtype]).sort(2).values
        q = torch.randn(b.n_rows, heads, 16, generator=g).to(TYPES[dtype])
        q[:, ::4, 3] = INF
        above = [int((bounds[torch.from_numpy(b.table[s, :n].astype(np.int64)), 0, 1, 3] > 0).sum()) for s, n in ((0, 40), (1, 91))]
        for most in sorted({3, 10, *(a + x for a in above for x in range(-1, 6))}):
            select(b, dtype, q, bounds, most, 1, 2)
