"""vla_paged_attention against the formulas in fp64, in pages whose unused places are NaN.

Tolerance, with A = sum w |v| per output.  A score q.k scale is a sum of d products in fp32: off by at most d 2^-24 sum |q||k| scale; a capped one by a further
cap 2^-20 (hardware exponential and reciprocal), a biased one by 2^-22 of the bias; all carry |s| 2^-21 of the change of base for exp2.  With ds the sum of these, a
weight before its norm is off by a factor exp(ds), so an output by 2 ds A; sums over n keys add n 2^-24 A.  bf16: every weight is rounded
once more (2^-8 A) and the output too (2^-8 |o|)."""
import numpy as np
import pytest
import torch

from paged_ref import DEV, TYPES, Batch, attention, visible
from paper_2510_06710_amd import binding as vb

pytestmark = pytest.mark.gpu


def make(b, dtype, heads, kv, d, window, prefix, seed, shared):
    g = torch.Generator().manual_seed(seed)
    pools = []
    for _ in range(2):
        full = torch.randn(b.n_pages, kv, b.page, d, generator=g).to(TYPES[dtype])
        pool = torch.full_like(full, float("nan"))
        for s, (n, length) in enumerate(b.spec):
            see = np.zeros(length, bool)
            for i in range(n):
                see |= visible(length - n + i, length, window, 0 if prefix is None else prefix[s])
            for p in np.nonzero(see)[0]:
                page, at = b.place(s, p)
                pool[page, :, at] = full[page, :, at]
        pools.append(pool)
    return torch.randn(b.n_rows, heads, d, generator=g).to(TYPES[dtype]), pools


def run(b, dtype, heads, kv, d, cap=0.0, bias=False, prefix=None, window=0, shared=0, seed=0, layout="packed", stretch=1.0):
    q, pools = make(b, dtype, heads, kv, d, window, prefix, seed, shared)
    q = (q.float() * stretch).to(q.dtype)
    scale = d ** -0.5
    slopes = 2.0 ** (-8.0 * (torch.arange(heads) + 1.0) / heads) if bias else None
    qd = q.to(DEV)
    out = torch.full((b.n_rows, heads, d), -77.0, dtype=TYPES[dtype], device=DEV)
    if layout == "unaligned":
        big = torch.zeros(b.n_rows, heads * d + 5, dtype=TYPES[dtype], device=DEV)
        big[:, 3:3 + heads * d] = qd.view(b.n_rows, -1)
        qd = big[:, 3:3 + heads * d].unflatten(1, (heads, d))
        wide = torch.full((b.n_rows, heads * d + 7), -77.0, dtype=TYPES[dtype], device=DEV)
        out = wide[:, 1:1 + heads * d].unflatten(1, (heads, d))
    lse = torch.full((b.n_rows, heads), -77.0, device=DEV)
    cache = vb.make_paged_cache(*[p.to(DEV) for p in pools])
    mask = vb.make_paged_mask(scale, cap, None if slopes is None else slopes.to(DEV),
                              None if prefix is None else torch.tensor(prefix, dtype=torch.int32, device=DEV), window, shared)
    batch = b.on_device()
    ws = torch.empty(vb.vla_paged_attention_workspace_bytes(cache, batch, mask, heads), dtype=torch.uint8, device=DEV)
    ws.fill_(255)
    vb.vla_paged_attention(cache, batch, mask, qd, out, lse, ws)
    first = out.clone()
    vb.vla_paged_attention(cache, batch, mask, qd, out, None, ws)
    torch.cuda.synchronize()
    assert torch.equal(first, out)                           # the same call, the same bits
    if layout == "unaligned":
        assert (wide[:, 0] == -77).all() and (wide[:, 1 + heads * d:] == -77).all()
    o, l, mag, reach = attention(b, q.double().numpy(), *[p.double().numpy() for p in pools], scale, cap, None if slopes is None else slopes.double().numpy(), prefix, window)
    got, got_l = out.double().cpu().numpy(), lse.double().cpu().numpy()
    assert (got[b.live:] == -77).all() and (got_l[b.live:] == -77).all()
    got, got_l, o, l, mag, reach = got[:b.live], got_l[:b.live], o[:b.live], l[:b.live], mag[:b.live], reach[:b.live]
    bound = max(1, max(n for _, n in b.spec))
    size = reach + (bound * slopes.double().numpy() if bias else 0)
    ds = d * 2.0 ** -24 * reach + cap * 2.0 ** -20 + size * 2.0 ** -21
    tol = (2 * ds[..., None] + bound * 2.0 ** -24) * mag + ((mag + np.abs(o)) * 2.0 ** -8 if dtype == "bf16" else 0) + 1e-30
    assert np.isfinite(got).all()
    assert (np.abs(got - o) <= tol).all(), (np.abs(got - o) - tol).max()
    blind = np.isinf(l)
    assert (got_l[blind] == -np.inf).all() and (got[blind] == 0).all()
    assert (np.abs(got_l[~blind] - l[~blind]) <= (ds + bound * 2.0 ** -24 + np.abs(l) * 2.0 ** -22)[~blind]).all()


BOTH = pytest.mark.parametrize("dtype", ["bf16", "f32"])
DECODE = [(1, 1), (1, 2), (0, 9), (1, 31), (1, 32), (1, 33), (1, 64), (1, 65), (1, 200)]
PROMPT = [(1, 1), (33, 33), (64, 64), (65, 65), (0, 7), (20, 150), (129, 129), (2, 257)]


@BOTH
@pytest.mark.parametrize("heads,kv,d", [(4, 4, 64), (8, 1, 128), (7, 1, 128), (6, 2, 80), (3, 3, 16), (16, 8, 256), (40, 1, 64), (4, 4, 176)])
def test_single_tokens(dtype, heads, kv, d):
    run(Batch(DECODE, 16, padding=2), dtype, heads, kv, d)
    run(Batch(DECODE, 64), dtype, heads, kv, d, cap=3.0, bias=True)


@BOTH
@pytest.mark.parametrize("heads,kv,d", [(4, 4, 64), (8, 2, 128), (6, 2, 80), (2, 1, 256), (3, 1, 48)])
def test_prompts(dtype, heads, kv, d):
    run(Batch(PROMPT, 16, padding=1), dtype, heads, kv, d)
    run(Batch(PROMPT, 128), dtype, heads, kv, d, cap=2.0, bias=True)


@BOTH
@pytest.mark.parametrize("spec", [DECODE, PROMPT])
@pytest.mark.parametrize("window", [1, 31, 100])
def test_window(dtype, spec, window):
    run(Batch(spec, 16), dtype, 4, 2, 64, window=window)
    run(Batch(spec, 32), dtype, 4, 2, 64, window=window, prefix=[min(l, 7 * i) for i, (_, l) in enumerate(spec)], bias=True)


@BOTH
def test_prefix_mask(dtype):
    for share in (0, 1, 2):
        run(Batch(PROMPT, 16), dtype, 4, 2, 64, prefix=[l * share // 2 for _, l in PROMPT], cap=30.0)
    run(Batch(PROMPT, 16), dtype, 4, 2, 128, prefix=[1000] * len(PROMPT))          # longer than the sequence: all of it


@BOTH
def test_rows_that_see_nothing(dtype):
    run(Batch([(3, 0), (5, 2), (1, 0), (40, 3)], 16), dtype, 4, 1, 64)


@BOTH
@pytest.mark.parametrize("rows", [1, 3])
def test_long_context_is_split(dtype, rows):
    run(Batch([(rows, 5000)], 64), dtype, 8, 2, 64)
    run(Batch([(rows, 3001), (rows, 17), (rows, 800)], 32), dtype, 8, 2, 128, cap=20.0)
    run(Batch([(rows, 4097)], 16), dtype, 4, 4, 64, window=1500)


@BOTH
def test_chunk_behind_a_long_context(dtype):
    run(Batch([(70, 2500), (9, 40)], 64), dtype, 4, 2, 64)


@BOTH
@pytest.mark.parametrize("heads,kv,d", [(8, 8, 64), (4, 4, 128), (2, 2, 256)])
def test_many_whole_tiles(dtype, heads, kv, d):
    spec = [(130, 1030), (1, 1500), (129, 1129), (140, 1400)]                      # key ranges of dozens of tiles that every row sees
    run(Batch(spec, 16), dtype, heads, kv, d)
    run(Batch(spec, 64), dtype, heads, kv, d, window=900)


@BOTH
@pytest.mark.parametrize("heads,kv,d", [(4, 4, 64), (8, 2, 128)])
def test_shared_prefix(dtype, heads, kv, d):
    run(Batch([(1, 130), (1, 128), (0, 200), (1, 200), (2, 140)], 64, shared=128), dtype, heads, kv, d, shared=128)
    run(Batch([(1, 1024 + i) for i in range(1, 40)], 16, shared=1024), dtype, heads, kv, d, shared=1024, cap=10.0, bias=True)
    run(Batch([(3, 300), (1, 131), (130, 260)], 32, shared=128), dtype, heads, kv, d, shared=128)      # new rows within the shared part too


@BOTH
def test_layouts_and_sharp_scores(dtype):
    run(Batch(DECODE, 16), dtype, 4, 2, 64, layout="unaligned")
    run(Batch(PROMPT, 16), dtype, 4, 2, 80, layout="unaligned")
    run(Batch(PROMPT, 16), dtype, 4, 2, 64, stretch=30.0)                          # scores of a hundred and more: one weight takes all
    run(Batch(DECODE, 16), dtype, 4, 2, 64, stretch=30.0)


@BOTH
def test_loose_host_bounds_and_bad_pages(dtype):
    run(Batch(DECODE, 16, max_len=4000), dtype, 4, 2, 64)
    run(Batch(PROMPT, 16, max_len=700, extra_entries=3), dtype, 4, 2, 64)
    b = Batch([(1, 100), (40, 90)], 16)
    q, pools = make(b, dtype, 2, 1, 64, 0, None, 0, 0)
    dev = [p.to(DEV) for p in pools]
    outs = []
    for bad in (False, True):                                # a page that is not there reads as zeros
        if bad:
            b.table[0, 3], b.table[1, 1] = b.n_pages, -1
        else:
            for p in dev:
                p[b.table[0, 3]] = 0
                p[b.table[1, 1]] = 0
        out = torch.zeros(b.n_rows, 2, 64, dtype=TYPES[dtype], device=DEV)
        cache, batch, mask = vb.make_paged_cache(*dev), b.on_device(), vb.make_paged_mask(0.125)
        ws = torch.empty(vb.vla_paged_attention_workspace_bytes(cache, batch, mask, 2), dtype=torch.uint8, device=DEV)
        vb.vla_paged_attention(cache, batch, mask, q.to(DEV), out, None, ws)
        outs.append(out)
    assert torch.equal(*outs)


@BOTH
@pytest.mark.parametrize("shared", [0, 16])
def test_thousands_of_sequences(dtype, shared):
    run(Batch([(1, 17 + s % 40) for s in range(2051)], 16, shared=shared, padding=3), dtype, 2, 1, 32, shared=shared)


@pytest.mark.parametrize("heads,kv", [(4, 2), (64, 1)])
@pytest.mark.parametrize("shared", [0, 32])
def test_rows_beyond_the_host_bound_are_left(heads, kv, shared):
    b = Batch([(5, 60), (1, 200), (3, 35)], 16, shared=shared)
    q, pools = make(b, "f32", heads, kv, 64, 0, None, 0, shared)
    dev, outs = [p.to(DEV) for p in pools], []
    for b.max_rows in (5, 2):
        out, lse = torch.full((b.n_rows, heads, 64), -77.0, device=DEV), torch.full((b.n_rows, heads), -77.0, device=DEV)
        cache, batch, mask = vb.make_paged_cache(*dev), b.on_device(), vb.make_paged_mask(0.125, shared_len=shared)
        ws = torch.full((vb.vla_paged_attention_workspace_bytes(cache, batch, mask, heads),), 255, dtype=torch.uint8, device=DEV)
        vb.vla_paged_attention(cache, batch, mask, q.to(DEV), out, lse, ws)
        outs.append((out.cpu(), lse.cpu()))
    (full, full_l), (some, some_l) = outs
    kept = torch.tensor([0, 1, 5, 6, 7])
    # two evaluations, each off by 2 ds A + n 2^-24 A with ds < 64 2^-24 x 40 + 5 x 2^-21, A < 5, n = 200
    assert (full[kept] - some[kept]).abs().max() <= 2 * (2 * (64 * 40 * 2.0 ** -24 + 5 * 2.0 ** -21) + 200 * 2.0 ** -24) * 5 and (full_l[kept] - some_l[kept]).abs().max() <= 1e-3
    left = torch.tensor([2, 3, 4, 8])
    assert (some[left] == -77).all() and (some_l[left] == -77).all() and (full != -77).all()
