"""vla_paged_append against the formulas in fp64.

Tolerance.  fp32 arithmetic: a value is x f g cos +- x' f g sin (f of the norm), every factor and step off by half an fp32 step, 2^-24; the mean of d squares,
added by eight in a lane and then pairwise, by at most (8 + log2 d) of them, and the root halves that.  With M = |x f g| + |x' f g| the whole is within
(8 + (8 + log2 d) / 2 + 4) 2^-24 M < 20 * 2^-24 M; bf16 storage adds half its step, 2^-8 |y| (of the fp32 value: (1 + 2^-8) covers that)."""
import numpy as np
import pytest
import torch

from paged_ref import DEV, TYPES, Batch, rotated
from paper_2510_06710_amd import binding as vb

pytestmark = pytest.mark.gpu
MARK = -77.0


def run(b, src, dtype, heads, kv, d, rot, interleaved, norms, split="fused", with_q=True, pages=None, seed=0, scale=1.0, base=10000.0):
    g = torch.Generator().manual_seed(seed)
    wide = heads + 2 * kv
    x = torch.randn(b.n_rows, wide, d, generator=g).to(TYPES[src])
    x[b.live:] = float("nan")
    xd = x.to(DEV)
    if split == "fused":
        q, k, v = xd[:, :heads], xd[:, heads:heads + kv], xd[:, heads + kv:]
    elif split == "apart":
        q, k, v = (xd[:, i:j].contiguous() for i, j in ((0, heads), (heads, heads + kv), (heads + kv, wide)))
    else:                                                    # rows that start two or four bytes past a multiple of 16
        flat = torch.zeros(b.n_rows, wide * d + 3, dtype=TYPES[src], device=DEV)
        flat[:, 1:1 + wide * d] = xd.view(b.n_rows, -1)
        y = flat[:, 1:1 + wide * d].unflatten(1, (wide, d))
        q, k, v = y[:, :heads], y[:, heads:heads + kv], y[:, heads + kv:]
    half = rot // 2
    freq = base ** (-np.arange(half) / max(half, 1))
    gains = [1 + 0.2 * torch.randn(d, generator=g) for _ in range(2)] if norms else [None, None]
    pools = [torch.full((pages or b.n_pages, kv, b.page, d), MARK, dtype=TYPES[dtype], device=DEV) for _ in range(2)]
    q_out = torch.full((b.n_rows, heads, d), MARK, dtype=TYPES[dtype], device=DEV)
    rotary = vb.make_rotary(torch.from_numpy(freq).to(DEV) if half else None, interleaved, scale, *[None if t is None else t.to(DEV) for t in gains], eps=1e-5)
    vb.vla_paged_append(vb.make_paged_cache(*pools), b.on_device(), rotary, q if with_q else None, k, v, q_out if with_q else None)
    torch.cuda.synchronize()
    x = x.double().numpy()
    rows = [(r, s, p) for r, s, p in b.rows() if 0 <= p < b.max_len]
    at, pos = np.array([r for r, _, _ in rows], int), np.array([p for _, _, p in rows], float)
    want = {}
    for name, part, gain in (("q", x[:, :heads], gains[0]), ("k", x[:, heads:heads + kv], gains[1])):
        want[name] = rotated(part[at], pos, None if gain is None else gain.double().numpy(), 1e-5, freq, interleaved, scale)
    want["v"] = (x[at, heads + kv:], np.abs(x[at, heads + kv:]))

    def close(got, name, sel=slice(None)):
        y, mag = want[name]
        tol = 20 * 2.0 ** -24 * mag + (2.0 ** -8 * np.abs(y) * (1 + 2.0 ** -8) if dtype == "bf16" else 0)
        err = np.abs(got - y[sel]) - tol[sel]
        assert (err <= 0).all(), (name, err.max())

    qh = q_out.double().cpu().numpy()
    rest = np.ones(b.n_rows, bool)
    if with_q:
        close(qh[at], "q")
        rest[at] = False
    assert (qh[rest] == MARK).all()
    for pool, name in zip(pools, "kv"):
        pool = pool.double().cpu().numpy()
        ok = np.array([0 <= b.place(s, p)[0] < len(pool) for _, s, p in rows], bool)
        where = np.array([b.place(s, p) for _, s, p in rows]).reshape(-1, 2)[ok]
        close(pool[where[:, 0], :, where[:, 1]], name, ok)
        pool[where[:, 0], :, where[:, 1]] = MARK
        assert (pool == MARK).all()                          # nothing else was touched


SPEC = [(1, 1), (0, 5), (17, 17), (3, 40), (16, 48), (5, 130)]


@pytest.mark.parametrize("src,dtype", [("f32", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("bf16", "f32")])
@pytest.mark.parametrize("heads,kv,d,rot", [(4, 4, 64, 64), (8, 2, 128, 128), (6, 3, 80, 40), (3, 1, 16, 6), (2, 2, 256, 128), (7, 1, 48, 0)])
def test_types_and_heads(src, dtype, heads, kv, d, rot):
    for interleaved in (False, True):
        run(Batch(SPEC, 16, padding=3), src, dtype, heads, kv, d, rot, interleaved, norms=d != 48)


@pytest.mark.parametrize("split", ["apart", "unaligned"])
def test_layouts(split):
    run(Batch(SPEC, 32), "bf16", "bf16", 4, 2, 128, 128, False, True, split)
    run(Batch(SPEC, 32), "f32", "f32", 5, 1, 32, 30, True, False, split)


def test_far_positions_and_scaled_angles():
    run(Batch([(3, 1 << 20), (1, 999_999)], 1024), "f32", "f32", 2, 1, 128, 128, False, False, scale=1.25, base=5e5)


def test_more_rows_than_positions_and_keys_alone():
    run(Batch([(6, 4), (2, 2), (3, 0)], 16), "f32", "bf16", 4, 2, 64, 64, False, True)
    run(Batch(SPEC, 16), "f32", "bf16", 4, 2, 64, 64, False, True, with_q=False)


def test_many_rows():
    run(Batch([(700, 700), (1, 12), (333, 400)], 64), "f32", "bf16", 8, 8, 128, 128, False, False)


def test_work_beyond_the_host_bounds_is_left_out():
    b = Batch([(4, 40), (2, 12)], 16, max_len=38)            # positions 38 and 39 are beyond
    run(b, "f32", "f32", 2, 1, 64, 64, False, False)
    b = Batch([(4, 40), (2, 12)], 16)
    b.table[0, 2] = -5                                       # page of positions 32 .. 47: not written
    run(b, "f32", "f32", 2, 1, 64, 64, False, False)
    b.table[0, 2] = b.n_pages                                # one past the last
    run(b, "f32", "f32", 2, 1, 64, 64, False, False)


def test_in_place():
    b = Batch(SPEC, 16)
    x = torch.randn(b.n_rows, 4, 64, device=DEV)
    k = torch.randn(b.n_rows, 1, 64, device=DEV)
    freq = torch.rand(20, dtype=torch.float64, device=DEV)
    outs = []
    for same in (False, True):
        pools = [torch.zeros(b.n_pages, 1, 16, 64, device=DEV) for _ in range(2)]
        q = x.clone()
        out = q if same else torch.empty_like(q)
        gain = torch.ones(64, device=DEV)
        vb.vla_paged_append(vb.make_paged_cache(*pools), b.on_device(), vb.make_rotary(freq, q_gain=gain), q, k, k, out)
        outs.append(out)
    assert torch.equal(*outs)
