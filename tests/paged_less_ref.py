"""The operators that read less per token, in 64 bits and one row, node or head at a time, written from the formulas in include/vla.h."""
import numpy as np
import torch

from paged_ref import DEV, TYPES, gather


def softmax_rows(q, ks, vs, scale, cap):
    """out, lse, sum of weights |v| and the largest |q||k| scale of one head's query over the keys it sees."""
    d = vs.shape[1]
    if len(ks) == 0:
        return np.zeros(d), -np.inf, np.zeros(d), 0.0
    x = ks @ q * scale
    reach = (np.abs(ks) @ np.abs(q) * scale).max()
    if cap:
        x = cap * np.tanh(x / cap)
    w = np.exp(x - x.max())
    total = w.sum()
    return w @ vs / total, x.max() + np.log(total), w @ np.abs(vs) / total, reach


def rows_of(b, q, k, v, scale, cap, seen_by):
    """Attention of every row and head over the positions seen_by(row, sequence, position, key head); out, lse, magnitude, reach."""
    n_heads, d = q.shape[1:]
    group = n_heads // k.shape[1]
    out, lse, mag, reach = np.zeros((b.n_rows, n_heads, d)), np.full((b.n_rows, n_heads), -np.inf), np.zeros((b.n_rows, n_heads, d)), np.zeros((b.n_rows, n_heads))
    held = {}
    for row, s, p in b.rows():
        if s not in held:
            held[s] = gather(b, k, s, b.spec[s][1]), gather(b, v, s, b.spec[s][1])
        for h in range(n_heads):
            at = seen_by(row, s, p, h // group)
            out[row, h], lse[row, h], mag[row, h], reach[row, h] = softmax_rows(q[row, h], held[s][0][at, h // group], held[s][1][at, h // group], scale, cap)
    return out, lse, mag, reach


def check_rows(b, dtype, d, cap, got, got_l, want, most, split=True):
    """The tolerance of test_gpu_paged_attention.py (see there), with the weights' tail where they have one."""
    o, l, mag, reach = (x[:b.live] for x in want)
    got, got_l = got.double().cpu().numpy(), got_l.double().cpu().numpy()
    assert (got[b.live:] == -77).all() and (got_l[b.live:] == -77).all()
    got, got_l = got[:b.live], got_l[:b.live]
    ds = d * 2.0 ** -24 * reach + cap * 2.0 ** -20 + reach * 2.0 ** -21
    last = 2.0 ** -16 * mag + 2.0 ** -8 * np.abs(o) if dtype == "bf16" else 0
    tol = (2 * ds[..., None] + most * 2.0 ** -24) * mag + last + 1e-30
    assert np.isfinite(got).all()
    assert (np.abs(got - o) <= tol).all(), (np.abs(got - o) - tol).max()
    blind = np.isinf(l)
    assert (got_l[blind] == -np.inf).all() and (got[blind] == 0).all()
    assert (np.abs(got_l[~blind] - l[~blind]) <= (ds + most * 2.0 ** -24 + np.abs(l) * 2.0 ** -22)[~blind]).all()


def pools_of(b, dtype, kv, d, seed, layers=None):
    """K and V of the positions held; whatever else there is in the pages is NaN."""
    g = torch.Generator().manual_seed(seed)
    shape = ((layers,) if layers else ()) + (b.n_pages, kv, b.page, d)
    pools = []
    for _ in range(2):
        full = torch.randn(shape, generator=g).to(TYPES[dtype])
        pool = torch.full_like(full, float("nan"))
        for s, (_, length) in enumerate(b.spec):
            for p in range(length):
                page, at = b.place(s, p)
                pool[..., page, :, at, :] = full[..., page, :, at, :]
        pools.append(pool)
    return pools


def random_tree(n, rng):
    """Parents: mostly of the last few nodes, some of any earlier one."""
    return [-1] + [int(rng.integers(0, i)) if rng.random() < 0.2 else max(0, i - 1 - int(rng.integers(0, 4))) for i in range(1, n)]


def ancestors(parents):
    """[n, n]: node i sees node j."""
    n = len(parents)
    see = np.zeros((n, n), bool)
    depth = np.zeros(n, int)
    for i, p in enumerate(parents):
        if 0 <= p < i:
            see[i], depth[i] = see[p], depth[p] + 1
        see[i, i] = True
    return see, depth


def bits(see, words):
    """Rows of truth values as 32-bit words."""
    full = np.zeros((see.shape[0], words * 32), bool)
    full[:, :see.shape[1]] = see
    return (full.reshape(-1, words, 32).astype(np.uint64) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32).view(np.int32)


def follow(parents, ids, chosen):
    path, n = [], len(parents)
    cur = 0 if n else None
    while cur is not None:
        path.append(cur)
        cur = next((i for i in range(cur + 1, n) if parents[i] == cur and ids[i] == chosen[cur] and chosen[cur] >= 0), None)
    return path


def page_bounds(b, k, s, number):
    """[2, heads, d] of a sequence's page: least and largest of the positions held."""
    at = range(number * b.page, min((number + 1) * b.page, b.spec[s][1]))
    keys = np.stack([k[b.table[s, p // b.page], :, p % b.page] for p in at])
    return np.stack([keys.min(0), keys.max(0)])


def choose(score, most, first, recent):
    """Numbers of the pages taken of len(score) pages."""
    n = len(score)
    always = [i < first or i >= n - recent for i in range(n)]
    rank = sorted(range(n), key=lambda i: (not always[i], 0 if not np.isnan(score[i]) else 1, -score[i] if not np.isnan(score[i]) else 0, i))
    return sorted(rank[:most])


def to_device(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x))
    return (t if dtype is None else t.to(dtype)).to(DEV)
