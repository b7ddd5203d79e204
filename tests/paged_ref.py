"""The paged operators in 64 bits, one row and one head at a time, and the ragged batches that their tests use.  Written from the formulas in include/vla.h;
what no row of a call may read (pages nobody owns, positions behind a sequence's end or before every window) is NaN."""
import numpy as np
import torch

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def visible(p, n_keys, window, prefix):
    """Positions a row at position p sees, of a sequence that holds n_keys."""
    j = np.arange(n_keys)
    return ((j <= p) & ((j > p - window) if window else True)) | (j < prefix)


class Batch:
    """spec: (rows, positions held) per sequence.  Pages in random order; the first `shared` positions in the same pages for all."""

    def __init__(self, spec, page, seed=0, shared=0, extra_entries=0, padding=0, max_len=None):
        rng = np.random.default_rng(seed)
        self.spec, self.page, self.padding = spec, page, padding
        self.max_rows, self.max_len = max(r for r, _ in spec), max(l for _, l in spec) if max_len is None else max_len
        per = max(1, -(-self.max_len // page)) + extra_entries
        need = [-(-l // page) for _, l in spec]
        self.n_pages = sum(need) + 2
        ids = iter(rng.permutation(self.n_pages))
        self.table = np.full((len(spec), per), -1, np.int32)
        for s, n in enumerate(need):
            for e in range(n):
                self.table[s, e] = self.table[0, e] if s and e < shared // page else next(ids)
        self.start = np.concatenate([[0], np.cumsum([r for r, _ in spec])]).astype(np.int32)
        self.live = int(self.start[-1])
        self.n_rows = self.live + padding

    def rows(self):
        """(row, sequence, position) of the rows that are not padding."""
        for s, (n, length) in enumerate(self.spec):
            for i in range(n):
                yield int(self.start[s]) + i, s, length - n + i

    def place(self, s, p):
        return self.table[s, p // self.page], p % self.page

    def on_device(self):
        from paper_2510_06710_amd import binding as vb
        t = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
        return vb.make_paged_batch(t(self.start), t(np.array([l for _, l in self.spec], np.int32)), t(self.table), self.n_rows, self.max_rows, self.max_len)


def gather(b, pool, s, n):
    """Positions 0 .. n - 1 of sequence s: [n, heads, dim]."""
    p = np.arange(n)
    return pool[b.table[s, p // b.page], :, p % b.page]


def attention(b, q, k, v, scale, cap=0.0, slopes=None, prefix=None, window=0):
    """out, lse, sum of weights |v|, and a bound of |q||k| scale per row and head; all fp64."""
    n_heads, d = q.shape[1:]
    group = n_heads // k.shape[1]
    out, lse, mag = np.zeros((b.n_rows, n_heads, d)), np.full((b.n_rows, n_heads), -np.inf), np.zeros((b.n_rows, n_heads, d))
    reach = np.zeros((b.n_rows, n_heads))
    held = {}
    for row, s, p in b.rows():
        n = b.spec[s][1]
        see = visible(p, n, window, 0 if prefix is None else prefix[s])
        if p < 0 and prefix is None or not see.any():
            continue
        if s not in held:
            held[s] = gather(b, k, s, n), gather(b, v, s, n)
        ks, vs = held[s][0][see], held[s][1][see]
        j = np.arange(n)[see]
        for h in range(n_heads):
            x = ks[:, h // group] @ q[row, h] * scale
            reach[row, h] = (np.abs(ks[:, h // group]) @ np.abs(q[row, h]) * scale).max()
            if cap:
                x = cap * np.tanh(x / cap)
            if slopes is not None:
                x = x - slopes[h] * np.abs(p - j)
            w = np.exp(x - x.max())
            lse[row, h] = x.max() + np.log(w.sum())
            w /= w.sum()
            out[row, h], mag[row, h] = w @ vs[:, h // group], w @ np.abs(vs[:, h // group])
    return out, lse, mag, reach


def rotated(x, pos, gain, eps, freq, interleaved, scale):
    """x [rows, heads, d] in fp64 at positions pos; also the sum of the magnitudes that each value was formed from."""
    y = x.copy()
    if gain is not None:
        y = y / np.sqrt((y ** 2).mean(-1, keepdims=True) + eps) * gain
    mag = np.abs(y)
    half = len(freq)
    if half:
        c, s = np.cos(pos[:, None] * freq)[:, None] * scale, np.sin(pos[:, None] * freq)[:, None] * scale
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
        ya, yb = y[..., a].copy(), y[..., b].copy()
        y[..., a], y[..., b] = c * ya - s * yb, c * yb + s * ya
        mag[..., a] = mag[..., b] = (np.abs(ya) + np.abs(yb)) * abs(scale)
    return y, mag


def sample(z, t, k, p, least, u):
    """token, n_kept, logp, logp_kept of one row of fp64 logits."""
    ok = z > -np.inf
    if not ok.any():
        return -1, 0, -np.inf, -np.inf
    y = z / t if t > 0 else z
    order = np.lexsort((np.arange(len(z)), -np.where(ok, z, -np.inf)))[:ok.sum()]
    if z[order[0]] == np.inf:
        w = (z == np.inf).astype(float)
        order = order[:int(w.sum())]
    else:
        w = np.where(ok, np.exp(np.where(ok, y, 0) - y[order[0]]), 0.0)
    total = w.sum()
    if k > 0:
        order = order[:k]
    m = w[order]
    if p < 1:
        n = int(((np.cumsum(m) - m) < max(p, 0) * m.sum()).sum())
        order = order[:max(n, 1)]
    order = order[:max(1, int((w[order] >= least).sum()))]
    ids = np.sort(order)
    run = np.cumsum(w[ids])
    token = order[0]
    if u is not None and t > 0:
        token = ids[min(int((run <= u * run[-1]).sum()), int(np.nonzero(w[ids])[0].max()))]
    with np.errstate(divide="ignore"):
        return int(token), len(ids), np.log(w[token]) - np.log(total), np.log(w[token]) - np.log(run[-1])
