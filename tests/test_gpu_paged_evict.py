"""Softmax weights summed per position, and caches cut to their heaviest positions.

Tolerance of a mass.  A score is off by ds = d 2^-24 R + |s| 2^-21 (R = sum |q||k| scale; see test_gpu_paged_attention.py), plus cap 2^-20 where capped and 2^-22 of the bias; a
weight exp(s - lse), with the lse that the call is given, by a factor of exp(ds + |lse| 2^-22) and the exponential's own 2^-22; sums of n weights add n 2^-24.  Since all
weights of a mass are positive it is off by at most (2 max ds + n 2^-24) of it, and its old value's addition by 2^-24 of both.  Evictions are whole numbers and moved bits."""
import numpy as np
import pytest
import torch

from paged_less_ref import pools_of, to_device
from paged_ref import DEV, TYPES, Batch, attention, gather, visible
from paper_2510_06710_amd import binding as vb

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("dtype", ["bf16", "f32"])
DECODE = [(1, 1), (1, 2), (0, 9), (1, 31), (1, 32), (1, 33), (1, 65), (1, 200)]
PROMPT = [(1, 1), (33, 33), (64, 64), (65, 65), (0, 7), (20, 150), (129, 129), (2, 257)]


def weigh(b, dtype, heads, kv, d, cap=0.0, bias=False, prefix=None, window=0, shared=0, layout="packed", seed=0):
    pools = pools_of(b, dtype, kv, d, seed)
    q = torch.randn(b.n_rows, heads, d, generator=torch.Generator().manual_seed(seed + 1)).to(TYPES[dtype])
    scale, slopes = d ** -0.5, 2.0 ** (-8.0 * (torch.arange(heads) + 1.0) / heads) if bias else None
    k = pools[0].double().numpy()
    _, lse, _, reach = attention(b, q.double().numpy(), k, pools[1].double().numpy(), scale, cap, None if slopes is None else slopes.double().numpy(), prefix, window)
    lse = lse.astype(np.float32)
    qd = q.to(DEV)
    if layout == "unaligned":
        qd = torch.zeros(b.n_rows, heads * d + 5, dtype=TYPES[dtype], device=DEV)[:, 3:3 + heads * d].unflatten(1, (heads, d))
        qd.copy_(q)
    n_seq, stride = len(b.spec), b.max_len + 3
    old = torch.rand(n_seq, kv, stride, generator=torch.Generator().manual_seed(seed + 2))
    for s, (n, length) in enumerate(b.spec):
        old[s, :, length - n:length] = float("nan")           # what new positions held counts for nothing
    pools[1].fill_(float("nan"))                              # (V is not read)
    cache, batch = vb.make_paged_cache(*[p.to(DEV) for p in pools]), b.on_device()
    mask = vb.make_paged_mask(scale, cap, None if slopes is None else slopes.to(DEV), None if prefix is None else torch.tensor(prefix, dtype=torch.int32, device=DEV), window, shared)
    ws = torch.full((vb.vla_paged_weights_workspace_bytes(cache, batch, mask, heads),), 255, dtype=torch.uint8, device=DEV)
    got = []
    for _ in range(2):
        mass = old.to(DEV)
        vb.vla_paged_weights(cache, batch, mask, qd, to_device(lse), mass, ws)
        got.append(mass.cpu())
    assert torch.equal(got[0].view(torch.int32), got[1].view(torch.int32))
    got, group = got[0].double().numpy(), heads // kv
    for s, (n, length) in enumerate(b.spec):
        keys, a = gather(b, k, s, length), b.start[s]
        want = old[s].double().numpy().copy()
        if n:
            want[:, max(0, length - n):length] = 0
        added = np.zeros((kv, length))
        ds, j = 0.0, np.arange(length)
        for i in range(n):
            p = length - n + i
            see = visible(p, length, window, 0 if prefix is None else prefix[s])
            for h in range(heads):
                if lse[a + i, h] == -np.inf:
                    continue
                x = keys[:, h // group] @ q[a + i, h].double().numpy() * scale
                if cap:
                    x = cap * np.tanh(x / cap)
                size = reach[a + i, h]
                if bias:
                    x = x - slopes[h].double().item() * np.abs(p - j)
                    size += slopes[h].item() * length
                added[h // group] += np.where(see, np.exp(x - np.float64(lse[a + i, h])), 0)
                ds = max(ds, d * 2.0 ** -24 * reach[a + i, h] + size * 2.0 ** -21 + cap * 2.0 ** -20 + (abs(lse[a + i, h]) + 1) * 2.0 ** -22)
        want[:, :length] += added
        tol = (2 * ds + (n * group + 2) * 2.0 ** -24) * added + 2.0 ** -23 * want[:, :length] + 1e-37
        assert (np.abs(got[s, :, :length] - want[:, :length]) <= tol).all(), (s, (np.abs(got[s, :, :length] - want[:, :length]) - tol).max())
        assert np.array_equal(got[s, :, length:], old[s, :, length:].double().numpy())


@BOTH
@pytest.mark.parametrize("heads,kv,d", [(4, 4, 64), (8, 1, 128), (7, 1, 128), (6, 2, 80), (16, 8, 256), (40, 1, 64), (3, 3, 16)])
@pytest.mark.parametrize("spec", [DECODE, PROMPT])
def test_weights(dtype, heads, kv, d, spec):
    weigh(Batch(spec, 16, padding=2), dtype, heads, kv, d)
    weigh(Batch(spec, 64), dtype, heads, kv, d, cap=3.0, bias=True)


@BOTH
@pytest.mark.parametrize("spec", [DECODE, PROMPT])
@pytest.mark.parametrize("window", [0, 1, 31, 100])
def test_weights_under_masks(dtype, spec, window):
    weigh(Batch(spec, 16), dtype, 4, 2, 64, window=window, layout="unaligned")
    weigh(Batch(spec, 32), dtype, 4, 2, 64, window=window, prefix=[min(l, 7 * i) for i, (_, l) in enumerate(spec)], bias=True)
    weigh(Batch(spec, 32), dtype, 4, 2, 64, window=window, prefix=[l // 2 for _, l in spec], cap=20.0)


@BOTH
def test_weights_of_long_and_blind_rows(dtype):
    weigh(Batch([(3, 0), (5, 2), (1, 0), (40, 3)], 16), dtype, 4, 1, 64)
    weigh(Batch([(1, 3000), (300, 700), (2, 40)], 64, max_len=4000), dtype, 8, 2, 64)
    weigh(Batch([(1, 130), (1, 128), (0, 200), (2, 140)], 64, shared=128), dtype, 4, 2, 64, shared=128)
    weigh(Batch([(700, 720)], 64), dtype, 4, 1, 128)


def test_weights_of_a_row_are_one():
    """Every row's weights over the whole cache sum to its number of heads, with the attention's own lse."""
    b = Batch(PROMPT, 16)
    pools, q = [p.to(DEV) for p in pools_of(b, "bf16", 2, 128, 4)], torch.randn(b.n_rows, 8, 128, generator=torch.Generator().manual_seed(1)).bfloat16().to(DEV)
    cache, batch, mask = vb.make_paged_cache(*pools), b.on_device(), vb.make_paged_mask(128 ** -0.5, 30.0)
    empty = lambda n: torch.empty(n, dtype=torch.uint8, device=DEV)
    out, lse, mass = torch.zeros_like(q), torch.zeros(b.n_rows, 8, device=DEV), torch.zeros(len(b.spec), 2, b.max_len, device=DEV)
    vb.vla_paged_attention(cache, batch, mask, q, out, lse, empty(vb.vla_paged_attention_workspace_bytes(cache, batch, mask, 8)))
    vb.vla_paged_weights(cache, batch, mask, q, lse, mass, empty(vb.vla_paged_weights_workspace_bytes(cache, batch, mask, 8)))
    for s, (n, _) in enumerate(b.spec):
        # scores of the two products are the same sums of 128 products in another order: 2 x 128 2^-24 R, R < 40; lse 2^-22 of 6, twice the cap's 30 2^-20
        assert abs(mass[s].double().sum().item() - 8 * n) <= 8 * n * (2 * 128 * 40 * 2.0 ** -24 + 60 * 2.0 ** -20 + 1e-5)


def rank(weight, length, keep, first, recent):
    w = [(-np.inf if np.isnan(x) else x) for x in weight]
    nan = [np.isnan(x) for x in weight]
    order = sorted(range(length), key=lambda j: (not (j < first or j >= length - recent), nan[j], -w[j], j))
    return sorted(order[:keep])


def cut(b, dtype, kv, d, keep, first, recent, masses, in_place=False, seed=0, own_pages=()):
    """own_pages: sequences that keep their table (they hold no more than keep)."""
    n, page = len(b.spec), b.page
    g = torch.Generator().manual_seed(seed)
    per = -(-keep // page) + 1
    extra = n * per
    pools = [torch.randn(b.n_pages + extra, kv, page, d, generator=g).to(TYPES[dtype]) for _ in range(2)]
    to_table = b.n_pages + torch.randperm(extra, generator=g).view(n, per).numpy().astype(np.int32)
    for s in own_pages:
        some = min(per, b.table.shape[1])
        to_table[s, :some] = b.table[s, :some]
    k, v = (p.to(DEV) for p in pools)
    mass = masses.to(DEV)
    out = mass if in_place else torch.full((n, kv, keep + 2), -77.0, device=DEV)
    kept, new_len = torch.full((n, kv, keep), -77, dtype=torch.int32, device=DEV), torch.full((n,), -77, dtype=torch.int32, device=DEV)
    vb.vla_paged_evict(vb.make_paged_cache(k, v), b.on_device(), mass, first, recent, to_device(to_table), kept, out, new_len)
    want_out = masses.clone() if in_place else torch.full((n, kv, keep + 2), -77.0)
    for s, (_, length) in enumerate(b.spec):
        assert new_len[s].item() == min(length, keep)
        for h in range(kv):
            at = rank(masses[s, h, :length].tolist(), length, keep, first, recent) if length > keep else list(range(length))
            assert kept[s, h].tolist() == at + [-1] * (keep - len(at)), (s, h)
            want_out[s, h, :len(at)] = masses[s, h, at]
            for to, j in enumerate(at):
                for pool in pools:
                    pool[to_table[s, to // page], h, to % page] = pool[b.table[s, j // page], h, j % page]
    assert torch.equal(out.cpu().view(torch.int32), want_out.view(torch.int32))
    assert all(torch.equal(x.cpu().view(torch.int16), y.view(torch.int16)) for x, y in ((k, pools[0]), (v, pools[1])))


HELD = [(0, 0), (1, 1), (1, 16), (0, 40), (1, 41), (3, 200), (0, 333), (1, 39)]


@BOTH
@pytest.mark.parametrize("kv,d", [(1, 16), (2, 80), (8, 128), (3, 256)])
@pytest.mark.parametrize("keep,first,recent", [(1, 0, 0), (1, 1, 0), (16, 0, 1), (40, 4, 10), (40, 20, 20), (100, 0, 0), (400, 3, 3)])
def test_evict(dtype, kv, d, keep, first, recent):
    b = Batch(HELD, 16)
    masses = torch.rand(len(HELD), kv, b.max_len, generator=torch.Generator().manual_seed(keep))
    cut(b, dtype, kv, d, keep, first, recent, masses)


def test_evict_ties_and_odd_masses():
    b = Batch([(0, 3000), (0, 1025), (0, 1024), (0, 2)], 64)
    g = torch.Generator().manual_seed(2)
    few = torch.randint(0, 3, (4, 2, b.max_len), generator=g).float()
    odd = torch.randn(4, 2, b.max_len, generator=g)
    odd[:, :, ::7], odd[:, :, 1::7], odd[:, :, 2::7], odd[:, :, 3::7] = float("nan"), -0.0, 0.0, float("inf")
    for masses in (torch.zeros(4, 2, b.max_len), few, odd, torch.full((4, 2, b.max_len), float("nan")), -few):
        for keep, first, recent in ((1000, 0, 0), (700, 5, 300), (2900, 1, 1), (3, 1, 1)):
            cut(b, "bf16", 2, 16, keep, first, recent, masses)
            cut(b, "f32", 2, 16, keep, first, recent, masses, in_place=True)


def test_evict_of_more_than_are_held():
    """Above 32,768 positions the masses are read again for every pass; the same by small caches under a loose bound."""
    b = Batch([(0, 40000), (0, 33000), (0, 70)], 128)
    g = torch.Generator().manual_seed(5)
    for masses in (torch.rand(3, 1, b.max_len, generator=g), torch.randint(0, 2, (3, 1, b.max_len), generator=g).float()):
        for in_place in (False, True):
            cut(b, "f32", 1, 16, 3000, 2, 1000, masses, in_place=in_place)
    b = Batch(HELD, 16, max_len=40000)
    cut(b, "bf16", 2, 16, 40, 4, 10, torch.rand(len(HELD), 2, b.max_len, generator=g), in_place=True)


def test_evict_in_place_masses_and_own_pages():
    b = Batch([(0, 50), (0, 10), (0, 500), (0, 64)], 16)
    masses = torch.rand(4, 2, b.max_len, generator=torch.Generator().manual_seed(3))
    cut(b, "bf16", 2, 64, 64, 4, 8, masses, in_place=True, own_pages=(0, 1, 3))
    cut(b, "f32", 2, 64, 64, 4, 8, masses, own_pages=(1,))


def test_evict_bad_pages_and_bounds():
    b = Batch([(0, 90), (0, 70)], 16)
    masses = torch.rand(2, 1, b.max_len, generator=torch.Generator().manual_seed(3))
    k, v = (torch.randn(b.n_pages + 4, 1, 16, 16, device=DEV) for _ in range(2))
    before = k.clone(), v.clone()
    to_table = np.array([[b.n_pages, -1], [b.n_pages + 4, b.n_pages + 1]], np.int32)
    b.table[0, :] = -1                                        # sequence 0 reads zeros; half of both targets is nowhere
    kept, out = torch.zeros(2, 1, 32, dtype=torch.int32, device=DEV), torch.zeros(2, 1, 32, device=DEV)
    vb.vla_paged_evict(vb.make_paged_cache(k, v), b.on_device(), masses.to(DEV), 0, 4, to_device(to_table), kept, out)
    at = kept[1, 0, 16:].long().cpu().numpy()
    for pool, old in ((k, before[0]), (v, before[1])):
        old[b.n_pages] = 0
        old[b.n_pages + 1, 0] = torch.stack([old[b.table[1, j // 16], 0, j % 16] for j in at])
        assert torch.equal(pool, old)
    b.max_len = 64                                            # positions from max_len on are not there
    lens = torch.zeros(2, dtype=torch.int32, device=DEV)
    vb.vla_paged_evict(vb.make_paged_cache(k, v), b.on_device(), masses.to(DEV), 0, 4, to_device(to_table), kept, out, lens)
    assert lens.tolist() == [32, 32] and kept[:, 0].max().item() == 63 and kept[:, 0, -4:].tolist() == [[60, 61, 62, 63]] * 2


@BOTH
@pytest.mark.parametrize("n,length", [(2, 90), (40, 150)])
def test_rows_left_out_read_no_scores(dtype, n, length):
    """A row whose lse is -inf adds nothing, also where K is NaN or its scores are infinite."""
    b = Batch([(n, length)], 16)
    pools = [p.to(DEV) for p in pools_of(b, dtype, 2, 64, 3)]
    pools[0][:, :, 3] = float("nan")
    pools[0][:, :, 5] = float("inf")
    q = torch.randn(b.n_rows, 4, 64, generator=torch.Generator().manual_seed(1)).to(TYPES[dtype]).to(DEV)
    cache, batch, mask = vb.make_paged_cache(*pools), b.on_device(), vb.make_paged_mask(0.125)
    old = torch.rand(1, 2, length, generator=torch.Generator().manual_seed(2)).to(DEV)
    mass, ws = old.clone(), torch.empty(vb.vla_paged_weights_workspace_bytes(cache, batch, mask, 4), dtype=torch.uint8, device=DEV)
    vb.vla_paged_weights(cache, batch, mask, q, torch.full((n, 4), -float("inf"), device=DEV), mass, ws)
    assert torch.equal(mass[..., :length - n], old[..., :length - n]) and not mass[..., length - n:].any()


@BOTH
@pytest.mark.parametrize("n_seq", [70, 300, 2049])
def test_weights_of_many_sequences(dtype, n_seq):
    """Equal shares found behind the first 64 sequences; above 2048 of them, chunks of each."""
    weigh(Batch([(1 if i % 5 else 0, 1 + 37 * i % (300 if n_seq < 100 else 70)) for i in range(n_seq)], 16, padding=3), dtype, 2, 1, 32)
    if n_seq == 2049:
        weigh(Batch([(1, 700)] + [(1, 3)] * 2048, 16), dtype, 1, 1, 16)
