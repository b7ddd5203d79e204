"""Trees of drafted tokens: what their nodes see, the attention to them, the accepted path and its K and V, rotation by depth.

Tolerances of the attention: those of test_gpu_paged_attention.py, where weights enter the product with V with a bf16 tail (2^-16 A) whatever the
number of rows.  Everything else is whole numbers or moved bits."""
import numpy as np
import pytest
import torch

from paged_less_ref import ancestors, bits, check_rows, follow, pools_of, random_tree, rows_of, to_device
from paged_ref import DEV, TYPES, Batch, rotated
from paper_2510_06710_amd import binding as vb

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("dtype", ["bf16", "f32"])
SMALL = [(1, 1), (4, 9), (0, 40), (3, 3), (8, 100), (2, 33), (1, 70)]
WIDE = [(33, 40), (1, 200), (64, 300), (0, 5), (70, 70), (100, 131)]


def trees(b, seed):
    rng = np.random.default_rng(seed)
    return [random_tree(n, rng) if n else [] for n, _ in b.spec]


def view_of(b, cache=None):
    k = torch.zeros(b.n_pages, 1, b.page, 16, device=DEV) if cache is None else None
    return cache or vb.make_paged_cache(k, k.clone())


@pytest.mark.parametrize("spec", [SMALL, WIDE, [(1024, 1500), (1, 1), (1000, 1000)]])
@pytest.mark.parametrize("more", [0, 3])
def test_what_nodes_see(spec, more):
    b = Batch(spec, 64, padding=2)
    tree = trees(b, 1)
    for t in tree:                                            # a parent that is no earlier node: none
        if len(t) > 5:
            t[3], t[4] = 4, -7
    words = min(32, -(-b.max_rows // 32) + more)
    parent = np.array([p for t in tree for p in t] + [0] * 2, np.int32)
    seen, position = torch.full((b.n_rows, words), -77, dtype=torch.int32, device=DEV), torch.full((b.n_rows,), -77, dtype=torch.int32, device=DEV)
    vb.vla_paged_tree(view_of(b), b.on_device(), to_device(parent), seen, position)
    want, depth = np.full((b.n_rows, words), -77, np.int32), np.full(b.n_rows, -77)
    for s, t in enumerate(tree):
        if t:
            a = b.start[s]
            see, deep = ancestors(t)
            want[a:a + len(t)], depth[a:a + len(t)] = bits(see, words), b.spec[s][1] - len(t) + deep
    assert np.array_equal(seen.cpu().numpy(), want) and np.array_equal(position.cpu().numpy(), depth)


def attend(b, dtype, heads, kv, d, see, cap=0.0, shared=0, seed=0, layout="packed"):
    """see[s] [n, n]: which of a sequence's new rows its rows see."""
    pools = pools_of(b, dtype, kv, d, seed)
    q = torch.randn(b.n_rows, heads, d, generator=torch.Generator().manual_seed(seed + 1)).to(TYPES[dtype])
    words = max(1, -(-b.max_rows // 32))
    rows = np.full((b.n_rows, words), -1, np.int32)           # (padding sees everything, and nothing)
    for s, m in enumerate(see):
        rows[b.start[s]:b.start[s + 1]] = bits(m, words) if len(m) else rows[:0]
        if len(m):                                            # bits of rows that are not there mean nothing
            rows[b.start[s]:b.start[s + 1]] |= bits(np.tile(np.arange(32 * words) >= len(m), (len(m), 1)), words)
    qd, out = q.to(DEV), torch.full((b.n_rows, heads, d), -77.0, dtype=TYPES[dtype], device=DEV)
    if layout == "unaligned":
        big = torch.zeros(b.n_rows, heads * d + 5, dtype=TYPES[dtype], device=DEV)
        big[:, 3:3 + heads * d] = qd.view(b.n_rows, -1)
        qd = big[:, 3:3 + heads * d].unflatten(1, (heads, d))
        out = torch.full((b.n_rows, heads * d + 7), -77.0, dtype=TYPES[dtype], device=DEV)[:, 1:1 + heads * d].unflatten(1, (heads, d))
    lse = torch.full((b.n_rows, heads), -77.0, device=DEV)
    cache, batch, mask = vb.make_paged_cache(*[p.to(DEV) for p in pools]), b.on_device(), vb.make_paged_mask(d ** -0.5, cap, shared_len=shared)
    ws = torch.full((vb.vla_paged_attention_workspace_bytes(cache, batch, mask, heads),), 255, dtype=torch.uint8, device=DEV)
    vb.vla_paged_tree_attention(cache, batch, mask, to_device(rows), qd, out, lse, ws)
    first = out.clone()
    vb.vla_paged_tree_attention(cache, batch, mask, to_device(rows), qd, out, None, ws)
    assert torch.equal(first, out)

    def seen_by(row, s, p, h):
        n, length = b.spec[s]
        return np.concatenate([np.arange(length - n), length - n + np.nonzero(see[s][row - b.start[s]])[0]])

    want = rows_of(b, q.double().numpy(), *[p.double().numpy() for p in pools], d ** -0.5, cap, seen_by)
    check_rows(b, dtype, d, cap, out, lse, want, max(l for _, l in b.spec) or 1)


@BOTH
@pytest.mark.parametrize("heads,kv,d", [(4, 4, 64), (8, 2, 128), (6, 2, 80), (4, 2, 256), (40, 1, 32)])
@pytest.mark.parametrize("spec", [SMALL, WIDE])
def test_attention(dtype, heads, kv, d, spec):
    b = Batch(spec, 16, padding=2)
    attend(b, dtype, heads, kv, d, [ancestors(t)[0] if t else [] for t in trees(b, 2)])
    b = Batch(spec, 64)
    attend(b, dtype, heads, kv, d, [ancestors(t)[0] if t else [] for t in trees(b, 3)], cap=3.0)


@BOTH
@pytest.mark.parametrize("spec", [SMALL, WIDE])
def test_any_bits_and_layouts(dtype, spec):
    rng = np.random.default_rng(7)
    for layout in ("packed", "unaligned"):
        b = Batch(spec, 32)
        attend(b, dtype, 4, 2, 64, [rng.random((n, n)) < 0.4 for n, _ in spec], layout=layout)
    b = Batch([(5, 5), (40, 40), (1, 1)], 16)                 # nothing in the cache, and some rows see none of the others either
    attend(b, dtype, 4, 2, 64, [np.zeros((5, 5), bool), rng.random((40, 40)) < 0.02, np.zeros((1, 1), bool)])


@BOTH
def test_long_contexts_and_shared_prefix(dtype):
    see = lambda b: [ancestors(t)[0] if t else [] for t in trees(b, 4)]
    for spec in ([(7, 5000)], [(61, 3001), (3, 17), (20, 800)], [(300, 700)]):
        b = Batch(spec, 64)
        attend(b, dtype, 8, 2, 64, see(b))
    for spec, heads, kv in (([(5, 70 + 64), (1, 65), (8, 64 + 8), (0, 90), (3, 200)], 4, 2), ([(40, 64 + 40 + i) for i in range(9)], 8, 1)):
        b = Batch(spec, 32, shared=64)
        attend(b, dtype, heads, kv, 128, see(b), shared=64)


@BOTH
def test_a_chain_is_the_causal_mask(dtype):
    for spec in (SMALL, [(n, l) for n, l in WIDE]):
        b = Batch(spec, 16)
        pools, q = pools_of(b, dtype, 2, 64, 5), torch.randn(b.n_rows, 4, 64, generator=torch.Generator().manual_seed(6)).to(TYPES[dtype]).to(DEV)
        words = -(-b.max_rows // 32)
        rows = np.concatenate([bits(np.tril(np.ones((n, n), bool)), words) for n, _ in spec if n])
        cache, batch, mask = vb.make_paged_cache(*[p.to(DEV) for p in pools]), b.on_device(), vb.make_paged_mask(0.125)
        ws = torch.empty(vb.vla_paged_attention_workspace_bytes(cache, batch, mask, 4), dtype=torch.uint8, device=DEV)
        tree, plain = torch.zeros_like(q), torch.zeros_like(q)
        vb.vla_paged_tree_attention(cache, batch, mask, to_device(rows), q, tree, None, ws)
        vb.vla_paged_attention(cache, batch, mask, q, plain, None, ws)
        # each is off by half a step of the output, and a bf16 prompt's weights by 2^-8 of A <= 4.5 (the largest of 10^5 normal values) at most
        assert (tree.float() - plain.float()).abs().max().item() <= (3 * 2.0 ** -8 if dtype == "bf16" else 2.0 ** -18) * 4.5


@BOTH
@pytest.mark.parametrize("spec", [SMALL, WIDE, [(1024, 1100), (1, 1)]])
@pytest.mark.parametrize("kv,d,layers", [(2, 64, 3), (1, 16, 1), (8, 256, 2)])
def test_accept(dtype, spec, kv, d, layers):
    b, rng = Batch(spec, 16, padding=2), np.random.default_rng(kv)
    if max(n for n, _ in spec) == 1024 and d > 64:
        d = 16
    tree = trees(b, 8)
    ids = rng.integers(0, 3, b.n_rows).astype(np.int32)       # few tokens: siblings that are alike, long paths
    chosen = rng.integers(-1, 3, b.n_rows).astype(np.int32)
    for s, t in enumerate(tree):                              # most nodes chose what one of their children, the last, carries
        for i, p in enumerate(t):
            if p >= 0 and rng.random() < 0.9:
                chosen[b.start[s] + p] = ids[b.start[s] + i]
    parent = np.array([p for t in tree for p in t] + [0] * 2, np.int32)
    pools = [torch.randn(layers, b.n_pages, kv, 16, d, generator=torch.Generator().manual_seed(i)).to(TYPES[dtype]) for i in range(2)]
    k, v = (p.to(DEV) for p in pools)
    path, count = torch.full((len(spec), b.max_rows), -77, dtype=torch.int32, device=DEV), torch.full((len(spec),), -77, dtype=torch.int32, device=DEV)
    follow_up, new_len = count.clone(), count.clone()
    vb.vla_paged_accept(vb.make_paged_cache(k[0], v[0]), layers, k[0].numel(), b.on_device(), *map(to_device, (parent, ids, chosen)), path, count, follow_up, new_len)
    longest = 0
    for s, (n, length) in enumerate(spec):
        a = b.start[s]
        want = follow(tree[s], ids[a:a + n], chosen[a:a + n])
        longest = max(longest, len(want))
        assert path[s].tolist() == want + [-1] * (b.max_rows - len(want))
        assert count[s].item() == len(want) and new_len[s].item() == length - n + len(want) and follow_up[s].item() == (chosen[a + want[-1]] if want else -1)
        for pool in pools:
            rows = [pool[:, b.table[s, (length - n + i) // 16], :, (length - n + i) % 16].clone() for i in want]
            for to, x in enumerate(rows):
                pool[:, b.table[s, (length - n + to) // 16], :, (length - n + to) % 16] = x
    assert torch.equal(k.cpu(), pools[0]) and torch.equal(v.cpu(), pools[1])
    assert longest > 1


def test_accept_moves_nothing_without_layers_or_pages():
    b = Batch([(4, 20), (0, 0)], 16)
    k = torch.randn(b.n_pages, 1, 16, 16, device=DEV)
    before, path, count = k.clone(), torch.zeros(2, 4, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)
    args = [to_device(np.array(x, np.int32)) for x in ([-1, 0, 0, 2], [0, 5, 6, 7], [6, 1, 7, 1])]
    vb.vla_paged_accept(vb.make_paged_cache(k, k), 0, 0, b.on_device(), *args, path, count)
    assert path.tolist() == [[0, 2, 3, -1], [-1] * 4] and count.tolist() == [3, 0] and torch.equal(k, before)
    b.table[0, 1] = b.n_pages                                 # the rows' page is not there: nothing is written, and what comes from there is zero
    vb.vla_paged_accept(vb.make_paged_cache(k, k), 1, 0, b.on_device(), *args, path, count)
    assert torch.equal(k, before)
    b.spec[0] = (4, 2)                                        # rows at negative positions
    new_len = count.clone()
    vb.vla_paged_accept(vb.make_paged_cache(k, k), 1, 0, b.on_device(), *args, path, count, None, new_len)
    before[b.table[0, 0], :, 0] = before[b.table[0, 0], :, 1]          # path[2] = 3 lies at 1 and goes to 0; path[1] would go to -1
    assert torch.equal(k, before) and new_len.tolist() == [1, 0]


@BOTH
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_by_given_positions(dtype, interleaved):
    b = Batch(SMALL, 16, padding=1)
    g = torch.Generator().manual_seed(9)
    q, k, v = (torch.randn(b.n_rows, h, 64, generator=g).to(DEV) for h in (4, 2, 2))
    freq = 10000.0 ** (-np.arange(32) / 32)
    place = np.zeros(b.n_rows, np.int32)
    for row, _, p in b.rows():
        place[row] = p
    got = []
    for position in (None, place, place // 2 + 3, place + 10 ** 6):
        pools = [torch.zeros(b.n_pages, 2, 16, 64, dtype=TYPES[dtype], device=DEV) for _ in range(2)]
        out = torch.zeros(b.n_rows, 4, 64, dtype=TYPES[dtype], device=DEV)
        cache, rotary = vb.make_paged_cache(*pools), vb.make_rotary(to_device(freq), interleaved=interleaved)
        if position is None:
            vb.vla_paged_append(cache, b.on_device(), rotary, q, k, v, out)
        else:
            vb.vla_paged_append_at(cache, b.on_device(), rotary, to_device(position), q, k, v, out)
            want, mag = rotated(q.double().cpu().numpy(), position.astype(float), None, 0.0, freq, interleaved, 1.0)
            # cos and sin in fp32 (half a step each, of values up to 1), one product and one sum more, the output's rounding
            tol = mag * 4 * 2.0 ** -24 + (np.abs(want) * 2.0 ** -8 if dtype == "bf16" else 0)
            assert (np.abs(out.double().cpu().numpy() - want)[:b.live] <= tol[:b.live]).all()
            rows = np.stack([pools[0].double().cpu().numpy()[b.table[s, p // 16], :, p % 16] for _, s, p in b.rows()])
            want, mag = rotated(k.double().cpu().numpy(), position.astype(float), None, 0.0, freq, interleaved, 1.0)
            assert (np.abs(rows - want[:b.live]) <= (mag * 4 * 2.0 ** -24 + (np.abs(want) * 2.0 ** -8 if dtype == "bf16" else 0))[:b.live]).all()
        got.append((out, *pools))
    assert all(torch.equal(x, y) for x, y in zip(got[0], got[1]))


def test_accept_where_rows_lie_before_the_cache():
    """More rows than positions: rows at negative positions are nowhere, those behind them move as always."""
    b = Batch([(6, 4)], 16)
    k = torch.randn(b.n_pages, 2, 16, 16, generator=torch.Generator().manual_seed(1))
    v, kd = 2 * k, k.to(DEV)
    vd = v.to(DEV)
    path, count = torch.zeros(1, 6, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    new_len = torch.zeros(1, dtype=torch.int32, device=DEV)
    args = [to_device(np.array(x, np.int32)) for x in ([-1, 0, 0, 2, 3, 4], [0, 5, 6, 7, 8, 9], [6, 1, 7, 8, 9, 1])]
    vb.vla_paged_accept(vb.make_paged_cache(kd, vd), 1, 0, b.on_device(), *args, path, count, None, new_len)
    assert path.tolist() == [[0, 2, 3, 4, 5, -1]] and count.item() == 5 and new_len.item() == 3
    for pool, got in ((k, kd), (v, vd)):
        page = b.table[0, 0]
        pool[page, :, 0:3] = pool[page, :, 1:4].clone()      # row path[i] is at path[i] - 2 and goes to i - 2
        assert torch.equal(got.cpu(), pool)


@BOTH
def test_attention_of_many_sequences(dtype):
    for n_seq, rows in ((70, 5), (300, 2), (2049, 1)):
        b = Batch([((i + 1) % (rows + 1), rows + 37 * i % (200 if n_seq < 100 else 40)) for i in range(n_seq)], 16, padding=2)
        attend(b, dtype, 2, 1, 32, [ancestors(t)[0] if t else [] for t in trees(b, 5)])
