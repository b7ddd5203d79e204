"""The operators that read less per token as a rollout uses them: trees of drafts through the decoder, decoding on selected pages, caches cut by weight; and all of them in captured graphs."""
import numpy as np
import pytest
import torch

import vla_inputs as vi
from paged_less_ref import pools_of, random_tree
from paged_ref import DEV, TYPES, Batch
from paper_2510_06710_amd import binding as vb
from paper_2510_06710_amd.harness import PagedRollout, Rollout
from parity import TOL

pytestmark = pytest.mark.gpu
SHAPES = {"f32": vi.ModelShape(n_layers=2, hidden=256, n_heads=4, ffn=512, vocab=1024, dtype="f32"), "bf16": vi.ModelShape(n_layers=2, hidden=256, n_heads=2, ffn=512, vocab=1024, dtype="bf16")}
LENGTHS = [(5, 3), (0, 1), (48, 16), (31, 2), (100, 29)]


def setup(shape, lengths=LENGTHS, seed=3):
    run = Rollout(vi.SynthModel(shape, seed, device=DEV), 4, 16, value_b=vi.VALUE_BIAS)
    obs = [vi.observation(vi.Workload("w", shape, 1, p, t, 4), seed + i, device=DEV) for i, (p, t) in enumerate(lengths)]
    return run, [p[0] for p, _ in obs], [t[0] for _, t in obs]


def started(run, patches, ids, n_pages=96, **k):
    paged = PagedRollout(run, n_pages, 16, **k)
    return paged, paged.prefill(patches, ids)[1]


def first_id(run):
    return run.shape.vocab - vb.VLA_N_BINS


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_drafts_are_what_decoding_gives(name):
    run, patches, ids = setup(SHAPES[name])
    plain, logits = started(run, patches, ids)
    bins, _, _, steps = plain.decode(logits, 30)
    want = (bins + first_id(run)).tolist()
    top = steps.sort(dim=2, descending=True).values
    sure = (top[..., 0] - top[..., 1] > 4 * TOL[name]["logits"]).int().cumprod(1).sum(1).tolist()          # greedy choices, from the first on, that rounding cannot turn over
    assert sum(sure) > (100 if name == "f32" else 4)
    paged, logits = started(run, patches, ids)
    rng, n = np.random.default_rng(1), len(ids)
    have = [[int(b)] for b in (logits.argmax(1) + first_id(run)).tolist()]
    while min(len(h) for h in have) < 6:
        tokens, parents = [], []
        for i, h in enumerate(have):
            # some of what will come (for one sequence none of it), among drafts that will not
            right, tree, wanted = want[i][len(h):len(h) + int(rng.integers(0, 4)) if i else len(h)], [h[-1]], [-1]
            at = 0
            for token in right:
                for _ in range(int(rng.integers(0, 3))):
                    tree.append(first_id(run) + (token - first_id(run) + 1 + int(rng.integers(0, 200))) % 256)
                    wanted.append(at)
                tree.append(token)
                wanted.append(at)
                at = len(tree) - 1
            tokens.append(tree), parents.append(wanted)
        before = list(paged.length)
        new = paged.decode_drafts(tokens, parents)
        for i in range(n):
            assert paged.length[i] == before[i] + len(new[i])
            have[i] += new[i]
            m = min(len(have[i]), sure[i])
            assert have[i][:m] == want[i][:m], i
    # what is in the cache now is what decoding has there: the next logits are the same to the rounding of two evaluations
    _, a, _ = paged.forward(list(range(n)), torch.tensor([h[-1] for h in have], dtype=torch.int32, device=DEV), [1] * n)
    for i in range(n):
        if len(have[i]) < sure[i]:
            assert (a[i] - steps[i, len(have[i])]).abs().max().item() <= 2 * TOL[name]["logits"]


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_sampled_drafts_and_long_trees(name):
    """With u per node the sampled path is that of sampling one by one; a tree of 70 nodes."""
    run, patches, ids = setup(SHAPES[name], [(5, 3), (40, 9)])
    paged, logits = started(run, patches, ids)
    tokens = [[int(t) for t in torch.randint(first_id(run), run.shape.vocab, (k,), generator=torch.Generator().manual_seed(k))] for k in (70, 1)]
    parents = [random_tree(70, np.random.default_rng(2)), [-1]]
    for tree in range(2):
        u = torch.rand(71, generator=torch.Generator().manual_seed(3 + tree)).to(DEV)
        before = list(paged.length)
        out = paged.decode_drafts(tokens, parents, temperature=1.6, top_k=40, u=u)
        assert [l - b for l, b in zip(paged.length, before)] == [len(o) for o in out] and all(first_id(run) <= x < run.shape.vocab for o in out for x in o)


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_selected_pages(name):
    run, patches, ids = setup(SHAPES[name])
    plain, logits = started(run, patches, ids)
    want = plain.decode(logits, 4)
    for select in (64, 9, 3, 2, 1):
        paged, logits = started(run, patches, ids)
        bins, logp, kept, z = paged.decode(logits, 4, select=select)
        off = (z - want[3]).abs()
        whole = [i for i, (p, t) in enumerate(LENGTHS) if (p + t + 3 + 15) // 16 <= select]          # all of the sequence's pages are selected
        assert torch.isfinite(z).all()
        if whole:
            same = torch.equal(bins[whole], want[0][whole])
            assert off[whole][:, :2 if same else 1].max().item() <= 2 * TOL[name]["logits"]
    assert off[-1].max().item() > 1e-3                        # one page of nine: other logits


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_evict_is_a_window_where_the_last_stay(name):
    """One layer: keys and values do not depend on what came before, rotated scores on distances alone; so a cache cut to its last positions is a prefill of these."""
    s = SHAPES[name]
    shape = vi.ModelShape(n_layers=1, hidden=s.hidden, n_heads=s.n_heads, ffn=s.ffn, vocab=s.vocab, dtype=s.dtype)
    run, _, ids = setup(shape, [(0, 60), (0, 7), (0, 130)])
    keep = 25
    paged, logits = started(run, [None] * 3, ids, weigh=True)
    assert paged.shift == [0] * 3 and torch.allclose(paged.mass.sum(3)[0].cpu(), torch.tensor([[60.0], [7.0], [130.0]]).expand(3, s.n_heads), rtol=1e-3)
    held = sum(len(p) for p in paged.pages)
    paged.evict(keep, recent=keep)
    assert paged.length == [25, 7, 25] and paged.shift == [35, 0, 105] and sum(len(p) for p in paged.pages) + len(paged.free) == 96 and sum(len(p) for p in paged.pages) < held
    short, _ = started(run, [None] * 3, [t[-keep:] for t in ids])
    token = torch.tensor([first_id(run) + 3, first_id(run) + 9, first_id(run) + 77], dtype=torch.int32, device=DEV)
    for _ in range(3):
        a, b = paged.forward([0, 1, 2], token, [1] * 3)[1], short.forward([0, 1, 2], token, [1] * 3)[1]
        assert (a - b).abs().max().item() <= 2 * TOL[name]["logits"]
        token = token + 1
    # drafts behind a cut cache, whose rotation counts on from where the cache was: a chain of two is two steps
    new = paged.decode_drafts([[int(t), int(t) + 1] for t in token.tolist()], [[-1, 0]] * 3)
    want = short.decode_drafts([[int(t), int(t) + 1] for t in token.tolist()], [[-1, 0]] * 3)
    assert new == want and paged.length == short.length


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_evict_keeps_what_had_weight(name):
    run, patches, ids = setup(SHAPES[name], [(0, 90), (3, 20), (40, 30)])
    paged, logits = started(run, patches, ids, weigh=True)
    plain, same = started(run, patches, ids)
    assert (logits - same).abs().max().item() <= 2 * TOL[name]["logits"]
    mass, keys = paged.mass.clone(), [p.clone() for p in paged.pools]
    pages, lens = [list(p) for p in paged.pages], list(paged.length)
    paged.evict(40, first=2, recent=8)
    assert paged.length == [40, 23, 40]
    for l in range(run.shape.n_layers):
        for s in range(3):
            for h in range(run.shape.n_heads):
                m = mass[l, s, h, :lens[s]].double().cpu().numpy()
                order = sorted(range(lens[s]), key=lambda j: (not (j < 2 or j >= lens[s] - 8), -m[j], j))
                at = sorted(order[:40]) if lens[s] > 40 else range(lens[s])
                for pool, old in zip(paged.pools, keys):
                    was = torch.stack([old[l, pages[s][j // 16], h, j % 16] for j in at])
                    now = torch.stack([pool[l, paged.pages[s][i // 16], h, i % 16] for i in range(len(at))])
                    assert torch.equal(was, now)
    bins, _, _, z = paged.decode(logits, 5)                   # and on it goes
    assert torch.isfinite(z).all() and paged.length == [44, 27, 44]
    paged.evict(30)
    assert paged.length == [30, 27, 30] and paged.shift == [90 + 4 - 30, 0, 70 + 4 - 30]


def test_refusals():
    run, patches, ids = setup(SHAPES["f32"], [(0, 20), (3, 5)])
    paged, logits = started(run, patches, ids)
    for call in (lambda: paged.evict(10), lambda: paged.decode_drafts([[1]], [[-1]]), lambda: paged.decode_drafts([[1, 2], [3]], [[-1, 1], [-1]]), lambda: paged.decode_drafts([[1], []], [[-1], []]),
                 lambda: paged.decode_drafts([[1], [2]], [[-1], [-1]], u=torch.zeros(3, device=DEV)), lambda: paged.decode(logits, 2, select=-1)):
        with pytest.raises(ValueError):
            call()
    heavy, logits = started(run, patches, ids, n_pages=4, weigh=True)
    before = [list(p) for p in heavy.pages], list(heavy.length), list(heavy.free)
    for call in (lambda: heavy.evict(17), lambda: heavy.evict(0), lambda: heavy.evict(4, 3, 3), lambda: heavy.prefill_group(None, ids[0], 2), lambda: heavy.forward([1], torch.zeros(1, dtype=torch.int32, device=DEV), [1]),
                 lambda: heavy.decode(logits, 2, select=3)):
        with pytest.raises(ValueError):
            call()
        assert (heavy.pages, heavy.length, heavy.free) == before
    heavy.evict(16)                                           # one page wanted, one free
    assert heavy.length == [16, 8] and len(heavy.free) == 2


def test_forward_rows_refuses():
    run, _, ids = setup(SHAPES["f32"], [(0, 4)])
    s = run.shape
    pools = [torch.zeros(s.n_layers, 4, s.n_heads, 16, s.head_dim, device=DEV) for _ in range(2)]
    cache, i = vb.make_paged_cache(pools[0][0], pools[1][0]), lambda *v: torch.tensor(v, dtype=torch.int32, device=DEV)
    batch = vb.make_paged_batch(i(0, 4), i(4), i(0)[None], 4, 4, 16)
    seen, mass, bounds = torch.zeros(4, 1, dtype=torch.int32, device=DEV), torch.zeros(2, 1, s.n_heads, 16, device=DEV), torch.zeros(2, 4, s.n_heads, 2, s.head_dim, device=DEV)
    ws, out = torch.empty(1 << 24, dtype=torch.uint8, device=DEV), torch.zeros(4, 256, device=DEV)
    call = lambda rows, ws=ws, out=out: vb.vla_forward_paged_rows(run.model.handle, cache, pools[0][0].numel(), 2, batch, rows, i(1, 2, 3, 4), ws, out)
    for bad in (dict(seen=seen, mass=mass), dict(seen=seen, bounds=bounds, n_select=3), dict(bounds=bounds, n_select=3, mass=mass), dict(n_select=3), dict(bounds=bounds, n_select=1),
                dict(bounds=bounds, n_select=3, recent=0), dict(mass=torch.zeros(2, 1, s.n_heads, 15, device=DEV)), dict(mass=mass[:1]), dict(seen=seen[:3]), dict(position=i(1)),
                dict(bounds=bounds[:1]), dict(prefix_len=i(1, 2)), dict(seen=seen, prefix_len=i(2))):
        with pytest.raises(vb.VlaError):
            call(vb.make_paged_rows(**bad))
    with pytest.raises(vb.VlaError):
        call(vb.make_paged_rows(), ws=ws[:256])
    with pytest.raises(vb.VlaError):
        call(vb.make_paged_rows(), out=out[:3])
    call(vb.make_paged_rows(seen=seen + 1))
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 9, 40])
def test_replays(dtype, rows):
    """All of them in one captured graph, replayed with other lengths, tables, trees and inputs, against eager calls on the same."""
    n, kv, heads, d, page, entries, keep, most = 4, 2, 8, 64, 16, 20, 48, 6
    g = torch.Generator().manual_seed(0)
    T, I = TYPES[dtype], torch.int32
    total, cap = n * rows, entries * page
    z = lambda *shape, dtype=I: torch.zeros(*shape, dtype=dtype, device=DEV)
    k, v = z(n * (entries + 3), kv, page, d, dtype=T), z(n * (entries + 3), kv, page, d, dtype=T)
    start, lens, table, to = torch.arange(0, total + 1, rows, dtype=I, device=DEV), z(n), z(n, entries), z(n, 3)
    parent, ids, chosen, position, seen = z(total), z(total), z(total), z(total), z(total, 2)
    q, ql, kl, vl = z(total, heads, d, dtype=T), z(total, heads, d, dtype=T), z(total, kv, d, dtype=T), z(total, kv, d, dtype=T)
    out, tree_out, some, lse = z(total, heads, d, dtype=T), z(total, heads, d, dtype=T), z(total, heads, d, dtype=T), z(total, heads, dtype=torch.float32)
    bounds, selected, mass = z(k.shape[0], kv, 2, d, dtype=T), z(total, kv, most), z(n, kv, cap, dtype=torch.float32)
    kept, mass_out, path, count, follow, new_len = z(n, kv, keep), z(n, kv, keep, dtype=torch.float32), z(n, rows), z(n), z(n), z(n)
    freq = (10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32)).to(DEV)
    cache, batch, mask, rotary = vb.make_paged_cache(k, v), vb.make_paged_batch(start, lens, table, total, rows, cap), vb.make_paged_mask(d ** -0.5), vb.make_rotary(freq)
    empty = lambda size: torch.empty(size, dtype=torch.uint8, device=DEV)
    ws = [empty(vb.vla_paged_attention_workspace_bytes(cache, batch, mask, heads)), empty(vb.vla_paged_select_workspace_bytes(cache, batch)),
          empty(vb.vla_paged_sparse_attention_workspace_bytes(cache, batch, mask, heads, most)), empty(vb.vla_paged_weights_workspace_bytes(cache, batch, mask, heads))]
    given = [k, v, mass]
    results = [k, v, mass, q, out, tree_out, some, lse, bounds, selected, kept, mass_out, path, count, follow, new_len, position, seen]

    def step():
        vb.vla_paged_tree(cache, batch, parent, seen, position)
        vb.vla_paged_append_at(cache, batch, rotary, position, ql, kl, vl, q)
        vb.vla_paged_tree_attention(cache, batch, mask, seen, q, tree_out, None, ws[0])
        vb.vla_paged_attention(cache, batch, mask, q, out, lse, ws[0])
        vb.vla_paged_weights(cache, batch, mask, q, lse, mass, ws[3])
        vb.vla_paged_bounds(cache, batch, bounds)
        vb.vla_paged_select(cache, batch, bounds, q, selected, 1, 1, ws[1])
        vb.vla_paged_sparse_attention(cache, batch, mask, selected, q, some, None, ws[2])
        vb.vla_paged_accept(cache, 1, 0, batch, parent, ids, chosen, path, count, follow, new_len)
        vb.vla_paged_evict(cache, batch, mass, 1, 5, to, kept, mass_out)

    def inputs(seed):
        r, rng = torch.Generator().manual_seed(seed), np.random.default_rng(seed)
        lens.copy_(torch.randint(rows, cap + 1, (n,), generator=r))
        own = torch.randperm(k.shape[0], generator=r).view(n, entries + 3)
        table.copy_(own[:, :entries]), to.copy_(own[:, entries:])
        parent.copy_(torch.tensor([p for _ in range(n) for p in random_tree(rows, rng)]))
        ids.copy_(torch.randint(0, 3, (total,), generator=r)), chosen.copy_(torch.randint(0, 3, (total,), generator=r))
        for x in (ql, kl, vl):
            x.copy_(torch.randn(x.shape, generator=r))
        return [torch.randn(x.shape, generator=r).abs().to(x.dtype).to(DEV) if x is mass else torch.randn(x.shape, generator=r).to(x.dtype).to(DEV) for x in given]

    inputs(0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (1, 2, 3, 1):
        fill, got = inputs(seed), []
        for call in (graph.replay, step):
            for x in results:
                x.zero_()
            for x, f in zip(given, fill):
                x.copy_(f)
            for w in ws:
                w.fill_(255)
            call()
            torch.cuda.synchronize()
            got.append([x.clone() for x in results])
        assert all(torch.equal(a, b) for a, b in zip(*got)) and torch.isfinite(got[0][5].float()).all() and got[0][13].min() >= 1


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_two_streams_at_once(dtype):
    """Calls on two streams, each with its own workspace, on one cache that both read: what they give one after the other."""
    b = Batch([(1, 900), (1, 333), (1, 64)], 16)
    pools, kv, heads, d = [p.to(DEV) for p in pools_of(b, dtype, 2, 64, 1)], 2, 8, 64
    cache, batch, mask = vb.make_paged_cache(*pools), b.on_device(), vb.make_paged_mask(0.125)
    bounds = torch.zeros(b.n_pages, kv, 2, d, dtype=TYPES[dtype], device=DEV)
    vb.vla_paged_bounds(cache, batch, bounds)
    empty = lambda size: torch.empty(size, dtype=torch.uint8, device=DEV)
    states = []
    for i in range(2):
        q = torch.randn(3, heads, d, generator=torch.Generator().manual_seed(i)).to(TYPES[dtype]).to(DEV)
        states.append(dict(q=q, out=torch.zeros_like(q), selected=torch.zeros(3, kv, 7, dtype=torch.int32, device=DEV), mass=torch.zeros(3, kv, 900, device=DEV), lse=torch.zeros(3, heads, device=DEV),
                           seen=torch.ones(3, 1, dtype=torch.int32, device=DEV), tree=torch.zeros_like(q),
                           ws=[empty(vb.vla_paged_attention_workspace_bytes(cache, batch, mask, heads)), empty(vb.vla_paged_select_workspace_bytes(cache, batch)),
                               empty(vb.vla_paged_sparse_attention_workspace_bytes(cache, batch, mask, heads, 7)), empty(vb.vla_paged_weights_workspace_bytes(cache, batch, mask, heads))]))

    def calls(s, stream):
        vb.vla_paged_select(cache, batch, bounds, s["q"], s["selected"], 1, 1, s["ws"][1], stream=stream)
        vb.vla_paged_sparse_attention(cache, batch, mask, s["selected"], s["q"], s["out"], None, s["ws"][2], stream=stream)
        vb.vla_paged_tree_attention(cache, batch, mask, s["seen"], s["q"], s["tree"], s["lse"], s["ws"][0], stream=stream)
        vb.vla_paged_weights(cache, batch, mask, s["q"], s["lse"], s["mass"], s["ws"][3], stream=stream)

    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        for s, st in zip(states, streams):
            s["mass"].zero_()
    torch.cuda.synchronize()
    for s, st in zip(states, streams):
        calls(s, st)
    torch.cuda.synchronize()
    first = [[s[x].clone() for x in ("selected", "out", "tree", "mass")] for s in states]
    for s in states:
        s["mass"].zero_()
        calls(s, None)
    torch.cuda.synchronize()
    for s, f in zip(states, first):
        assert all(torch.equal(s[x], y) for x, y in zip(("selected", "out", "tree", "mass"), f))
