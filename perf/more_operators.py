"""Operators that let a step on a paged KV cache read less per token, as measurable cases.

Trees of drafted tokens are attended to in one pass and the accepted path's keys and values moved together; single tokens attend to the
pages that a bound of their scores selects; caches are cut to the positions that past rows gave most weight.  `run` computes each operator
in elementary torch operations, or calls the library's (`own`).

Queries and values are N(0, 1); keys are too, but for the sparse cases', where a page's keys have a part in common, as neighbouring tokens
do.  Page tables are a random permutation of the pages, as after many sequences have come and gone.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
FIRST, RECENT = 1, 2                     # pages that every selection holds


def listed():
    return [
        # one robot's drafted action tokens: latency of the smallest tree
        dict(name="tree_one_row", op="tree", n_seq=1, rows=8, len=708, ragged=False, heads=32, kv_heads=8, dim=128, page=16, cap=0.0, shared=0, dtype="bf16"),
        # a ragged batch of drafts behind prompts of any length
        dict(name="tree_ragged_b32", op="tree", n_seq=32, rows=24, len=4096, ragged=True, heads=32, kv_heads=8, dim=128, page=16, cap=0.0, shared=0, dtype="bf16"),
        # a wide tree behind one long context, capped scores: the keys have to be split
        dict(name="tree_wide_long", op="tree", n_seq=1, rows=61, len=32768, ragged=False, heads=16, kv_heads=4, dim=128, page=64, cap=30.0, shared=0, dtype="bf16"),
        # one sequence's accepted path through all layers
        dict(name="accept_b1", op="accept", n_seq=1, rows=8, past=700, ragged=False, layers=32, kv_heads=8, dim=128, page=16, dtype="bf16"),
        # the accepted paths of a ragged batch with every head its own keys
        dict(name="accept_ragged_b64", op="accept", n_seq=64, rows=33, past=120, ragged=True, layers=16, kv_heads=32, dim=128, page=16, dtype="bf16"),
        # bounds of all pages of a few long prompts, as after their prefill
        dict(name="bounds_prefill_b4", op="bounds", n_seq=4, rows=32768, len=32768, ragged=True, kv_heads=8, dim=128, page=64, dtype="bf16"),
        # one token behind a very long history, of which it reads a thirtieth
        dict(name="sparse_long_b1", op="sparse", n_seq=1, rows=1, len=131072, ragged=False, heads=32, kv_heads=8, dim=128, page=64, select=64, cap=0.0, dtype="bf16"),
        # single tokens of a ragged batch of long sequences
        dict(name="sparse_ragged_b32", op="sparse", n_seq=32, rows=1, len=32768, ragged=True, heads=32, kv_heads=8, dim=128, page=32, select=64, cap=0.0, dtype="bf16"),
        # a decode step's weights added to those of the positions it read
        dict(name="weights_decode_b64", op="weights", n_seq=64, rows=1, len=4096, ragged=True, heads=32, kv_heads=8, dim=128, page=16, cap=0.0, window=0, dtype="bf16"),
        # a whole prompt's weights: matrix products
        dict(name="weights_prompt_4k", op="weights", n_seq=1, rows=4096, len=4096, ragged=False, heads=32, kv_heads=8, dim=128, page=16, cap=0.0, window=0, dtype="bf16"),
        # a long batch cut to an eighth
        dict(name="evict_b16", op="evict", n_seq=16, len=32768, ragged=True, keep=4096, recent=512, kv_heads=8, dim=128, page=64, dtype="bf16"),
        # a small fp32 decoder's cache of one sequence, odd sizes
        dict(name="evict_small_f32", op="evict", n_seq=1, len=1003, ragged=False, keep=250, recent=33, kv_heads=4, dim=80, page=16, dtype="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["tree", "tree", "accept", "bounds", "sparse", "sparse", "weights", "weights", "evict", "evict"])
    kv_heads, page, dim, dtype = rng.choice([1, 2, 4, 8]), rng.choice([16, 32, 64, 128]), rng.choice([64, 80, 128, 128, 256]), rng.choice(["bf16", "bf16", "f32"])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 7, 8])
    case = dict(op=op, ragged=rng.random() < 0.6, kv_heads=kv_heads, dim=dim, page=page, dtype=dtype)
    # positions whose K and V, and pairs of a row and a position whose products, a call of the largest listed one's time takes
    many = 19 * 10 ** 7 // (kv_heads * dim * (4 if dtype == "f32" else 2))
    pairs = 10 ** 10 // (heads * dim) // (8 if dtype == "f32" else 1)
    if op == "tree":
        n_seq = _log(rng, 1, 64)
        rows = _log(rng, 1, min(100, 2048 // n_seq))
        shared = page * _log(rng, 1, 2048 // page) if n_seq > 1 and rng.random() < 0.2 else 0
        length = shared + rows + _log(rng, 1, max(1, min(32768, many // n_seq, pairs // (rows * n_seq)))) - 1
        return dict(case, n_seq=n_seq, rows=rows, len=length, heads=heads, cap=rng.choice([0.0, 0.0, 20.0]), shared=shared)
    if op == "accept":
        n_seq, rows, past = _log(rng, 1, 64), _log(rng, 1, 100), _log(rng, 1, 300)
        return dict(case, n_seq=n_seq, rows=rows, past=past, layers=_log(rng, 1, max(1, min(32, 2 ** 29 // (kv_heads * dim * n_seq * (past + rows + page))))))
    if op == "bounds":
        n_seq = _log(rng, 1, 64)
        length = _log(rng, 1, many // n_seq)
        return dict(case, n_seq=n_seq, rows=rng.choice([1, length, _log(rng, 1, length)]), len=length)
    if op == "sparse":
        n_seq = _log(rng, 1, 32)
        length = _log(rng, 10, min(131072, 262144 // n_seq))
        return dict(case, n_seq=n_seq, rows=min(length, rng.choice([1, 1, 2, 5])), len=length, heads=heads,
                    select=_log(rng, FIRST + RECENT, max(FIRST + RECENT, min(2048, many // n_seq) // page)), cap=rng.choice([0.0, 0.0, 20.0]))
    if op == "weights":
        rows = 1 if rng.random() < 0.5 else _log(rng, 2, 2048)
        n_seq = _log(rng, 1, max(1, min(64, 2048 // rows)))
        length = rows + _log(rng, 1, max(1, min(32768, many // n_seq, pairs // (rows * n_seq)))) - 1
        return dict(case, n_seq=n_seq, rows=rows, len=length, heads=heads, cap=rng.choice([0.0, 0.0, 20.0]), window=rng.choice([0, 0, _log(rng, 1, length)]))
    n_seq = _log(rng, 1, 64)
    length = _log(rng, 4, min(65536, many // n_seq))
    keep = max(2, int(length * rng.uniform(0.05, 0.9)))
    return dict(case, n_seq=n_seq, len=length, keep=keep, recent=int(keep * rng.uniform(0.0, 0.5)))


def _lengths(case):
    """New rows and positions held, per sequence; fixed by the case, so that all seeds do the same work."""
    n, op = case["n_seq"], case["op"]
    gen = torch.Generator().manual_seed(n)
    most = case["past"] + case["rows"] if op == "accept" else case["len"]
    rows, least = case.get("rows", 0), case.get("shared", 0)
    if not case["ragged"]:
        return [min(rows, most - least)] * n, [most] * n
    held = torch.randint(least + 1, most + 1, (n,), generator=gen).tolist()
    held[-1] = most
    new = torch.randint(1, rows + 1, (n,), generator=gen).tolist() if rows > 1 else [rows] * n
    new[-1] = rows
    if op == "bounds" and rows == case["len"]:
        new = held
    return [min(r, l - least) for r, l in zip(new, held)], held


def _trees(case, rows):
    """Per sequence, its nodes' parents (the first is the committed token) and the path that will be accepted; fixed by the case."""
    gen = torch.Generator().manual_seed(case["n_seq"] + 1)
    parents, paths = [], []
    for n in rows:
        back = (torch.rand(n, generator=gen) ** 2 * 8).long().tolist()       # mostly of the last few nodes: chains with branches
        parents.append([-1] + [max(0, i - 1 - back[i]) for i in range(1, n)])
        node, path = int(torch.randint(0, n, (2,), generator=gen).max()), []
        while node >= 0:
            path.append(node)
            node = parents[-1][node]
        paths.append(path[::-1])
    return parents, paths


def _bits(parents, words):
    """Which nodes each node sees, its ancestors and itself, 32 to a word."""
    rows = []
    for tree in parents:
        seen = []
        for i, p in enumerate(tree):
            seen.append((seen[p] if p >= 0 else 0) | 1 << i)
        rows += seen
    return torch.tensor([[(r >> 32 * w & 0xffffffff) - (1 << 32 if r >> 32 * w & 0x80000000 else 0) for w in range(words)] for r in rows], dtype=torch.int32)


def _table(n_seq, per_seq, shared, extra, gen):
    """Page ids [n_seq, per_seq] out of a random permutation, the first `shared` the same for all, and `extra` more for each sequence."""
    each = per_seq - shared + extra
    ids = torch.randperm(n_seq * each + shared, generator=gen).to(torch.int32)
    own_ids = ids[shared:].view(n_seq, each)
    table = torch.cat([ids[:shared].expand(n_seq, shared), own_ids[:, :per_seq - shared]], 1)
    return table.contiguous().to(DEV), own_ids[:, per_seq - shared:].contiguous().to(DEV), ids.numel()


def prepare(case, seed):
    gen = torch.Generator().manual_seed(seed)
    g = torch.Generator(DEV).manual_seed(seed)
    op, page, kv, dim, n, dtype = case["op"], case["page"], case["kv_heads"], case["dim"], case["n_seq"], TYPES[case["dtype"]]
    normal = lambda *shape, dtype=dtype: torch.randn(*shape, generator=g, device=DEV, dtype=dtype)
    ints = lambda values: torch.tensor(values, dtype=torch.int32, device=DEV)
    rows, held = _lengths(case)
    s = dict(case, live=sum(rows), max_rows=max(rows), max_len=max(held), scale=dim ** -0.5)
    per_seq, pages_to = -(-s["max_len"] // page), -(-case["keep"] // page) if op == "evict" else 0
    s["table"], s["to_table"], n_pages = _table(n, per_seq, case.get("shared", 0) // page, pages_to, gen)
    s.update(row_start=ints([0] + rows).cumsum(0).to(torch.int32), kv_len=ints(held))
    pool = (case["layers"],) if op == "accept" else ()
    s["k_pool"] = normal(*pool, n_pages, kv, page, dim)
    if op in ("bounds", "sparse"):
        s["k_pool"] += normal(n_pages, kv, 1, dim) * 0.7
        s["bounds"] = torch.zeros(n_pages, kv, 2, dim, dtype=dtype, device=DEV)
    if op not in ("bounds", "weights"):
        s["v_pool"] = normal(*pool, n_pages, kv, page, dim)
    if op in ("tree", "sparse", "weights"):
        s["q"] = normal(s["live"], case["heads"], dim)
        s["out"] = torch.zeros_like(s["q"])
    if op in ("tree", "accept"):
        parents, paths = _trees(case, rows)
        s["words"] = -(-s["max_rows"] // 32)
        s["parent"] = ints([p for tree in parents for p in tree])
        s["seen"] = _bits(parents, s["words"]).to(DEV)
    if op == "accept":
        # drafts that are all different; the model's own tokens are those along the path, and others elsewhere
        ids, start = torch.randint(0, 1000, (s["live"],), generator=gen) * 1000, 0
        chosen = torch.full((s["live"],), -5)
        for n_nodes, path in zip(rows, paths):
            ids[start:start + n_nodes] += torch.arange(n_nodes)
            for a, b in zip(path, path[1:]):
                chosen[start + a] = ids[start + b]
            chosen[start + path[-1]] = 7 + 1000 * int(torch.randint(1000, 2000, (1,), generator=gen))
            start += n_nodes
        s.update(ids=ids.to(torch.int32).to(DEV), chosen=chosen.to(torch.int32).to(DEV), path=torch.full((n, s["max_rows"]), -1, dtype=torch.int32, device=DEV),
                 accepted=torch.zeros(n, dtype=torch.int32, device=DEV), next=torch.zeros(n, dtype=torch.int32, device=DEV), new_len=torch.zeros(n, dtype=torch.int32, device=DEV))
    if op == "sparse":
        pages = s["table"].reshape(-1).long()
        s["bounds"][pages] = torch.stack(_page_bounds(s, torch.arange(n, device=DEV).repeat_interleave(per_seq), torch.arange(per_seq, device=DEV).repeat(n)), 2)
        s["selected"] = torch.full((s["live"], kv, case["select"]), -1, dtype=torch.int32, device=DEV)
    if op == "weights":
        s["mass"] = torch.rand(n, kv, s["max_len"], generator=g, device=DEV)
        _, s["lse"] = _scores(s)
    if op == "evict":
        mass = torch.exp(3 * normal(n, kv, s["max_len"], dtype=torch.float32))
        s["mass"] = torch.where(mass < 0.05, 0.0, mass)                     # many positions have no weight worth the name
        s["mass_out"] = torch.zeros(n, kv, case["keep"], device=DEV)
        s["kept"] = torch.full((n, kv, case["keep"]), -1, dtype=torch.int32, device=DEV)
        s["new_len"] = torch.zeros(n, dtype=torch.int32, device=DEV)
    return s


def run(s):
    if own:
        return _own(s)
    return {"tree": _tree, "accept": _accept, "bounds": _bounds, "sparse": _sparse, "weights": _weights, "evict": _evict}[s["op"]](s)


def _own(s):
    from paper_2510_06710_amd import binding as vb
    op = s["op"]
    k, v = s["k_pool"], s.get("v_pool", s["k_pool"])
    cache = vb.make_paged_cache(k[0], v[0]) if op == "accept" else vb.make_paged_cache(k, v)
    batch = vb.make_paged_batch(s["row_start"], s["kv_len"], s["table"], s["live"], s["max_rows"], s["max_len"])
    if op == "accept":
        vb.vla_paged_accept(cache, s["layers"], k[0].numel(), batch, s["parent"], s["ids"], s["chosen"], s["path"], s["accepted"], s["next"], s["new_len"])
        return {"path": s["path"], "accepted": s["accepted"], "next": s["next"], "new_len": s["new_len"], "k": k, "v": v}
    if op == "bounds":
        vb.vla_paged_bounds(cache, batch, s["bounds"])
        return s["bounds"]
    if op == "evict":
        vb.vla_paged_evict(cache, batch, s["mass"], 0, s["recent"], s["to_table"], s["kept"], s["mass_out"], s["new_len"])
        return {"kept": s["kept"], "mass": s["mass_out"], "new_len": s["new_len"], "k": k, "v": v}
    mask = vb.make_paged_mask(s["scale"], softcap=s["cap"], window=s.get("window", 0), shared_len=s.get("shared", 0))
    empty = lambda size: torch.empty(size, dtype=torch.uint8, device=DEV)
    if op == "tree":
        vb.vla_paged_tree_attention(cache, batch, mask, s["seen"], s["q"], s["out"], None, empty(vb.vla_paged_attention_workspace_bytes(cache, batch, mask, s["heads"])))
        return s["out"]
    if op == "sparse":
        vb.vla_paged_select(cache, batch, s["bounds"], s["q"], s["selected"], FIRST, RECENT, empty(vb.vla_paged_select_workspace_bytes(cache, batch)))
        ws = empty(vb.vla_paged_sparse_attention_workspace_bytes(cache, batch, mask, s["heads"], s["select"]))
        vb.vla_paged_sparse_attention(cache, batch, mask, s["selected"], s["q"], s["out"], None, ws)
        return {"selected": s["selected"], "out": s["out"]}
    vb.vla_paged_weights(cache, batch, mask, s["q"], s["lse"], s["mass"], empty(vb.vla_paged_weights_workspace_bytes(cache, batch, mask, s["heads"])))
    return s["mass"]


def _places(s):
    """Sequence, number within it and position of every row."""
    start = s["row_start"].long()
    count = start[1:] - start[:-1]
    seq = torch.repeat_interleave(torch.arange(count.numel(), device=DEV), count, output_size=s["live"])
    within = torch.arange(s["live"], device=DEV) - start[seq]
    return seq, within, s["kv_len"].long()[seq] - count[seq] + within


def _softmax(score):
    """Weights over the last dimension, zeros where all is hidden."""
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - torch.where(top.isinf(), 0.0, top))
    mass = weight.sum(-1, keepdim=True)
    return weight / torch.where(mass == 0, 1.0, mass)


def _scores(s):
    """Scores [n_seq, kv_heads, group, rows, positions], hidden ones -inf, and each row's ln sum exp [rows of all, heads]."""
    seq, within, _ = _places(s)
    n, heads, kv, dim, rows, length = s["n_seq"], s["heads"], s["kv_heads"], s["dim"], s["max_rows"], s["max_len"]
    q = torch.zeros(n, rows, heads, dim, device=DEV)
    q[seq, within] = s["q"].float()
    q = q.view(n, rows, kv, heads // kv, dim).permute(0, 2, 3, 1, 4).reshape(n, kv, heads // kv * rows, dim)
    k = s["k_pool"][s["table"].long()].transpose(1, 2).reshape(n, kv, -1, dim)[:, :, :length].float()
    score = ((q @ k.transpose(2, 3).contiguous()) * s["scale"]).view(n, kv, heads // kv, rows, length)
    if s["cap"]:
        score = s["cap"] * torch.tanh(score / s["cap"])
    start, kv_len = s["row_start"].long(), s["kv_len"].long()
    base = (kv_len - (start[1:] - start[:-1]))[:, None, None]
    p, j = base + torch.arange(rows, device=DEV)[:, None], torch.arange(length, device=DEV)
    if s["op"] == "tree":
        bit = (j - base).clamp(0, 32 * s["words"] - 1).expand(n, rows, length)
        word = torch.zeros(n, rows, s["words"], dtype=torch.int32, device=DEV)
        word[seq, within] = s["seen"]
        see = (j < base) | (word.gather(2, bit // 32) >> (bit % 32) & 1 == 1)
    else:
        see = (j <= p) & (j > p - s["window"]) if s["window"] else j <= p
    see = see & (j < kv_len[:, None, None])
    score = score.masked_fill(~see[:, None, None], float("-inf"))
    lse = torch.logsumexp(score, -1).permute(0, 3, 1, 2).reshape(n, rows, heads)[seq, within]
    return score, lse


def _tree(s):
    seq, within, _ = _places(s)
    n, heads, kv, dim, rows, length = s["n_seq"], s["heads"], s["kv_heads"], s["dim"], s["max_rows"], s["max_len"]
    weight = _softmax(_scores(s)[0])
    v = s["v_pool"][s["table"].long()].transpose(1, 2).reshape(n, kv, -1, dim)[:, :, :length].float()
    o = (weight.view(n, kv, -1, length) @ v).view(n, kv, heads // kv, rows, dim).permute(0, 3, 1, 2, 4).reshape(n, rows, heads, dim)
    s["out"].copy_(o[seq, within])
    return s["out"]


def _accept(s):
    # a node is on the path if it and all its ancestors carry the token that their parent's row chose, and none of their elder siblings does
    seq, within, _ = _places(s)
    n, rows, words = s["n_seq"], s["max_rows"], s["words"]
    place = lambda x, fill: torch.full((n, rows), fill, dtype=torch.long, device=DEV).index_put_((seq, within), x.long())
    parent, ids, chosen = place(s["parent"], -2), place(s["ids"], -1), place(s["chosen"], -3)
    i = torch.arange(rows, device=DEV)
    agrees = (i == 0) & (parent == -1) | (parent >= 0) & (chosen.gather(1, parent.clamp(min=0)) == ids)
    elder = (parent[:, :, None] == parent[:, None]) & (i < i[:, None]) & agrees[:, None]
    agrees = agrees & ~elder.any(2)
    seen = torch.zeros(n, rows, words, dtype=torch.int32, device=DEV)
    seen[seq, within] = s["seen"]
    above = (seen[:, :, i // 32] >> (i % 32) & 1) == 1
    on = agrees & ~(above & ~agrees[:, None]).any(2) & (parent > -2)
    count, kv_len, start = on.sum(1), s["kv_len"].long(), s["row_start"].long()
    base = kv_len - (start[1:] - start[:-1])
    order = torch.where(on, i, rows + i).sort(1).values                     # the path's nodes ascend
    path = torch.where(i < count[:, None], order, -1)
    s["path"].copy_(path)
    s["accepted"].copy_(count)
    s["next"].copy_(chosen.gather(1, path.gather(1, count[:, None] - 1))[:, 0])
    s["new_len"].copy_(base + count)
    b, to = (path >= 0).nonzero(as_tuple=True)
    src, dst, table, page = base[b] + path[b, to], base[b] + to, s["table"].long(), s["page"]
    dst, src = (slice(None), table[b, dst // page], slice(None), dst % page), (slice(None), table[b, src // page], slice(None), src % page)
    s["k_pool"][dst], s["v_pool"][dst] = s["k_pool"][src], s["v_pool"][src]
    return {"path": s["path"], "accepted": s["accepted"], "next": s["next"], "new_len": s["new_len"], "k": s["k_pool"], "v": s["v_pool"]}


def _page_bounds(s, seq, number):
    """Least and largest key of the pages `number` of sequences `seq`, each [pages, kv_heads, dim]."""
    keys = s["k_pool"][s["table"].long()[seq, number]]
    gone = (number[:, None] * s["page"] + torch.arange(s["page"], device=DEV) >= s["kv_len"][seq, None])[:, None, :, None]
    return keys.masked_fill(gone, float("inf")).amin(2), keys.masked_fill(gone, float("-inf")).amax(2)


def _bounds(s):
    start = s["row_start"].long()
    base = s["kv_len"] - (start[1:] - start[:-1])
    number = torch.arange(s["table"].shape[1], device=DEV)
    seq, number = ((number >= base[:, None] // s["page"]) & (number * s["page"] < s["kv_len"][:, None])).nonzero(as_tuple=True)
    s["bounds"][s["table"].long()[seq, number]] = torch.stack(_page_bounds(s, seq, number), 2)
    return s["bounds"]


def _sparse(s):
    seq, _, pos = _places(s)
    kv, dim, page, most = s["kv_heads"], s["dim"], s["page"], s["select"]
    table, kv_index = s["table"].long(), torch.arange(kv, device=DEV)
    q = s["q"].view(-1, kv, s["heads"] // kv, dim)
    # 64 bits: which pages are taken is decided next to borders
    lo, hi = s["bounds"][table].double().unbind(3)                          # [n_seq, pages, kv, dim]
    up, down = q.double().clamp(min=0).sum(2), q.double().clamp(max=0).sum(2)
    bound = (hi.transpose(1, 2)[seq] @ up[..., None] + lo.transpose(1, 2)[seq] @ down[..., None])[..., 0]          # [rows, kv, pages]
    number, last = torch.arange(table.shape[1], device=DEV), (pos // page)[:, None, None]
    always = (number < FIRST) | (number > last - RECENT)
    bound = torch.where(always, float("inf"), bound).masked_fill(number > last, float("-inf"))
    order = torch.sort(bound, dim=2, descending=True, stable=True).indices[:, :, :most]
    taken = torch.arange(order.shape[2], device=DEV) <= last                # as many as there are
    far = 1 << 30
    number = torch.where(taken, order, far).sort(2).values
    s["selected"].fill_(-1)
    s["selected"][:, :, :number.shape[2]] = torch.where(number == far, -1, number)
    number = s["selected"].long()
    at = (number.clamp(min=0)[..., None] * page + torch.arange(page, device=DEV)).flatten(2)                      # [rows, kv, positions]
    see = ((number >= 0)[..., None].expand(*number.shape, page).flatten(2) & (at <= pos[:, None, None]))[:, :, None]
    pages = table[seq[:, None, None], number.clamp(min=0)]
    k, v = (p[pages, kv_index[:, None]].flatten(2, 3).float() for p in (s["k_pool"], s["v_pool"]))
    score = (q.float() @ k.transpose(2, 3).contiguous()) * s["scale"]
    if s["cap"]:
        score = s["cap"] * torch.tanh(score / s["cap"])
    o = _softmax(score.masked_fill(~see, float("-inf"))) @ v
    s["out"].copy_(o.view_as(s["out"]))
    return {"selected": s["selected"], "out": s["out"]}


def _weights(s):
    seq, within, _ = _places(s)
    n, heads, kv, rows = s["n_seq"], s["heads"], s["kv_heads"], s["max_rows"]
    score, _ = _scores(s)
    lse = torch.zeros(n, rows, heads, device=DEV)
    lse[seq, within] = s["lse"]
    weight = torch.exp(score - lse.view(n, rows, kv, heads // kv).permute(0, 2, 3, 1)[..., None])
    there = torch.zeros(n, rows, dtype=torch.bool, device=DEV)
    there[seq, within] = True
    added = (weight * there[:, None, None, :, None]).sum((2, 3))
    start = s["row_start"].long()
    base, j = (s["kv_len"] - (start[1:] - start[:-1]))[:, None, None], torch.arange(s["max_len"], device=DEV)
    s["mass"].copy_(torch.where(j < base, s["mass"] + added, torch.where(j < s["kv_len"][:, None, None], added, s["mass"])))
    return s["mass"]


def _evict(s):
    n, kv, page, keep = s["n_seq"], s["kv_heads"], s["page"], s["keep"]
    kv_len = s["kv_len"].long()[:, None, None]
    j = torch.arange(s["max_len"], device=DEV)
    weight = torch.where(j >= kv_len - s["recent"], float("inf"), s["mass"]).masked_fill(j >= kv_len, float("-inf"))
    order = torch.sort(weight, dim=2, descending=True, stable=True).indices[:, :, :keep]
    far = 1 << 30
    kept = torch.where(torch.arange(order.shape[2], device=DEV) < kv_len, order, far).sort(2).values
    there = kept < far
    s["kept"].fill_(-1)
    s["kept"][:, :, :kept.shape[2]] = torch.where(there, kept, -1)
    s["mass_out"][:, :, :kept.shape[2]] = torch.where(there, s["mass"].gather(2, kept.clamp(max=s["max_len"] - 1)), s["mass_out"][:, :, :kept.shape[2]])
    s["new_len"].copy_(kv_len[:, 0, 0].clamp(max=keep))
    b, h, to = there.nonzero(as_tuple=True)
    at = kept[b, h, to]
    src, dst = (s["table"].long()[b, at // page], h, at % page), (s["to_table"].long()[b, to // page], h, to % page)
    s["k_pool"][dst], s["v_pool"][dst] = s["k_pool"][src], s["v_pool"][src]
    return {"kept": s["kept"], "mass": s["mass_out"], "new_len": s["new_len"], "k": s["k_pool"], "v": s["v_pool"]}


def work(case):
    size, (rows, held) = {"f32": 4, "bf16": 2}[case["dtype"]], _lengths(case)
    op, kv, dim, page, n = case["op"], case["kv_heads"], case["dim"], case["page"], sum(rows)
    row = kv * dim * size                                                   # K or V of one position
    if op == "accept":
        moved = sum(1 for path in _trees(case, rows)[1] for i, node in enumerate(path) if i != node)
        return {"bytes": 4 * case["layers"] * moved * row + 16 * n, "flops": 0}
    if op == "bounds":
        pages = [(-(-l // page), (l - r) // page) for r, l in zip(rows, held)]
        return {"bytes": sum(l - b * page + 2 * (e - b) for (e, b), l in zip(pages, held)) * row, "flops": 0}
    if op == "evict":
        kept = sum(min(l, case["keep"]) for l in held)
        return {"bytes": 4 * kept * row + (sum(held) * 4 + kept * 8) * kv, "flops": 0}
    io, heads = 2 * n * case["heads"] * dim * size, case["heads"]
    if op == "sparse":
        read, pairs, bounds = 0, 0, 0
        for r, l in zip(rows, held):
            for p in range(l - r, l):
                some = min(p + 1, (case["select"] - 1) * page + p % page + 1)
                pairs += some
                read += some if p == l - 1 else 0                           # the newest row's alone: the others' may be the same pages
            bounds += -(-l // page)
        return {"bytes": io + 2 * (read + bounds) * row, "flops": 4 * dim * heads * pairs + 4 * dim * kv * bounds}
    if op == "tree":
        pairs = sum((l - r) * r for r, l in zip(rows, held)) + sum(bin(b & 0xffffffff).count("1") for words in _bits(_trees(case, rows)[0], -(-max(rows) // 32)).tolist() for b in words)
        read = sum(held) - (len(held) - 1) * case["shared"]
        return {"bytes": io + 2 * read * row, "flops": 4 * dim * heads * pairs}
    window, pairs, read = case["window"], 0, 0
    for r, l in zip(rows, held):
        pairs += sum(min(p + 1, window) if window else p + 1 for p in range(l - r, l))
        read += l - (max(0, l - r + 1 - window) if window else 0)
    return {"bytes": io // 2 + n * heads * 4 + read * (row + 8 * kv), "flops": 2 * dim * heads * pairs}


def exact(case, seed):
    s = prepare(case, seed)
    rows, held = _lengths(case)
    s["spans"] = []                                                         # (sequence, first row, rows, positions held)
    for i, (r, l) in enumerate(zip(rows, held)):
        s["spans"].append((i, sum(rows[:i]), r, l))
    return {"tree": _exact_tree, "accept": _exact_accept, "bounds": _exact_bounds, "sparse": _exact_sparse, "weights": _exact_weights, "evict": _exact_evict}[case["op"]](s)


def _held(s, pool, i, length, h):
    """Positions 0 .. length - 1 of sequence i and key head h in 64 bits."""
    return pool[s["table"][i, :-(-length // s["page"])].long(), h].reshape(-1, s["dim"])[:length].double()


def _capped(s, score):
    return (score / s["cap"]).tanh() * s["cap"] if s["cap"] else score


def _exact_tree(s):
    out, group = s["out"].double(), s["heads"] // s["kv_heads"]
    for i, a, n, length in s["spans"]:
        hidden = torch.zeros(n, length, dtype=torch.bool, device=DEV)
        tree = s["parent"][a:a + n].tolist()
        for node in range(n):
            hidden[node, length - n:] = True
            up = node
            while up >= 0:
                hidden[node, length - n + up] = False
                up = tree[up]
        for h in range(s["heads"]):
            k, v = (_held(s, p, i, length, h // group) for p in (s["k_pool"], s["v_pool"]))
            score = _capped(s, s["q"][a:a + n, h].double() @ k.T * s["scale"])
            out[a:a + n, h] = torch.softmax(score.masked_fill(hidden, -math.inf), 1) @ v
    return out


def _exact_accept(s):
    """One sequence at a time, node after node."""
    k, v, path = s["k_pool"], s["v_pool"], torch.full_like(s["path"], -1)
    count, follow, new_len = [], [], []
    for i, a, n, length in s["spans"]:
        parent, ids, chosen = (s[x][a:a + n].tolist() for x in ("parent", "ids", "chosen"))
        taken, cur = [], 0
        while cur is not None:
            taken.append(cur)
            cur = next((c for c in range(n) if parent[c] == taken[-1] and ids[c] == chosen[taken[-1]]), None)
        for to, node in enumerate(taken):                                   # ascending: what is written was read before
            src, dst = length - n + node, length - n + to
            for pool in (k, v):
                pool[:, s["table"][i, dst // s["page"]], :, dst % s["page"]] = pool[:, s["table"][i, src // s["page"]], :, src % s["page"]]
        path[i, :len(taken)] = torch.tensor(taken, dtype=torch.int32)
        count.append(len(taken)), follow.append(chosen[taken[-1]]), new_len.append(length - n + len(taken))
    ints = lambda x: torch.tensor(x, dtype=torch.int32)
    return {"path": path, "accepted": ints(count), "next": ints(follow), "new_len": ints(new_len), "k": k, "v": v}


def _exact_bounds(s):
    bounds = s["bounds"].double()
    for i, _, n, length in s["spans"]:
        for h in range(s["kv_heads"]):
            first = (length - n) // s["page"]
            parts = _held(s, s["k_pool"], i, length, h)[first * s["page"]:].split(s["page"])
            at = s["table"][i, first:first + len(parts)].long()
            bounds[at, h, 0] = torch.stack([x.min(0).values for x in parts])
            bounds[at, h, 1] = torch.stack([x.max(0).values for x in parts])
    return bounds


def _exact_sparse(s):
    """One row and key head at a time; the bound as it is defined, the larger of two products for each dim."""
    out, selected, group, page = s["out"].double(), torch.full_like(s["selected"], -1), s["heads"] // s["kv_heads"], s["page"]
    for i, a, n, length in s["spans"]:
        for row in range(a, a + n):
            p = length - n + row - a
            last = p // page
            for h in range(s["kv_heads"]):
                q = s["q"][row, h * group:(h + 1) * group].double()
                lo, hi = s["bounds"][s["table"][i, :last + 1].long(), h].double().unbind(1)
                bound = torch.maximum(q[:, None] * lo, q[:, None] * hi).sum((0, 2)).tolist()
                rank = sorted(range(last + 1), key=lambda c: (not (c < FIRST or c > last - RECENT), -bound[c], c))
                taken = torch.tensor(sorted(rank[:s["select"]]), device=DEV)
                selected[row, h, :len(taken)] = taken.to(torch.int32)
                at = (taken[:, None] * page + torch.arange(page, device=DEV)).flatten()
                at = at[at <= p]
                k, v = (x[s["table"][i, at // page].long(), h, at % page].double() for x in (s["k_pool"], s["v_pool"]))
                out[row, h * group:(h + 1) * group] = torch.softmax(_capped(s, q @ k.T * s["scale"]), 1) @ v
    return {"selected": selected, "out": out}


def _exact_weights(s):
    mass, group = s["mass"].double(), s["heads"] // s["kv_heads"]
    for i, a, n, length in s["spans"]:
        j, p = torch.arange(length, device=DEV), torch.arange(length - n, length, device=DEV)[:, None]
        hidden = (j > p) | ((j <= p - s["window"]) if s["window"] else torch.zeros_like(j > p))
        mass[i, :, length - n:length] = 0
        for h in range(s["heads"]):
            score = _capped(s, s["q"][a:a + n, h].double() @ _held(s, s["k_pool"], i, length, h // group).T * s["scale"])
            weight = torch.exp(score - s["lse"][a:a + n, h, None].double()).masked_fill(hidden, 0.0)
            mass[i, h // group, :length] += weight.sum(0)
    return mass


def _exact_evict(s):
    """One sequence and key head at a time."""
    k, v, kept, mass = s["k_pool"], s["v_pool"], torch.full_like(s["kept"], -1), s["mass_out"].double()
    for i, _, _, length in s["spans"]:
        for h in range(s["kv_heads"]):
            weight = s["mass"][i, h, :length].tolist()
            rank = sorted(range(length), key=lambda j: (j < length - s["recent"], -weight[j], j))
            at = torch.tensor(sorted(rank[:s["keep"]]), device=DEV)
            to = torch.arange(len(at), device=DEV)
            kept[i, h, :len(at)] = at.to(torch.int32)
            mass[i, h, :len(at)] = s["mass"][i, h, at].double()
            for pool in (k, v):
                pool[s["to_table"][i, to // s["page"]].long(), h, to % s["page"]] = pool[s["table"][i, at // s["page"]].long(), h, at % s["page"]]
    return {"kept": kept, "mass": mass, "new_len": s["kv_len"].clamp(max=s["keep"]), "k": k, "v": v}
