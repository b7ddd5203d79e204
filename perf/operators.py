"""The operators of a rollout step on a paged KV cache, as measurable cases.

A serving loop over ragged batches appends the new rows' keys and values to pages (norms per head and rotation on the way),
attends to the pages (whole prompts, single tokens, batches that share a prefix) and samples from the logits.  `run` computes
each operator in elementary torch operations, or calls the library's (`own`).

Keys, queries and values are N(0, 1), so scores scaled by 1/sqrt(head_dim) are too; logits are N(0, 3) with a few raised ones.
Page tables are a random permutation of the pages, as after many sequences have come and gone.
"""
import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def listed():
    return [
        # one robot's next token: latency of the smallest append, grouped heads, projection already rounded
        dict(name="append_one_row", op="append", n_seq=1, rows=1, past=700, ragged=False, heads=32, kv_heads=8, dim=128, page=16,
             rot=128, interleaved=False, norms=True, src="bf16", dtype="bf16", pad=0),
        # observation prefixes of 64 environments at the 7B shape, from the fp32 projection: the largest append of a rollout
        dict(name="append_prefix_b64", op="append", n_seq=64, rows=288, past=0, ragged=False, heads=32, kv_heads=32, dim=128, page=16,
             rot=128, interleaved=False, norms=False, src="f32", dtype="bf16", pad=0),
        # ragged chunks of long conversations, padded batch: interleaved pairs on half of each head, norms per head, fp32 cache
        dict(name="append_ragged_f32", op="append", n_seq=13, rows=301, past=90000, ragged=True, heads=12, kv_heads=4, dim=80, page=32,
             rot=40, interleaved=True, norms=True, src="f32", dtype="f32", pad=37),
        # the action tokens of 256 environments at the 7B shape, whose own K and V are all there is to read
        dict(name="decode_b256", op="attention", n_seq=256, rows=1, len=294, ragged=False, heads=32, kv_heads=32, dim=128, page=16,
             cap=0.0, bias=False, prefix=False, window=0, shared=0, dtype="bf16"),
        # one sequence with a long context and grouped heads: one row, the keys have to be split
        dict(name="decode_long_b1", op="attention", n_seq=1, rows=1, len=32768, ragged=False, heads=32, kv_heads=8, dim=128, page=64,
             cap=0.0, bias=False, prefix=False, window=0, shared=0, dtype="bf16"),
        # a ragged batch of single tokens with capped scores and a bias by distance
        dict(name="decode_ragged_cap", op="attention", n_seq=48, rows=1, len=8192, ragged=True, heads=32, kv_heads=4, dim=128, page=32,
             cap=30.0, bias=True, prefix=False, window=0, shared=0, dtype="bf16"),
        # groups of rollouts from one state: 64 sequences that share a long prefix
        dict(name="decode_shared_b64", op="attention", n_seq=64, rows=1, len=4352, ragged=True, heads=32, kv_heads=8, dim=128, page=64,
             cap=0.0, bias=False, prefix=False, window=0, shared=4096, dtype="bf16"),
        # a long prompt in one go, grouped heads, causal: matrix products
        dict(name="prompt_8k", op="attention", n_seq=1, rows=8192, len=8192, ragged=False, heads=32, kv_heads=8, dim=128, page=64,
             cap=0.0, bias=False, prefix=False, window=0, shared=0, dtype="bf16"),
        # ragged observation prefixes that see themselves whole, instructions behind them causal, capped scores
        dict(name="prompt_prefix_ragged", op="attention", n_seq=13, rows=613, len=613, ragged=True, heads=16, kv_heads=16, dim=64, page=16,
             cap=50.0, bias=False, prefix=True, window=0, shared=0, dtype="bf16"),
        # the tiny fp32 decoder's prefixes with a window, a unit test's size
        dict(name="prompt_tiny_f32", op="attention", n_seq=8, rows=64, len=71, ragged=False, heads=4, kv_heads=4, dim=64, page=16,
             cap=0.0, bias=True, prefix=False, window=33, shared=0, dtype="f32"),
        # action bins of 256 environments
        dict(name="sample_bins_b256", op="sample", n=256, vocab=256, dtype="f32"),
        # text tokens of 256 sequences over a large vocabulary
        dict(name="sample_vocab_b256", op="sample", n=256, vocab=128000, dtype="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "attention", "attention", "sample"])
    if op == "sample":
        n, vocab = _log(rng, 1, 256), _log(rng, 200, 128000)
        return dict(op=op, n=n, vocab=vocab, dtype=rng.choice(["f32", "bf16"]))
    dtype, dim = rng.choice(["bf16", "bf16", "f32"]), rng.choice([64, 80, 128, 128, 256])
    kv_heads, page = rng.choice([1, 2, 4, 8]), rng.choice([16, 32, 64, 128])
    heads = kv_heads * rng.choice([1, 2, 3, 4, 7, 8])
    if op == "append":
        n_seq = _log(rng, 1, 128)
        most = 2 ** 27 // ((heads + 2 * kv_heads) * dim) // n_seq
        rows = 1 if rng.random() < 0.3 else _log(rng, 2, max(2, min(most, 16384 // n_seq)))
        past = _log(rng, 1, 100000 // (1 + n_seq // 8))
        return dict(op=op, n_seq=n_seq, rows=rows, past=past, ragged=rng.random() < 0.6, heads=heads, kv_heads=kv_heads, dim=dim, page=page,
                    rot=rng.choice([dim, dim // 2, 0]), interleaved=rng.random() < 0.5, norms=rng.random() < 0.5,
                    src=rng.choice(["f32", dtype]), dtype=dtype, pad=rng.choice([0, 0, 1, 19]))
    kind = rng.choice(["decode", "decode", "prompt", "shared"])
    if kind == "decode":
        n_seq = _log(rng, 1, 256)
        length, rows, shared = _log(rng, 1, min(32768, 65536 // n_seq)), rng.choice([1, 1, 1, 2, 5]), 0
    elif kind == "shared":
        n_seq, rows = _log(rng, 2, 64), 1
        shared = page * _log(rng, 1, 4096 // page)
        length = shared + _log(rng, 1, 512)
    else:
        n_seq = _log(rng, 1, 16)
        rows = _log(rng, 2, 4096 // n_seq)
        length, shared = rows + rng.choice([0, 0, _log(rng, 1, 1024)]), 0
    rows = min(rows, length - shared)
    return dict(op=op, n_seq=n_seq, rows=rows, len=length, ragged=rng.random() < 0.6, heads=heads, kv_heads=kv_heads, dim=dim, page=page,
                cap=rng.choice([0.0, 0.0, 20.0, 50.0]), bias=rng.random() < 0.3, prefix=kind == "prompt" and rng.random() < 0.4,
                window=rng.choice([0, 0, 0, _log(rng, 1, length)]) if kind != "shared" else 0, shared=shared, dtype=dtype)


def _lengths(case):
    """New rows and positions before them, per sequence; fixed by the case, so that all seeds do the same work."""
    n = case["n_seq"]
    gen = torch.Generator().manual_seed(n)
    if case["op"] == "append":
        rows, past = [case["rows"]] * n, [case["past"]] * n
        if case["ragged"]:
            rows = torch.randint(1, case["rows"] + 1, (n,), generator=gen).tolist()
            past = torch.randint(0, case["past"] + 1, (n,), generator=gen).tolist()
            rows[0], past[-1] = case["rows"], case["past"]
        return rows, past
    length, rows = [case["len"]] * n, [case["rows"]] * n
    if case["ragged"]:
        length = torch.randint(case["shared"] + 1, case["len"] + 1, (n,), generator=gen).tolist()
        length[-1] = case["len"]
        if case["rows"] > 1:
            share = torch.rand(n, generator=gen).tolist()
            rows = [max(1, min(case["rows"], l, round(case["rows"] * f))) for f, l in zip(share, length)]
            if case["rows"] == case["len"]:
                rows = length
            rows[-1] = case["rows"]
    return rows, [l - r for l, r in zip(length, rows)]


def _table(n_seq, per_seq, shared, gen):
    """Page ids [n_seq, per_seq] out of a random permutation; the first `shared` are the same for all."""
    own_pages = n_seq * (per_seq - shared)
    ids = torch.randperm(own_pages + shared, generator=gen).to(torch.int32)
    first = ids[:shared].expand(n_seq, shared)
    return torch.cat([first, ids[shared:].view(n_seq, per_seq - shared)], 1).contiguous(), own_pages + shared


def prepare(case, seed):
    gen = torch.Generator().manual_seed(seed)
    g = torch.Generator(DEV).manual_seed(seed)
    normal = lambda *shape, dtype=torch.float32: torch.randn(*shape, generator=g, device=DEV, dtype=dtype)
    s = dict(case)
    if case["op"] == "sample":
        n, vocab = case["n"], case["vocab"]
        z = normal(n, vocab) * 3
        z[torch.arange(n, device=DEV)[:, None], torch.randint(0, vocab, (n, 4), generator=g, device=DEV)] += 6
        pick = lambda values, dtype: torch.tensor(values)[torch.randint(0, len(values), (n,), generator=gen)].to(dtype).to(DEV)
        s.update(logits=z.to(TYPES[case["dtype"]]), temperature=pick([1.0, 0.7, 1.6], torch.float32),
                 top_k=pick([0, 0, 1, 20, 50, 300], torch.int32), top_p=pick([1.0, 0.95, 0.9, 0.5], torch.float32),
                 min_p=pick([0.0, 0.0, 0.05, 0.01], torch.float32), u=torch.rand(n, generator=g, device=DEV))
        for name, kind in (("token", torch.int32), ("n_kept", torch.int32), ("logp", torch.float32), ("logp_kept", torch.float32)):
            s[name] = torch.zeros(n, dtype=kind, device=DEV)
        return s
    dtype, dim, heads, kv = TYPES[case["dtype"]], case["dim"], case["heads"], case["kv_heads"]
    rows, past = _lengths(case)
    s["max_rows"], s["max_len"] = max(rows), max(r + p for r, p in zip(rows, past))
    live = sum(rows)
    total = live + case.get("pad", 0)
    pages = -(-s["max_len"] // case["page"])
    table, n_pages = _table(case["n_seq"], pages, case.get("shared", 0) // case["page"], gen)
    starts = torch.tensor([0] + rows).cumsum(0)
    s.update(live=live, table=table.to(DEV), row_start=starts.to(torch.int32).to(DEV),
             kv_len=torch.tensor([r + p for r, p in zip(rows, past)], dtype=torch.int32).to(DEV))
    if case["op"] == "append":
        s["k_pool"], s["v_pool"] = (torch.zeros(n_pages, kv, case["page"], dim, dtype=dtype, device=DEV) for _ in range(2))
        qkv = normal(total, heads + 2 * kv, dim).to(TYPES[case["src"]])           # one projection's output, split by views
        s.update(q=qkv[:, :heads], k=qkv[:, heads:heads + kv], v=qkv[:, heads + kv:], q_out=torch.zeros(total, heads, dim, dtype=dtype, device=DEV))
        half = case["rot"] // 2
        s["freq"] = (10000.0 ** (-torch.arange(half, dtype=torch.float64) / max(half, 1)) / 4.0).to(DEV) if half else None    # scaled for long contexts
        s["q_gain"], s["k_gain"] = (1 + 0.1 * normal(dim), 1 + 0.1 * normal(dim)) if case["norms"] else (None, None)
        return s
    s["k_pool"], s["v_pool"] = (normal(n_pages, kv, case["page"], dim, dtype=dtype) for _ in range(2))
    s.update(q=normal(total, heads, dim, dtype=dtype), out=torch.zeros(total, heads, dim, dtype=dtype, device=DEV), scale=dim ** -0.5)
    s["slopes"] = torch.exp2(-8.0 * (torch.arange(heads, device=DEV) + 1.0) / heads) if case["bias"] else None
    s["prefix_len"] = (s["kv_len"] * 4 // 5).to(torch.int32) if case["prefix"] else None
    return s


def run(s):
    if own:
        return _own(s)
    return {"append": _append, "attention": _attention, "sample": _sample}[s["op"]](s)


def _own(s):
    from paper_2510_06710_amd import binding as vb
    if s["op"] == "sample":
        ws = torch.empty(vb.vla_sample_logits_workspace_bytes(s["n"], s["vocab"]), dtype=torch.uint8, device=DEV)
        vb.vla_sample_logits(s["logits"], s["token"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], u=s["u"],
                             logp=s["logp"], logp_kept=s["logp_kept"], n_kept=s["n_kept"], ws=ws)
        return {name: s[name] for name in ("token", "n_kept", "logp", "logp_kept")}
    cache = vb.make_paged_cache(s["k_pool"], s["v_pool"])
    batch = vb.make_paged_batch(s["row_start"], s["kv_len"], s["table"], s["q"].shape[0], s["max_rows"], s["max_len"])
    if s["op"] == "append":
        rotary = vb.make_rotary(s["freq"], interleaved=s["interleaved"], scale=1.0, q_gain=s["q_gain"], k_gain=s["k_gain"], eps=1e-6)
        vb.vla_paged_append(cache, batch, rotary, s["q"], s["k"], s["v"], s["q_out"])
        return {"q": s["q_out"], "k": s["k_pool"], "v": s["v_pool"]}
    mask = vb.make_paged_mask(s["scale"], softcap=s["cap"], slopes=s["slopes"], prefix_len=s["prefix_len"], window=s["window"], shared_len=s["shared"])
    ws = torch.empty(vb.vla_paged_attention_workspace_bytes(cache, batch, mask, s["heads"]), dtype=torch.uint8, device=DEV)
    vb.vla_paged_attention(cache, batch, mask, s["q"], s["out"], None, ws)
    return s["out"]


def _places(s):
    """Sequence, number within it and position of every live row."""
    start, live = s["row_start"].long(), s["live"]
    count = start[1:] - start[:-1]
    seq = torch.repeat_interleave(torch.arange(count.numel(), device=DEV), count, output_size=live)
    within = torch.arange(live, device=DEV) - start[seq]
    return seq, within, s["kv_len"].long()[seq] - count[seq] + within


def _append(s):
    seq, _, pos = _places(s)
    live, half = s["live"], s["rot"] // 2

    def turned(x, gain):
        x = x[:live].float()
        if gain is not None:
            x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * gain
        if half:
            angle = (pos.double()[:, None] * s["freq"])[:, None]
            cos, sin = angle.cos().float(), angle.sin().float()
            a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if s["interleaved"] else (x[..., :half], x[..., half:2 * half])
            ya, yb = a * cos - b * sin, b * cos + a * sin
            pairs = torch.stack([ya, yb], -1).flatten(-2) if s["interleaved"] else torch.cat([ya, yb], -1)
            x = torch.cat([pairs, x[..., 2 * half:]], -1)
        return x.to(s["q_out"].dtype)

    page, row = s["table"].long()[seq, pos // s["page"]], pos % s["page"]
    s["q_out"][:live] = turned(s["q"], s["q_gain"])
    s["k_pool"][page, :, row] = turned(s["k"], s["k_gain"])
    s["v_pool"][page, :, row] = s["v"][:live].to(s["v_pool"].dtype)
    return {"q": s["q_out"], "k": s["k_pool"], "v": s["v_pool"]}


def _attention(s):
    seq, within, _ = _places(s)
    n, heads, kv, dim, rows, length = s["n_seq"], s["heads"], s["kv_heads"], s["dim"], s["max_rows"], s["max_len"]
    q = torch.zeros(n, rows, heads, dim, device=DEV)
    q[seq, within] = s["q"].float()
    q = q.view(n, rows, kv, heads // kv, dim).permute(0, 2, 3, 1, 4).reshape(n, kv, heads // kv * rows, dim)
    pages = s["table"].long()
    k, v = (p[pages].transpose(1, 2).reshape(n, kv, -1, dim)[:, :, :length].float() for p in (s["k_pool"], s["v_pool"]))
    start = s["row_start"].long()
    kv_len = s["kv_len"].long()
    p = (kv_len - (start[1:] - start[:-1]))[:, None, None] + torch.arange(rows, device=DEV)[:, None]
    j = torch.arange(length, device=DEV)
    seen = j <= p
    if s["window"]:
        seen = seen & (j > p - s["window"])
    if s["prefix_len"] is not None:
        seen = seen | (j < s["prefix_len"][:, None, None])
    seen = (seen & (j < kv_len[:, None, None]))[:, None, None]                    # [n, 1, 1, rows, length]
    # positions behind a sequence's end hold other sequences' values, which are finite: weights of zero leave them out
    score = ((q @ k.transpose(2, 3)) * s["scale"]).view(n, kv, heads // kv, rows, length)
    if s["cap"]:
        score = s["cap"] * torch.tanh(score / s["cap"])
    if s["slopes"] is not None:
        score = score - s["slopes"].view(1, kv, heads // kv, 1, 1) * (p - j).abs()[:, None, None]
    score = score.masked_fill(~seen, float("-inf"))
    top = score.amax(-1, keepdim=True)
    weight = torch.exp(score - torch.where(top.isinf(), 0.0, top))
    mass = weight.sum(-1, keepdim=True)
    weight = weight / torch.where(mass == 0, 1.0, mass)
    o = (weight.view(n, kv, -1, length) @ v).view(n, kv, heads // kv, rows, dim).permute(0, 3, 1, 2, 4).reshape(n, rows, heads, dim)
    s["out"][:s["live"]] = o[seq, within].to(s["out"].dtype)
    return s["out"]


def _sample(s):
    # 64 bits: which tokens the cut of top-p keeps, and where u falls, are decided next to borders
    z = s["logits"].double() / s["temperature"].double()[:, None]
    value, index = torch.sort(z, dim=1, descending=True, stable=True)
    mass = torch.exp(value - value[:, :1])
    rank = torch.arange(z.shape[1], device=DEV)
    k = torch.where(s["top_k"] > 0, s["top_k"].long(), z.shape[1])[:, None]
    keep = rank < k
    leading = torch.where(keep, mass, 0.0)
    before = leading.cumsum(1) - leading
    p = s["top_p"].double()[:, None]
    keep = keep & ((p >= 1) | (before < p * leading.sum(1, keepdim=True))) & (mass >= s["min_p"].double()[:, None])
    kept = torch.zeros_like(z).scatter_(1, index, torch.where(keep, mass, 0.0))
    running = kept.cumsum(1)
    total = running[:, -1:]
    token = (running <= s["u"].double()[:, None] * total).sum(1, keepdim=True)
    token = torch.minimum(token, (kept > 0).long().mul(rank).amax(1, keepdim=True))
    weight = kept.gather(1, token)
    s["token"].copy_(token[:, 0])
    s["n_kept"].copy_(keep.sum(1))
    s["logp"].copy_((weight.log() - mass.sum(1, keepdim=True).log())[:, 0])
    s["logp_kept"].copy_((weight.log() - total.log())[:, 0])
    return {name: s[name] for name in ("token", "n_kept", "logp", "logp_kept")}


def work(case):
    size = {"f32": 4, "bf16": 2}
    if case["op"] == "sample":
        return {"bytes": case["n"] * (case["vocab"] * size[case["dtype"]] + 36), "flops": 4 * case["n"] * case["vocab"]}
    rows, past = _lengths(case)
    dim, heads, kv, n = case["dim"], case["heads"], case["kv_heads"], sum(rows)
    if case["op"] == "append":
        moved = n * (heads + 2 * kv) * dim * (size[case["src"]] + size[case["dtype"]])
        return {"bytes": moved + 8 * n, "flops": n * (heads + kv) * dim * 6}
    pairs, read = 0, case["shared"]
    for r, b in zip(rows, past):
        length, first = r + b, 0
        window = case["window"]
        prefix = length * 4 // 5 if case["prefix"] else 0
        seen = lambda p: max(p + 1, prefix) - (max(0, p + 1 - window - prefix) if window and p + 1 > prefix else 0)
        pairs += sum(seen(b + i) for i in range(r))
        if window and not prefix:
            first = max(0, b + 1 - window)
        read += length - max(first, case["shared"])
    moved = 2 * n * heads * dim * size[case["dtype"]] + 2 * read * kv * dim * size[case["dtype"]]
    return {"bytes": moved, "flops": 4 * dim * heads * pairs}


def exact(case, seed):
    s = prepare(case, seed)
    return {"append": _exact_append, "attention": _exact_attention, "sample": _exact_sample}[case["op"]](s)


def _exact_append(s):
    """Rotation as a product of complex numbers, one sequence at a time."""
    start, lens, table = s["row_start"].tolist(), s["kv_len"].tolist(), s["table"].long()
    q_out, k_pool, v_pool = s["q_out"].double(), s["k_pool"].double(), s["v_pool"].double()
    half = s["rot"] // 2
    for i, length in enumerate(lens):
        a, b = start[i], start[i + 1]
        pos = torch.arange(length - (b - a), length, device=DEV)
        done = []
        for x, gain in ((s["q"], s["q_gain"]), (s["k"], s["k_gain"])):
            x = x[a:b].double()
            if gain is not None:
                x = x / (x.pow(2).sum(-1, keepdim=True) / s["dim"] + 1e-6).sqrt() * gain.double()
            if half:
                part = x[..., :2 * half]
                part = part.unflatten(-1, (half, 2)) if s["interleaved"] else part.unflatten(-1, (2, half)).transpose(-1, -2)
                turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), torch.outer(pos.double(), s["freq"]))
                part = torch.view_as_real(torch.view_as_complex(part.contiguous()) * turn[:, None])
                part = part.flatten(-2) if s["interleaved"] else part.transpose(-1, -2).flatten(-2)
                x = torch.cat([part, x[..., 2 * half:]], -1)
            done.append(x)
        q_out[a:b] = done[0]
        page, row = table[i][pos // s["page"]], pos % s["page"]
        k_pool[page, :, row], v_pool[page, :, row] = done[1], s["v"][a:b].double()
    return {"q": q_out, "k": k_pool, "v": v_pool}


def _exact_attention(s):
    """One sequence and one key head at a time, by torch's softmax in 64 bits."""
    start, lens = s["row_start"].tolist(), s["kv_len"].tolist()
    prefix = s["prefix_len"].tolist() if s["prefix_len"] is not None else [0] * len(lens)
    out, group = s["out"].double(), s["heads"] // s["kv_heads"]
    for i, length in enumerate(lens):
        a, b = start[i], start[i + 1]
        pages = s["table"][i, :-(-length // s["page"])].long()
        j, pos = torch.arange(length, device=DEV), torch.arange(length - (b - a), length, device=DEV)
        away = pos[:, None] - j
        hidden = (away < 0) | ((away >= s["window"]) if s["window"] else torch.zeros_like(away, dtype=torch.bool))
        hidden &= j >= prefix[i]
        blind = hidden.all(1)
        for h in range(s["kv_heads"]):
            k, v = (p[pages, h].reshape(-1, s["dim"])[:length].double() for p in (s["k_pool"], s["v_pool"]))
            for e in range(h * group, (h + 1) * group):
                score = s["q"][a:b, e].double() @ k.T * s["scale"]
                if s["cap"]:
                    score = (score / s["cap"]).tanh() * s["cap"]
                if s["slopes"] is not None:
                    score -= s["slopes"][e].double() * away.abs()
                weight = torch.softmax(score.masked_fill(hidden, -math.inf), 1).masked_fill(blind[:, None], 0.0)
                out[a:b, e] = weight @ v
    return out


def _exact_sample(s):
    """One row at a time."""
    rows = {"token": [], "n_kept": [], "logp": [], "logp_kept": []}
    settings = zip(*(s[name].tolist() for name in ("temperature", "top_k", "top_p", "min_p", "u")))
    for z, (t, k, p, least, u) in zip(s["logits"], settings):
        logp = torch.log_softmax(z.double() / t, 0)
        order = torch.argsort(logp, descending=True, stable=True)
        if k > 0:
            order = order[:k]
        share = torch.softmax(logp[order], 0)
        if p < 1:
            order = order[:int((share.cumsum(0) - share < p).sum())]
        order = order[torch.exp(logp[order] - logp[order[0]]) >= least]
        order = order.sort().values
        share = torch.softmax(logp[order], 0)
        at = min(int((share.cumsum(0) <= u).sum()), order.numel() - 1)
        for name, x in (("token", order[at]), ("n_kept", torch.tensor(order.numel())), ("logp", logp[order[at]]), ("logp_kept", share[at].log())):
            rows[name].append(x.cpu())
    return {name: torch.stack(x) for name, x in rows.items()}
