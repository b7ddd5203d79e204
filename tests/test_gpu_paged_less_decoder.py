"""The decoder on selected pages against the oracle with the same selection, and sampled drafts against sampling one by one.

Logits are compared with parity.py's fp32 tolerance, from the first token on up to where a choice (of a page, of a token) hangs on less than rounding may move."""
import numpy as np
import pytest
import torch

import vla_inputs as vi
from oracle import vla_oracle as vo
from oracle.from_inputs import oracle_config, oracle_weights, to_f64
from paged_less_ref import choose
from paged_ref import DEV
from paper_2510_06710_amd import binding as vb
from paper_2510_06710_amd.harness import PagedRollout
from parity import TOL
from test_gpu_paged_less_rollout import SHAPES, first_id, setup, started

pytestmark = pytest.mark.gpu
SHAPE, SEED, PAGE = SHAPES["f32"], 3, 16


def selected_step(cfg, w, past, token, select, first, recent):
    """Logits of one more token whose heads read the pages they select, the K and V with it, and by how much the nearest choice of a page was made."""
    x, sure, grown = w.embed[token][None], np.inf, []
    for l in range(cfg.n_layers):
        lw, p = w.layer(l), past[l][0].shape[1]
        heads = lambda m: (vo.rmsnorm(x, lw["attn_norm"], cfg.rms_eps) @ m.T).reshape(cfg.n_heads, 1, cfg.head_dim)
        at = np.array([p])
        q = vo.rotary(heads(lw["wq"]), at, cfg.rope_theta)
        k = np.concatenate([past[l][0], vo.rotary(heads(lw["wk"]), at, cfg.rope_theta)], 1)
        v = np.concatenate([past[l][1], heads(lw["wv"])], 1)
        grown.append((k, v))
        out = np.zeros((cfg.n_heads, cfg.head_dim))
        for h in range(cfg.n_heads):
            pages = [k[h, a:a + PAGE] for a in range(0, p + 1, PAGE)]
            score = np.array([np.maximum(q[h, 0] * s.min(0), q[h, 0] * s.max(0)).sum() for s in pages])
            taken = choose(score, select, first, recent)
            free = [i for i in range(first, len(pages) - recent)]
            left, had = [score[i] for i in free if i not in taken], [score[i] for i in free if i in taken]
            if left and had:
                sure = min(sure, min(had) - max(left))
            j = np.concatenate([np.arange(i * PAGE, min((i + 1) * PAGE, p + 1)) for i in taken])
            s = k[h, j] @ q[h, 0] / np.sqrt(cfg.head_dim)
            weight = np.exp(s - s.max())
            out[h] = weight @ v[h, j] / weight.sum()
        x = x + out.reshape(1, -1) @ lw["wo"].T
        n = vo.rmsnorm(x, lw["ffn_norm"], cfg.rms_eps)
        x = x + (vo.silu(n @ lw["w_gate"].T) * (n @ lw["w_up"].T)) @ lw["w_down"].T
    return vo.bin_logits(cfg, w, vo.rmsnorm(x, w.final_norm, cfg.rms_eps))[0], grown, sure


@pytest.mark.parametrize("select", [1, 2, 3, 4, 7])
def test_selected_pages_are_those_of_the_oracle(select):
    lengths, steps = [(5, 3), (48, 16), (100, 29), (31, 17)], 6
    run, patches, ids = setup(SHAPE, lengths)
    paged, logits = started(run, patches, ids)
    bins, _, _, z = paged.decode(logits, steps, select=select)
    cfg, w = oracle_config(SHAPE), oracle_weights(vi.SynthModel(SHAPE, SEED), vi.VALUE_BIAS)
    compared = 0
    for i in range(len(lengths)):
        kv, h, _ = vo.ovla_prefill(cfg, w, to_f64(patches[i])[None], ids[i].cpu().numpy()[None])
        assert np.abs(z[i, 0].double().cpu().numpy() - vo.bin_logits(cfg, w, h)[0]).max() <= TOL["f32"]["logits"]
        past = [(k[0], v[0]) for k, v in kv]
        for j in range(steps - 1):
            want, past, sure = selected_step(cfg, w, past, first_id(run) + int(bins[i, j]), select, int(select > 2), min(2, select))
            if sure <= 4 * TOL["f32"]["logits"]:
                break
            assert np.abs(z[i, j + 1].double().cpu().numpy() - want).max() <= TOL["f32"]["logits"], (i, j)
            compared += 1
    assert compared >= 15


def a_draw(z, t, top_k, rng):
    """A number that draws the middle of one of the kept tokens, and whether rounding can neither change the token nor which are kept."""
    order, sure = np.argsort(-z, kind="stable"), 4 * TOL["f32"]["logits"]
    keep = np.sort(order[:top_k])
    mass = np.exp((z[keep] - z.max()) / t)
    mass /= mass.sum()
    i = rng.choice(np.nonzero(mass >= 0.5 / len(keep))[0])
    return mass[:i].sum() + mass[i] / 2, mass[i] / 2 > sure and (top_k >= len(z) or z[order[top_k - 1]] - z[order[top_k]] > sure)


@pytest.mark.parametrize("top_k", [3, 256])
def test_sampled_drafts_are_those_of_sampling_one_by_one(top_k):
    """Every node of a depth is given the draw that the token of that number is given: whichever path is taken, it is that of sampling one by one."""
    run, patches, ids = setup(SHAPE, [(5, 3), (40, 9), (0, 30)])
    n, steps, t, rng = 3, 24, 1.6, np.random.default_rng(top_k)
    plain, logits = started(run, patches, ids)
    U, want, sure, certain = torch.zeros(steps, n, device=DEV), [[] for _ in range(n)], [0] * n, [True] * n
    for j in range(steps):
        for s in range(n):
            u, good = a_draw(logits[s].double().cpu().numpy(), t, top_k, rng)
            U[j, s] = u
            certain[s] &= bool(good)
            sure[s] += certain[s]
        token = plain.decode(logits, 1, temperature=t, top_k=top_k, u=U[j:j + 1])[0][:, 0] + first_id(run)
        for s in range(n):
            want[s].append(int(token[s]))
        logits = plain.forward([0, 1, 2], token.to(torch.int32), [1] * n)[1]
    assert sum(sure) >= 24
    paged, logits = started(run, patches, ids)
    have, longest = [[w[0]] for w in want], 0
    while min(len(h) for h in have) < 16:
        tokens, parents, depths = [], [], []
        for s in range(n):
            right = want[s][len(have[s]):len(have[s]) + int(rng.integers(0, 6))]
            tree, parent, depth, at = [have[s][-1]], [-1], [0], 0
            for i, token in enumerate(right):
                for _ in range(int(rng.integers(0, 9))):
                    tree.append(first_id(run) + (token - first_id(run) + 1 + int(rng.integers(0, 200))) % 256)
                    parent.append(at), depth.append(i + 1)
                tree.append(token), parent.append(at), depth.append(i + 1)
                at = len(tree) - 1
            tokens.append(tree), parents.append(parent), depths.append(depth)
        u = torch.stack([U[min(len(have[s]) + d, steps - 1), s] for s in range(n) for d in depths[s]])
        new = paged.decode_drafts(tokens, parents, temperature=t, top_k=top_k, u=u)
        for s in range(n):
            longest = max(longest, len(new[s]))
            have[s] += new[s]
            m = min(len(have[s]), sure[s])
            assert have[s][:m] == want[s][:m], s
    assert longest > 3
