"""vla_sample_logits against the definition in fp64: tokens and counts equal, log-probabilities within the rounding to fp32 (2^-24 of the value) and the
fixed point of the masses (2^-45 per token against a mass of at least 1: 2^18 tokens give 2^-27)."""
import numpy as np
import pytest
import torch

from paged_ref import DEV, TYPES, sample
from paper_2510_06710_amd import binding as vb

pytestmark = pytest.mark.gpu


def run(z, settings, dtype="f32", pad=0, skip=()):
    """settings: dict of per-row lists (temperature, top_k, top_p, min_p, u)."""
    z = torch.as_tensor(z).to(TYPES[dtype])
    n, vocab = z.shape
    wide = torch.full((n, vocab + pad), 99.0, dtype=TYPES[dtype])
    wide[:, :vocab] = z
    zd = wide.to(DEV)[:, :vocab]
    kinds = dict(temperature=torch.float32, top_k=torch.int32, top_p=torch.float32, min_p=torch.float32, u=torch.float32)
    host = {k: torch.tensor(v, dtype=kinds[k]) for k, v in settings.items() if k not in skip}
    outs = dict(token=torch.full((n,), -9, dtype=torch.int32, device=DEV), n_kept=torch.full((n,), -9, dtype=torch.int32, device=DEV),
                logp=torch.full((n,), 9.0, device=DEV), logp_kept=torch.full((n,), 9.0, device=DEV))
    ws = torch.empty(vb.vla_sample_logits_workspace_bytes(n, vocab), dtype=torch.uint8, device=DEV).fill_(255)
    for _ in range(2):
        vb.vla_sample_logits(zd, outs["token"], **{k: v.to(DEV) for k, v in host.items()}, logp=outs["logp"], logp_kept=outs["logp_kept"], n_kept=outs["n_kept"], ws=ws)
    torch.cuda.synchronize()
    got = {k: v.cpu().double().numpy() for k, v in outs.items()}
    only = torch.full((n,), -9, dtype=torch.int32, device=DEV)
    vb.vla_sample_logits(zd, only, **{k: v.to(DEV) for k, v in host.items()}, ws=ws)
    assert torch.equal(only, outs["token"])
    pick = lambda name, i, other: host[name][i].item() if name in host else other
    for i in range(n):
        want = sample(z[i].double().numpy(), pick("temperature", i, 1.0), pick("top_k", i, 0), pick("top_p", i, 1.0), pick("min_p", i, 0.0), pick("u", i, None))
        assert (got["token"][i], got["n_kept"][i]) == want[:2], (i, got["token"][i], got["n_kept"][i], want)
        for name, w in (("logp", want[2]), ("logp_kept", want[3])):
            assert got[name][i] == w or abs(got[name][i] - w) <= 2.0 ** -24 * abs(w) + 2.0 ** -26, (i, name, got[name][i], w)


def mixed(n, seed):
    r = np.random.default_rng(seed)
    return dict(temperature=r.choice([1.0, 0.7, 1.6, 0.0], n, p=[.4, .3, .2, .1]), top_k=r.choice([0, 0, 1, 2, 20, 300, 10 ** 6], n), top_p=r.choice([1.0, 0.95, 0.5, 0.1, 0.0, 1.5], n),
                min_p=r.choice([0.0, 0.0, 0.05, 0.3, 1.0], n), u=r.choice([0.0, 1 - 2.0 ** -24, -1.0], n) * (r.uniform(size=n) < 0.1) + r.uniform(size=n).astype(np.float32) * 0.999)


def positive(s):
    s["u"] = np.clip(s["u"], 0.0, 1 - 2.0 ** -24)
    return s


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,vocab", [(64, 256), (40, 1), (40, 2), (33, 255), (33, 1000), (20, 4097), (24, 32000), (9, 131071), (3, 262144)])
def test_settings(dtype, n, vocab):
    r = np.random.default_rng(vocab)
    run(r.standard_normal((n, vocab)) * 3, positive(mixed(n, vocab)), dtype)
    run(r.standard_normal((n, vocab)) * 0.1, positive(mixed(n, vocab + 1)), dtype, pad=3)          # flat: long leading runs


@pytest.mark.parametrize("skip", [("u",), ("temperature", "top_k"), ("top_p", "min_p"), ("temperature", "top_k", "top_p", "min_p"), ("temperature", "top_k", "top_p", "min_p", "u")])
def test_settings_left_out(skip):
    run(np.random.default_rng(5).standard_normal((50, 999)) * 2, positive(mixed(50, 6)), skip=skip)


@pytest.mark.parametrize("vocab", [7, 300, 5000, 40000])
def test_equal_logits_and_few_values(vocab):
    n = 24
    r = np.random.default_rng(vocab)
    run(np.full((n, vocab), -3.25), positive(mixed(n, 1)))
    run(r.integers(0, 3, (n, vocab)) * 0.5, positive(mixed(n, 2)))
    run(np.where(r.uniform(size=(n, vocab)) < 0.5, 0.0, -0.0), positive(mixed(n, 3)))               # both zeros are one value


@pytest.mark.parametrize("vocab", [9, 700, 33000])
def test_masked_and_strange_logits(vocab):
    n = 30
    r = np.random.default_rng(vocab)
    z = r.standard_normal((n, vocab)) * 2
    z[r.uniform(size=z.shape) < 0.5] = -np.inf
    z[r.uniform(size=z.shape) < 0.1] = np.nan
    z[0], z[1], z[2] = -np.inf, np.nan, -3.3895e38           # nothing; nothing; the type's lowest value everywhere
    z[3, :], z[3, vocab // 2] = -np.inf, 1.0                 # one token left
    z[4, ::3] = np.inf
    z[5, -1] = np.inf
    z[6] = np.where(np.arange(vocab) % 2, -3.3895e38, z[6])
    z[7, 0] = 3.3895e38                                      # the largest value
    for dtype in ("f32", "bf16"):
        run(z, positive(mixed(n, 4)), dtype)


def test_wide_ranges():
    n, vocab = 24, 3000
    r = np.random.default_rng(3)
    run(r.standard_normal((n, vocab)) * 1000, positive(mixed(n, 7)))
    run(r.standard_normal((n, vocab)) * 1e-6, positive(mixed(n, 8)))
    s = positive(mixed(n, 9))
    s["temperature"] = np.where(np.arange(n) % 2, 1e-3, 100.0)
    run(r.standard_normal((n, vocab)) * 3, s)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_flat_logits(dtype):
    """More tokens in one step of the value than are sorted."""
    n, vocab = 12, 100003
    s = positive(mixed(n, 11))
    s["top_k"] = np.where(np.arange(n) % 2, 20000, 0)
    run(np.random.default_rng(12).standard_normal((n, vocab)) * 0.05, s, dtype)
