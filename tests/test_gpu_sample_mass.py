"""The log-probability under softmax(z / T) does not depend on the cuts: equal bits whatever top_k, top_p and min_p are, and the value of the definition.

Tolerance: the rounding to fp32, 2^-24 of the value, and masses: 2^-45 a token and 1e-12 of each weight, against a total of at least 1."""
import numpy as np
import pytest
import torch

from paged_ref import DEV, TYPES
from paper_2510_06710_amd import binding as vb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [300, 999, 9000, 40000])
def test_cuts_do_not_move_it(dtype, vocab):
    n = 64
    # a leader, and all others alike: whatever the error of their one weight is, it does not average out
    z = torch.zeros(n, vocab)
    z[:, 1:] = -np.log(vocab) - torch.linspace(0.0, 3.0, n)[:, None]
    z = z.to(TYPES[dtype])
    ws = torch.empty(vb.vla_sample_logits_workspace_bytes(n, vocab), dtype=torch.uint8, device=DEV)
    every = lambda v, kind: torch.full((n,), v, dtype=kind, device=DEV)
    got = []
    for k, p, least in ((0, 1.0, 0.0), (1, 1.0, 0.0), (50, 1.0, 0.0), (vocab - 1, 1.0, 0.0), (0, 0.6, 0.0), (20, 0.9, 0.5), (0, 1.0, 0.5)):
        token, logp = torch.zeros(n, dtype=torch.int32, device=DEV), torch.zeros(n, device=DEV)
        vb.vla_sample_logits(z.to(DEV), token, top_k=every(k, torch.int32), top_p=every(p, torch.float32), min_p=every(least, torch.float32), logp=logp, ws=ws)
        assert (token == 0).all()
        got.append(logp.cpu())
    want = torch.log_softmax(z.double(), 1)[:, 0]
    off = (got[0].double() - want).abs()
    assert (off <= 2.0 ** -24 * want.abs() + vocab * 2.0 ** -45 + 2e-12).all()
    assert all(torch.equal(g, got[0]) for g in got[1:])


def test_same_as_among_the_kept_where_all_are_kept():
    n, vocab = 40, 2000
    z = (torch.randn(n, vocab, generator=torch.Generator().manual_seed(0)) * 2).to(DEV)
    z[:, 7] = float("-inf")
    ws = torch.empty(vb.vla_sample_logits_workspace_bytes(n, vocab), dtype=torch.uint8, device=DEV)
    token, logp, kept = torch.zeros(n, dtype=torch.int32, device=DEV), torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    for k in (vocab - 1, vocab, 0):                              # 1999 are there
        vb.vla_sample_logits(z, token, top_k=torch.full((n,), k, dtype=torch.int32, device=DEV), u=torch.rand(n, device=DEV), logp=logp, logp_kept=kept, ws=ws)
        assert torch.equal(logp, kept)
