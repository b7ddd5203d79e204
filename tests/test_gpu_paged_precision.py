"""What vla_paged_attention keeps of a softmax weight on a bf16 cache where a sequence has up to 32 rows x heads of a key head: as much as the attention on the contiguous cache.

Tolerance, with A = sum w |v|: a weight is taken as a bf16 head and a bf16 tail, each off by half a step, so by 2^-8 of 2^-8 in all: 2^-16 A; scores, sums and the
output as in test_gpu_paged_attention.py: (2 ds + n 2^-24) A + 2^-8 |o|.  One bf16 alone would be off by 2^-8 A at most and by about 2^-9 A / sqrt(n) often, which outputs
near zero show."""
import numpy as np
import pytest
import torch

from paged_ref import DEV, Batch, attention
from paper_2510_06710_amd import binding as vb
from test_gpu_paged_attention import make

pytestmark = pytest.mark.gpu
FORMS = {"undivided": ([(1, 3 + s) for s in range(100)], 0), "divided": ([(1, 900), (1, 300), (1, 7)], 0), "few rows": ([(4, 40), (3, 200), (3, 9)], 0),
         "shared": ([(1, 65 + s) for s in range(30)], 64), "shared, few rows": ([(5, 60), (2, 160)], 64), "long shared": ([(1, 1025 + s) for s in range(30)], 1024)}


@pytest.mark.parametrize("heads,kv,d", [(8, 4, 16), (4, 4, 64), (4, 2, 128), (2, 2, 256)])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("cap,bias", [(0.0, False), (20.0, False), (0.0, True)])
def test_weights(form, heads, kv, d, cap, bias):
    spec, shared = FORMS[form]
    b = Batch([(n, max(l, shared)) for n, l in spec], 64, shared=shared)
    q, pools = make(b, "bf16", heads, kv, d, 0, None, 3, shared)
    slopes = 2.0 ** (-8.0 * (torch.arange(heads) + 1.0) / heads) / 16 if bias else None
    out = torch.zeros(b.n_rows, heads, d, dtype=torch.bfloat16, device=DEV)
    cache, batch, mask = vb.make_paged_cache(*[p.to(DEV) for p in pools]), b.on_device(), vb.make_paged_mask(d ** -0.5, cap, None if slopes is None else slopes.to(DEV), shared_len=shared)
    ws = torch.empty(vb.vla_paged_attention_workspace_bytes(cache, batch, mask, heads), dtype=torch.uint8, device=DEV)
    vb.vla_paged_attention(cache, batch, mask, q.to(DEV), out, None, ws)
    torch.cuda.synchronize()
    o, _, mag, reach = attention(b, q.double().numpy(), *[p.double().numpy() for p in pools], d ** -0.5, cap, None if slopes is None else slopes.double().numpy())
    n = max(n for _, n in spec)
    size = reach + (n * slopes.double().numpy() if bias else 0)
    ds = d * 2.0 ** -24 * reach + cap * 2.0 ** -20 + size * 2.0 ** -21
    off = np.abs(out.double().cpu().numpy() - o)
    assert (off <= (2 * ds[..., None] + n * 2.0 ** -24 + 2.0 ** -16) * mag + 2.0 ** -8 * np.abs(o)).all()
