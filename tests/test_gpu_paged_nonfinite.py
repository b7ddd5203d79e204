"""vla_paged_attention where scores are not numbers: the row and head that has one gets NaN, in out and in lse, in every form and however its keys are split;
all others keep their values.  Tolerance of those: as in test_gpu_paged_attention.py."""
import numpy as np
import pytest
import torch

from paged_ref import DEV, TYPES, Batch, attention, gather
from paper_2510_06710_amd import binding as vb
from test_gpu_paged_attention import make

pytestmark = pytest.mark.gpu
HEADS, KV, D = 4, 2, 64
# form: sequences (rows, positions), the sequence and row that is spoilt, shared prefix
FORMS = {"undivided": ([(1, 60), (1, 128), (1, 33)], 1, 0, 0), "divided, few parts": ([(1, 150), (1, 190), (1, 90)], 1, 0, 0),
         "divided, many parts": ([(1, 40), (1, 3000), (1, 90)], 1, 0, 0), "prompt": ([(40, 40), (33, 65), (2, 9)], 1, 20, 0),
         "prompt, split": ([(70, 2500), (9, 40)], 0, 30, 0), "shared, single tokens": ([(1, 130), (1, 200), (1, 129)], 1, 0, 128),
         "shared, prompt": ([(50, 200), (60, 260)], 1, 59, 128)}


def call(b, dtype, q, pools, shared, cap):
    out, lse = torch.full((b.n_rows, HEADS, D), -77.0, dtype=TYPES[dtype], device=DEV), torch.full((b.n_rows, HEADS), -77.0, device=DEV)
    cache, batch, mask = vb.make_paged_cache(*[p.to(DEV) for p in pools]), b.on_device(), vb.make_paged_mask(D ** -0.5, cap, shared_len=shared)
    ws = torch.zeros(vb.vla_paged_attention_workspace_bytes(cache, batch, mask, HEADS), dtype=torch.uint8, device=DEV)
    vb.vla_paged_attention(cache, batch, mask, q.to(DEV), out, lse, ws)
    torch.cuda.synchronize()
    return out.double().cpu().numpy(), lse.double().cpu().numpy()


def check(b, dtype, q, pools, shared, cap, got, got_l, spoilt):
    """spoilt [rows, heads]: NaN wanted; None elsewhere: the values of the clean inputs q and pools."""
    o, l, mag, reach = attention(b, q.double().numpy(), *[p.double().numpy() for p in pools], D ** -0.5, cap)
    ds = D * 2.0 ** -24 * reach + cap * 2.0 ** -20 + reach * 2.0 ** -21
    n = max(n for _, n in b.spec)
    tol = (2 * ds[..., None] + n * 2.0 ** -24) * mag + ((mag + np.abs(o)) * 2.0 ** -8 if dtype == "bf16" else 0)
    assert np.isnan(got[spoilt]).all() and np.isnan(got_l[spoilt]).all()
    assert (np.abs(got - o) <= tol)[~spoilt].all()
    assert (np.abs(got_l - l) <= ds + n * 2.0 ** -24 + np.abs(l) * 2.0 ** -22)[~spoilt].all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap", [0.0, 8.0])
@pytest.mark.parametrize("form", FORMS)
def test_query_that_is_no_number(form, dtype, cap):
    spec, s, i, shared = FORMS[form]
    b = Batch(spec, 32, shared=shared)
    q, pools = make(b, dtype, HEADS, KV, D, 0, None, 0, shared)
    bad, row, head = q.clone(), int(b.start[s]) + i, 2
    bad[row, head, 5] = float("nan")
    spoilt = np.zeros((b.n_rows, HEADS), bool)
    spoilt[row, head] = True
    check(b, dtype, q, pools, shared, cap, *call(b, dtype, bad, pools, shared, cap), spoilt)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
@pytest.mark.parametrize("form", [f for f in FORMS if "prompt" not in f])          # (where no row of the call masks the key)
def test_key_that_is_no_number(form, dtype, value):
    spec, s, i, shared = FORMS[form]
    b = Batch(spec, 32, shared=shared)
    q, pools = make(b, dtype, HEADS, KV, D, 0, None, 1, shared)
    at = spec[s][1] - 1 if shared else spec[s][1] // 2           # behind the shared pages, so that one sequence alone sees it
    page, place = b.place(s, at)
    group = HEADS // KV
    row = int(b.start[s]) + i
    bad = [p.clone() for p in pools]
    bad[0][page, 1, place, 7] = value
    spoilt = np.zeros((b.n_rows, HEADS), bool)
    spoilt[row, group:] = True
    if value == float("inf"):                                    # a score of +inf: no number among the weights
        q[row, group:, 7] = q[row, group:, 7].abs() + 0.5
    check(b, dtype, q, pools, shared, 0.0, *call(b, dtype, q, bad, shared, 0.0), spoilt)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("form", [f for f in FORMS if "shared" not in f])          # (every sequence with rows holds the shared positions)
def test_rows_without_keys_stay_zeros(form, dtype):
    """Parts without a visible key still count for nothing."""
    spec, s, i, shared = FORMS[form]
    b = Batch([(n, 0 if j == s else length) for j, (n, length) in enumerate(spec)], 32, max_len=max(n for _, n in spec))
    q, pools = make(b, dtype, HEADS, KV, D, 0, None, 2, shared)
    got, got_l = call(b, dtype, q, pools, shared, 0.0)
    rows = slice(int(b.start[s]), int(b.start[s + 1]))
    assert (got[rows] == 0).all() and (got_l[rows] == -np.inf).all()
    others = np.ones(b.n_rows, bool)
    others[rows] = False
    assert np.isfinite(got[others]).all() and np.isfinite(got_l[others]).all()
