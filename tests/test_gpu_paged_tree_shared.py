"""Trees behind a prefix that sequences share, whose end falls inside a tile of 32 keys: every key is read once, whatever lies between the prefix and the new rows.

Tolerances: those of test_gpu_paged_tree.py; of two evaluations of the decoder, twice parity.py's."""
import numpy as np
import pytest
import torch

from paged_less_ref import ancestors, random_tree
from paged_ref import DEV, Batch
from paper_2510_06710_amd.harness import PagedRollout
from parity import TOL
from test_gpu_paged_less_rollout import SHAPES, first_id, setup
from test_gpu_paged_tree import attend, trees

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("dtype", ["bf16", "f32"])


@BOTH
@pytest.mark.parametrize("shared", [16, 48, 272])
@pytest.mark.parametrize("heads,kv,most", [(4, 2, 5), (4, 4, 1), (8, 2, 40), (6, 1, 17)])
def test_from_0_to_15_positions_between(dtype, shared, heads, kv, most):
    """One to 32 packed rows of a sequence, and more."""
    new = [1 + 7 * gap % most for gap in range(16)]
    new[3] = most
    b = Batch([(n, shared + gap + n) for gap, n in enumerate(new)] + [(0, shared + 9)], 16, shared=shared, padding=1)
    see = [ancestors(t)[0] if t else [] for t in trees(b, shared)]
    attend(b, dtype, heads, kv, 64, see, shared=shared, seed=shared)
    attend(b, dtype, heads, kv, 64, see, cap=3.0, shared=shared, seed=shared + 5)


@BOTH
def test_any_bits_behind_a_shared_prefix(dtype):
    rng = np.random.default_rng(3)
    for spec in ([(3, 16 + 3), (16, 16 + 16), (5, 16 + 11)], [(40, 48 + 40), (33, 48 + 40), (1, 48 + 16)]):
        shared = 16 if spec[0][0] == 3 else 48
        attend(Batch(spec, 16, shared=shared), dtype, 4, 2, 128, [rng.random((n, n)) < 0.6 for n, _ in spec], shared=shared)


@pytest.mark.parametrize("name", ["f32", "bf16"])
@pytest.mark.parametrize("n", [17, 20, 31, 55, 275])
def test_drafts_of_a_group(name, n):
    """decode_drafts behind prefill_group is what it is behind a prefill of each rollout by itself."""
    run, patches, ids = setup(SHAPES[name], [(n - 3, 3)])
    group = PagedRollout(run, 96)
    group.prefill_group(patches[0], ids[0], 3)
    alone = PagedRollout(run, 96)
    alone.prefill(patches * 3, ids * 3)
    assert group.shared_len == (n - 1) // 16 * 16 and alone.length == group.length
    rng = np.random.default_rng(n)
    parents = [random_tree(k, rng) for k in (9, 1, 17)]
    tokens = [[first_id(run) + int(t) for t in rng.integers(0, 256, len(p))] for p in parents]
    before = list(group.length)
    got, want = group.decode_drafts(tokens, parents), alone.decode_drafts(tokens, parents)
    if name == "f32":
        assert got == want
    for s in range(3):
        if name == "f32":                                     # K and V of the last layer, which the first one's attention shows in
            rows = [torch.stack([p.pools[i][-1, p.pages[s][at // 16], :, at % 16] for i in range(2) for at in range(before[s], p.length[s])]) for p in (group, alone)]
            assert (rows[0] - rows[1]).abs().max().item() <= 2 * TOL[name]["logits"]
    if got == want:                                           # (bf16: unless rounding turned a choice over)
        last = torch.tensor([g[-1] for g in got], dtype=torch.int32, device=DEV)
        a, b = group.forward([0, 1, 2], last, [1] * 3)[1], alone.forward([0, 1, 2], last, [1] * 3)[1]
        assert (a - b).abs().max().item() <= 2 * TOL[name]["logits"]
