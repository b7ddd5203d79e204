"""A cache cut right behind drafts that took it past the room of its summed weights."""
import pytest
import torch

from paged_ref import DEV
from test_gpu_paged_less_rollout import SHAPES, first_id, setup, started

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_drafts_past_the_room_of_the_weights(name):
    run, patches, ids = setup(SHAPES[name], [(0, 1022), (0, 20)])
    paged, logits = started(run, patches, ids, n_pages=140, weigh=True)
    chain, plain = [], started(run, patches, ids, n_pages=140)
    token = (logits.argmax(1) + first_id(run)).to(torch.int32)
    for _ in range(6):                                        # what will be chosen, as far as rounding lets it
        chain.append(token.tolist())
        token = (plain[0].forward([0, 1], token, [1, 1])[1].argmax(1) + first_id(run)).to(torch.int32)
    before = paged.mass[:, 0, :, :1022].clone()
    paged.decode_drafts([[c[s] for c in chain] for s in range(2)], [[-1, 0, 1, 2, 3, 4]] * 2)
    if name == "f32":
        assert paged.length == [1028, 26]
    lengths = list(paged.length)
    pages = [list(p) for p in paged.pages]
    keys = paged.pools[0].clone()
    paged.evict(1000, first=2, recent=lengths[0] - 1022 + 1)
    assert paged.length == [1000, lengths[1]] and paged.shift == [lengths[0] - 1000, 0]
    for l in range(run.shape.n_layers):
        for h in range(run.shape.n_heads):
            m = before[l, h].double().tolist()
            always = {0, 1, *range(1021, lengths[0])}
            rest = sorted((j for j in range(2, 1021)), key=lambda j: (-m[j], j))[:1000 - len(always)]
            at = sorted(always | set(rest))
            was = torch.stack([keys[l, pages[0][j // 16], h, j % 16] for j in at])
            now = torch.stack([paged.pools[0][l, paged.pages[0][i // 16], h, i % 16] for i in range(1000)])
            assert torch.equal(was, now)
    last = torch.tensor([first_id(run) + 1] * 2, dtype=torch.int32, device=DEV)
    assert torch.isfinite(paged.forward([0, 1], last, [1, 1])[1]).all()
