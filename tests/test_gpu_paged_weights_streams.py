"""Summed weights that get more room on another stream than their own."""
import pytest
import torch

from paged_ref import DEV
from test_gpu_paged_less_rollout import SHAPES, first_id, setup, started

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_weights_in_use_elsewhere_are_not_given_out(name):
    run, patches, ids = setup(SHAPES[name], [(0, 1020), (0, 30)])
    paged, stream = started(run, patches, ids, n_pages=140, weigh=True)[0], torch.cuda.Stream()
    before = paged.mass.clone()
    torch.cuda.synchronize()
    size, place = before.numel(), paged.mass.data_ptr()
    with torch.cuda.stream(stream):
        torch.cuda._sleep(100_000_000)                       # (the copy to the larger array is yet to come)
        paged._room(2, 1025)
    fresh = [torch.full((size,), float("nan"), device=DEV) for _ in range(2)]
    assert all(t.data_ptr() != place for t in fresh)
    torch.cuda.synchronize()
    assert paged.mass.shape[3] == 2048 and torch.equal(paged.mass[..., :1024], before) and not paged.mass[..., 1024:].any()


@pytest.mark.parametrize("name", ["f32", "bf16"])
def test_calls_on_another_stream(name):
    run, patches, ids = setup(SHAPES[name], [(0, 1020), (0, 30)])
    token = torch.full((8,), first_id(run) + 5, dtype=torch.int32, device=DEV)
    both, stream = [started(run, patches, ids, n_pages=140, weigh=True)[0] for _ in range(2)], torch.cuda.Stream()
    torch.cuda.synchronize()
    for p, st in zip(both, (None, stream)):
        p.forward([0, 1], token, [7, 1], stream=st)
        p.decode_drafts([[int(token[0])] * 3, [int(token[0])]], [[-1, 0, 0], [-1]], stream=st)
        p.evict(900, first=4, recent=20, stream=st)
    torch.cuda.synchronize()
    assert both[0].length == both[1].length and torch.equal(both[0].mass, both[1].mass)
