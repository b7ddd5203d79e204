"""Several PagedRollouts and streams at once."""
import pytest
import torch

from paper_2510_06710_amd.harness import PagedRollout
from test_gpu_paged_rollout import DEV, setup

pytestmark = pytest.mark.gpu


def test_two_rollouts_of_one_model_at_once():
    lengths = [[(48, 21), (5, 3), (90, 40)], [(60, 30), (7, 2), (16, 8)]]
    run, first, _, _ = setup("bf16", lengths[0])
    obs = [first, setup("bf16", lengths[1], seed=9)[1]]
    u = torch.rand(6, 3, generator=torch.Generator().manual_seed(1)).to(DEV)
    both, streams = [PagedRollout(run, 32) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]

    def go(i, stream):
        logits = both[i].prefill([p for p, _ in obs[i]], [t for _, t in obs[i]], stream=stream)[1]
        return both[i].decode(logits, 6, top_k=40, u=u, stream=stream)

    alone = [go(i, None) for i in range(2)]
    torch.cuda.synchronize()
    for _ in range(5):
        together = [go(i, streams[i]) for i in range(2)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for i in range(2) for a, b in zip(alone[i], together[i]))


def test_a_workspace_in_use_elsewhere_is_not_given_out():
    run, obs, _, _ = setup("bf16", [(48, 21), (5, 3)])
    paged, stream = PagedRollout(run, 32), torch.cuda.Stream()
    logits = paged.prefill([p for p, _ in obs], [t for _, t in obs])[1]          # the workspace comes from the current stream's memory
    torch.cuda.synchronize()
    paged.decode(logits, 2, stream=stream)
    with torch.cuda.stream(stream):
        torch.cuda._sleep(100_000_000)                       # the stream is not through with it ...
    size, place = paged._bufs["ws_paged"].numel(), paged._bufs["ws_paged"].data_ptr()
    paged._bufs.clear()                                      # ... when a larger one takes its place
    fresh = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(2)]
    assert all(t.data_ptr() != place for t in fresh)
    torch.cuda.synchronize()
