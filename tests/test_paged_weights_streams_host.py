"""Which memory of a PagedRollout that sums weights is marked as used by the stream that a call goes to: on the CPU, with the library's calls recorded (paged_stub.py)."""
import types

import pytest
import torch

from paged_stub import Run, record
from paper_2510_06710_amd import binding as vb
from paper_2510_06710_amd.harness import PagedRollout

ids = lambda *v: torch.tensor(v, dtype=torch.int32)


@pytest.fixture
def rollout(monkeypatch):
    """A rollout of two sequences, 1020 and 5 positions, and the addresses that were marked since its last call began."""
    record(monkeypatch)
    marked = []
    monkeypatch.setattr(torch.Tensor, "is_cuda", property(lambda t: True))
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, stream: marked.append((t.data_ptr(), stream)))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: "here")

    def forward_rows(model, cache, layer_stride, n_layers, batch, rows, ids, ws, logits, patch=None, shared_len=0, stream=None):
        logits.zero_()

    def accept(cache, n_layers, layer_stride, batch, parent, ids, chosen, path, n_accepted, next=None, new_len=None, stream=None):
        path.fill_(-1), path[:, 0].zero_(), n_accepted.fill_(1), next.zero_()
        starts, lens, _ = batch.keep
        new_len.copy_(lens - (starts[1:] - starts[:-1]) + 1)

    monkeypatch.setattr(vb, "vla_forward_paged_rows", forward_rows)
    monkeypatch.setattr(vb, "vla_paged_accept", accept)
    for name in ("vla_paged_tree", "vla_paged_evict"):
        monkeypatch.setattr(vb, name, lambda *a, **k: None)
    p = PagedRollout(Run(), 160, weigh=True)
    p.prefill([None, None], [torch.zeros(1020, dtype=torch.int32), ids(1, 2, 3, 4, 5)])
    return types.SimpleNamespace(p=p, marked=marked)


def test_every_call_marks_the_weights_it_uses(rollout):
    p = rollout.p
    for call in (lambda: p.forward([0, 1], ids(1, 2), [1, 1]), lambda: p.decode(torch.zeros(2, 256), 2), lambda: p.decode_drafts([[1, 2], [3]], [[-1, 0], [-1]]), lambda: p.evict(100)):
        before = p.mass.data_ptr()
        del rollout.marked[:]
        call()
        assert p.mass.data_ptr() == before and (before, "here") in rollout.marked


@pytest.mark.parametrize("drafts", [False, True])
def test_what_is_replaced_by_more_room_is_marked_too(rollout, drafts):
    p, old = rollout.p, rollout.p.mass
    del rollout.marked[:]
    if drafts:
        p.decode_drafts([[1] * 6, [3]], [[-1, 0, 1, 2, 3, 4], [-1]])
    else:
        p.forward([0, 1], torch.zeros(12, dtype=torch.int32), [10, 2])
    assert p.mass.shape[3] == 2048 and p.mass.data_ptr() != old.data_ptr()
    assert (old.data_ptr(), "here") in rollout.marked
