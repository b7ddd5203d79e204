"""PagedRollout's own doings: buffers, pages and refusals, with the library's calls recorded (paged_stub.py)."""
import torch

from paged_stub import Run, record
from paper_2510_06710_amd.harness import PagedRollout

ids = lambda *v: torch.tensor(v, dtype=torch.int32)


def test_two_on_one_model_have_buffers_of_their_own(monkeypatch):
    calls, run = record(monkeypatch), Run()
    a, b = PagedRollout(run, 8), PagedRollout(run, 8)
    for p in (a, b):
        p.prefill([None], [ids(1, 2, 3)])
        p.decode(torch.zeros(1, 256), 2)
    places = [{c.ws.data_ptr() for c in calls[i:i + 4]} for i in (0, 4)]
    assert [c.name for c in calls] == ["forward", "sample", "forward", "sample"] * 2
    assert not places[0] & places[1]
