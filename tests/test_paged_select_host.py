"""PagedRollout.decode on selected pages: what is refused, before anything changes (paged_stub.py)."""
import pytest
import torch

from paged_stub import Run, record
from paper_2510_06710_amd import binding as vb
from paper_2510_06710_amd.harness import PagedRollout


def test_more_pages_than_are_chosen_from_are_refused_before_the_first_token(monkeypatch):
    calls = record(monkeypatch)
    monkeypatch.setattr(vb, "vla_paged_bounds", lambda *a, **k: None)
    monkeypatch.setattr(vb, "vla_forward_paged_rows", lambda *a, **k: calls.append("rows"))
    p = PagedRollout(Run(), 8200)
    p.prefill([None], [torch.zeros(16 * 8192 - 2, dtype=torch.int32)])
    before = [list(p.pages[0]), list(p.length), list(p.free)]
    del calls[:]
    with pytest.raises((ValueError, vb.VlaError), match="8193 pages"):
        p.decode(torch.zeros(1, 256), 5, select=4)           # the last two of its four new positions lie on a page too many
    assert [p.pages[0], p.length, p.free] == before and not calls
    p.decode(torch.zeros(1, 256), 3, select=4)
    assert p.length == [16 * 8192] and calls.count("rows") == 2
    p.decode(torch.zeros(1, 256), 3)                         # (all pages may be read)
