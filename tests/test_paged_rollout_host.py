"""PagedRollout's own doings: buffers, pages and refusals, with the library's calls recorded (paged_stub.py)."""
import pytest
import torch

from paged_stub import Run, record
from paper_2510_06710_amd import binding as vb
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


def state(p):
    return [list(q) for q in p.pages], list(p.length), list(p.free), p.shared_len


def started(monkeypatch, n_pages=8):
    """Two sequences of 40 and 5 positions in pages of 16: four pages held."""
    calls = record(monkeypatch)
    p = PagedRollout(Run(), n_pages)
    p.prefill([None, None], [torch.zeros(40, dtype=torch.int32), ids(1, 2, 3, 4, 5)])
    del calls[:]
    return calls, p, state(p)


def refused(p, before, calls, error, call, match):
    with pytest.raises(error, match=match):
        call()
    assert state(p) == before and not calls


def test_what_the_pages_do_not_hold_is_refused_before_anything_changes(monkeypatch):
    calls, p, before = started(monkeypatch)
    patch = torch.zeros(30, 256)
    for call, match in ((lambda: p.prefill([None] * 3, [torch.zeros(48, dtype=torch.int32)] * 3), "9 pages wanted, 8 of 8 free"),
                        (lambda: p.prefill_group(torch.zeros(120, 256), torch.zeros(9, dtype=torch.int32), 2), "9 pages wanted, 8 of 8 free"),
                        (lambda: p.prefill_group(patch, ids(1, 2, 3, 4), 8), "7 pages wanted, 5 of 8 free"),          # two shared, one each behind them
                        (lambda: p.forward([0, 1], torch.zeros(80, dtype=torch.int32), [10, 70]), "5 pages wanted, 4 of 8 free"),
                        (lambda: p.decode(torch.zeros(2, 256), 60), "pages wanted, 4 of 8 free")):
        refused(p, before, calls, ValueError, call, match)
    p.decode(torch.zeros(2, 256), 28)                        # sequences of 67 and 32: seven pages
    assert p.length == [67, 32] and len(p.free) == 1 and [c.name for c in calls].count("forward") == 27


def test_what_the_library_refuses_changes_nothing(monkeypatch):
    calls, p, before = started(monkeypatch)
    for call in (lambda: p.prefill([None], [ids(1, 2)]), lambda: p.prefill_group(torch.zeros(30, 256), ids(1, 2, 3), 3), lambda: p.forward([1], ids(4), [1]),
                 lambda: p.decode(torch.zeros(2, 256), 2)):
        calls.fail = vb.VlaError(vb.VLA_ESHAPE, "no")
        with pytest.raises(vb.VlaError, match="no"):
            call()
        assert state(p) == before
        del calls[:]
    # more rows than one pass holds: the group's second half, found before its first runs
    run = Run()
    run.cfg.ffn = 1 << 18                                    # ... of a wide model fewer than 2048
    p = PagedRollout(run, 160)
    p.prefill([None], [ids(1, 2, 3)])
    before = state(p)
    del calls[:]
    refused(p, before, calls, vb.VlaError, lambda: p.prefill_group(torch.zeros(1, 256), torch.zeros(14, dtype=torch.int32), 150), "one pass can hold")


def test_group_lays_its_pages_out_once(monkeypatch):
    calls = record(monkeypatch)
    p = PagedRollout(Run(), 8)
    p.prefill_group(torch.zeros(30, 256), ids(7, 8, 9), 3)
    assert [len(q) for q in p.pages] == [3] * 3 and all(q[:2] == p.pages[0][:2] for q in p.pages) and len({q[2] for q in p.pages}) == 3
    assert p.length == [33] * 3 and p.shared_len == 32 and len(p.free) == 3
    first, rest = calls
    assert (first.lens, first.ids, first.shared_len) == ([33], [-1 - i for i in range(30)] + [7, 8, 9], 0)
    assert (rest.lens, rest.ids, rest.starts, rest.shared_len) == ([33, 33], [9, 9], [0, 1, 2], 32)


def test_calls_that_make_no_sense(monkeypatch):
    calls, p, before = started(monkeypatch)
    z, group = torch.zeros(2, 256), torch.zeros(3, 256)
    for call in (lambda: p.forward([0, 0], ids(1, 2), [1, 1]),                     # one sequence twice
                 lambda: p.forward([0, 2], ids(1, 2), [1, 1]), lambda: p.forward([-1], ids(1), [1]), lambda: p.forward([], ids(), []),
                 lambda: p.forward([0, 1], ids(1, 2), [2]), lambda: p.forward([0, 1], ids(1), [2, -1]), lambda: p.forward([0, 1], ids(1, 2, 3), [1, 1]),
                 lambda: p.prefill([None], [ids(1), ids(2)]), lambda: p.prefill([], []), lambda: p.prefill_group(group, ids(1), 0), lambda: p.prefill_group(group, ids(1), -3),
                 lambda: p.decode(torch.zeros(1, 256), 2), lambda: p.decode(torch.zeros(3, 256), 2), lambda: p.decode(z, 0),
                 lambda: p.decode(z, 3, u=torch.zeros(2, 2)), lambda: p.decode(z, 3, u=torch.zeros(3, 1)), lambda: p.decode(z, 3, u=torch.zeros(3))):
        refused(p, before, calls, ValueError, call, "sequences|rows|ids|rollouts|tokens|u is")
    p.decode(z, 2, u=torch.zeros(3, 2))                      # numbers for more tokens than are wanted
    p.forward([1, 0], ids(1, 2, 3), [3, 0])                  # another order, and one without new rows
    assert p.length == [41, 9] and calls[-1].lens == [9, 41] and calls[-1].starts == [0, 3, 3]


def test_group_without_patches(monkeypatch):
    calls = record(monkeypatch)
    p = PagedRollout(Run(), 8)
    p.prefill_group(None, torch.arange(20, dtype=torch.int32), 2)
    first, rest = calls
    assert first.ids == list(range(20)) and rest.ids == [16, 17, 18, 19] and first.patch is rest.patch is None


@pytest.mark.parametrize("group", [1, 2])
def test_group_of_a_patch_that_is_a_view(monkeypatch, group):
    calls = record(monkeypatch)
    wide = torch.arange(20 * 512, dtype=torch.float32).view(20, 512)
    PagedRollout(Run(), 8).prefill_group(wide[:, ::2], ids(1, 2, 3), group)
    assert len(calls) == group and all(c.patch.is_contiguous() and torch.equal(c.patch, wide[:, ::2]) for c in calls)
