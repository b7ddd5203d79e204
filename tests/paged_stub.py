"""A PagedRollout on the CPU whose library calls are recorded instead of made: what it hands to the library and what it keeps, without a GPU."""
import types

import torch

import vla_inputs as vi
from paper_2510_06710_amd import binding as vb
from paper_2510_06710_amd.harness import Rollout


class Run:
    """What PagedRollout uses of a Rollout."""
    _buf = Rollout._buf

    def __init__(self):
        self.shape, self.device, self._bufs = vi.TINY, torch.device("cpu"), {}
        self.cfg = vb.make_config(vi.TINY, 4, 16)
        self.model = types.SimpleNamespace(handle=None, _keep=[None] * 5)

    def _value_out(self, n):
        return torch.empty(n)


def record(monkeypatch):
    """The library's calls from here on, in their order, with what the device arrays held.  `fail` of the list, an exception, is what the next forward raises."""
    class Calls(list):
        fail = None

    calls = Calls()

    def forward(model, cache, layer_stride, batch, ids, ws, h_last, patch=None, prefix_len=None, shared_len=0, logits=None, value=None, stream=None):
        if calls.fail is not None:
            fail, calls.fail = calls.fail, None
            raise fail
        starts, lens, table = batch.keep
        calls.append(types.SimpleNamespace(name="forward", starts=starts.tolist(), lens=lens.tolist(), table=table.tolist(), ids=ids.tolist(), ws=ws, shared_len=shared_len,
                                           patch=patch, prefix_len=None if prefix_len is None else prefix_len.tolist()))
        h_last.zero_(), logits.zero_()

    def sample(logits, token, *args, **kwargs):
        calls.append(types.SimpleNamespace(name="sample", ws=args[-1]))
        token.zero_()

    monkeypatch.setattr(vb, "vla_forward_paged", forward)
    monkeypatch.setattr(vb, "vla_sample_logits", sample)
    return calls
