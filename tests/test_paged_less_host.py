"""Refusals of the operators that read less per token, and their size queries: host code, no device."""
import ctypes as C

import pytest
import torch

from paper_2510_06710_amd import binding as vb
from test_paged_host import BAD_BOTH, P, batch, cache

E, S, W = vb.VLA_EINVAL, vb.VLA_ESHAPE, vb.VLA_EWORKSPACE


def mask(**k):
    m = vb.vla_paged_mask(0.125, 0.0, None, None, 0, 0)
    for name, v in k.items():
        setattr(m, name, v)
    return m


def call(name, c=None, b=None, m=None, **k):
    """The entry point with arguments that are right but for those given; all arrays at one made-up address (nothing is launched for what is refused)."""
    a = dict(position=P, parent=P, seen=P, words=1, q=P, k=P, v=P, qo=P + 0x100000, heads=4, qs=256, out=P, os=256, ws=P, n=1 << 40, layers=3, stride=1 << 20, ids=P, chosen=P, path=P,
             count=P, bounds=P, most=4, first=1, recent=1, selected=P, lse=P, mass=P, ms=64, keep=32, to=P, ts=2, kept=P, mo=P + 0x100000, mos=32)
    assert set(k) <= set(a)
    a.update(k)
    c, b, m = c or cache(), b or batch(), m or mask()
    cb, L = (C.byref(c), C.byref(b)), vb.lib()
    rot = vb.vla_rotary(P, 64, 0, 1.0, 1e-6, None, None)
    if name == "append_at":
        return L.vla_paged_append_at(*cb, C.byref(rot), a["position"], a["q"], a["k"], a["v"], vb.VLA_DTYPE_F32, a["heads"], a["qs"], 128, 128, a["qo"], 256, None)
    if name == "tree":
        return L.vla_paged_tree(*cb, a["parent"], a["seen"], a["words"], a["position"], None)
    if name == "tree_attention":
        return L.vla_paged_tree_attention(*cb, C.byref(m), a["seen"], a["words"], a["q"], a["heads"], a["qs"], a["out"], a["os"], None, a["ws"], a["n"], None)
    if name == "accept":
        return L.vla_paged_accept(cb[0], a["layers"], a["stride"], cb[1], a["parent"], a["ids"], a["chosen"], a["path"], a["count"], None, None, None)
    if name == "bounds":
        return L.vla_paged_bounds(*cb, a["bounds"], None)
    if name == "select":
        return L.vla_paged_select(*cb, a["bounds"], a["q"], a["heads"], a["qs"], a["most"], a["first"], a["recent"], a["selected"], a["ws"], a["n"], None)
    if name == "sparse_attention":
        return L.vla_paged_sparse_attention(*cb, C.byref(m), a["selected"], a["most"], a["q"], a["heads"], a["qs"], a["out"], a["os"], None, a["ws"], a["n"], None)
    if name == "weights":
        return L.vla_paged_weights(*cb, C.byref(m), a["q"], a["heads"], a["qs"], a["lse"], a["mass"], a["ms"], a["ws"], a["n"], None)
    return L.vla_paged_evict(*cb, a["mass"], a["ms"], a["keep"], a["first"], a["recent"], a["to"], a["ts"], a["kept"], a["mo"], a["mos"], None, None)


NAMES = ["append_at", "tree", "tree_attention", "accept", "bounds", "select", "sparse_attention", "weights", "evict"]


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("c,b,code", BAD_BOTH)
def test_cache_and_batch(name, c, b, code):
    assert call(name, cache(**c), batch(**b)) == code
    assert vb.vla_last_error()


REFUSED = {
    "append_at": [(dict(position=None), E), (dict(k=None), E), (dict(qs=255), S)],
    "tree": [(dict(parent=None), E), (dict(seen=None), E), (dict(words=0), S), (dict(words=33), S)],
    "tree_attention": [(dict(seen=None), E), (dict(words=0), S), (dict(words=33), S), (dict(q=None), E), (dict(out=None), E), (dict(ws=None), E), (dict(ws=P + 4), E), (dict(n=16), W),
                       (dict(heads=3), S), (dict(heads=0), S), (dict(qs=255), S), (dict(os=255), S)],
    "accept": [(dict(layers=-1), E), (dict(layers=70000), E), (dict(stride=100), S), (dict(stride=(1 << 20) + 1), E), (dict(parent=None), E), (dict(ids=None), E), (dict(chosen=None), E),
               (dict(path=None), E), (dict(count=None), E)],
    "bounds": [(dict(bounds=None), E), (dict(bounds=P + 8), E)],
    "select": [(dict(bounds=None), E), (dict(bounds=P + 8), E), (dict(q=None), E), (dict(selected=None), E), (dict(ws=None), E), (dict(ws=P + 4), E), (dict(n=16), W), (dict(heads=3), S),
               (dict(qs=255), S), (dict(recent=0), E), (dict(first=-1), E), (dict(most=1), E), (dict(most=9000), E), (dict(first=2 ** 31 - 1, recent=2 ** 31 - 1), E)],
    "sparse_attention": [(dict(selected=None), E), (dict(q=None), E), (dict(out=None), E), (dict(ws=None), E), (dict(ws=P + 4), E), (dict(n=16), W), (dict(heads=3), S), (dict(qs=255), S),
                         (dict(os=255), S), (dict(most=0), S), (dict(most=9000), S)],
    "weights": [(dict(q=None), E), (dict(lse=None), E), (dict(mass=None), E), (dict(ws=None), E), (dict(ws=P + 4), E), (dict(n=16), W), (dict(heads=3), S), (dict(qs=255), S), (dict(ms=39), S)],
    "evict": [(dict(mass=None), E), (dict(to=None), E), (dict(kept=None), E), (dict(mo=None), E), (dict(keep=0), E), (dict(first=-1), E), (dict(recent=-1), E), (dict(first=20, recent=20), E),
              (dict(ts=1), S), (dict(ts=-1), S), (dict(ms=39), S), (dict(mos=31), S), (dict(mo=P), S), (dict(first=2 ** 31 - 1, recent=2 ** 31 - 1), E)],
}


@pytest.mark.parametrize("name", NAMES)
def test_refuses(name):
    for k, code in REFUSED[name]:
        assert call(name, **k) == code, k


@pytest.mark.parametrize("name", ["tree_attention", "sparse_attention", "weights"])
def test_masks(name):
    nan, inf = float("nan"), float("inf")
    bad = [(dict(scale=0.0), E), (dict(scale=nan), E), (dict(scale=inf), E), (dict(softcap=-1.0), E), (dict(softcap=inf), E), (dict(window=-1), E)]
    if name != "weights":
        bad += [(dict(slopes=P), E), (dict(prefix_len=P), E), (dict(window=5), E)]
    if name == "sparse_attention":
        bad += [(dict(shared_len=16), E)]
    for m, code in bad:
        assert call(name, m=mask(**m)) == code, m


def test_sizes_of_trees_and_pages():
    long = dict(max_rows=1025, n_rows=1025, max_len=2000, table_stride=125)
    assert call("tree", b=batch(**long), words=33) == S and call("tree_attention", b=batch(**long), words=32) == S and call("accept", b=batch(**long)) == S
    assert call("tree", b=batch(max_rows=33), words=1) == S and call("tree_attention", b=batch(max_rows=33), words=1) == S
    assert call("select", b=batch(max_len=16 * 8192 + 1, table_stride=8193)) == S
    assert call("evict", c=cache(n_kv_heads=1024, head_dim=16), b=batch(n_seq=64)) == S
    assert call("evict", c=cache(n_kv_heads=1024, head_dim=16), b=batch(n_seq=63), keep=0) == E


def test_nothing_to_do():
    none = batch(n_rows=0)
    for name in ("append_at", "tree", "tree_attention", "bounds", "select", "sparse_attention", "weights"):
        assert call(name, b=none) == vb.VLA_OK, name


def test_workspace_queries():
    c, b, m, L = cache(), batch(), mask(), vb.lib()
    r = C.byref
    assert L.vla_paged_select_workspace_bytes(r(c), r(b)) > 0 and L.vla_paged_select_workspace_bytes(r(cache(dtype=9)), r(b)) == 0
    assert L.vla_paged_select_workspace_bytes(r(c), r(batch(max_len=16 * 8192 + 1, table_stride=8193))) == 0
    assert L.vla_paged_sparse_attention_workspace_bytes(r(c), r(b), r(m), 4, 3) > 0 and L.vla_paged_sparse_attention_workspace_bytes(r(c), r(b), r(m), 4, 0) == 0
    assert L.vla_paged_weights_workspace_bytes(r(c), r(b), r(m), 4) > 0 and L.vla_paged_weights_workspace_bytes(r(c), r(b), r(m), 3) == 0
    assert L.vla_paged_weights_workspace_bytes(r(c), r(b), None, 4) == 0


z = torch.zeros
I = torch.int32


def test_binding_refuses():
    """Shapes, types and places that the library could not see; the tensors are the host's, which is refused last."""
    pool = z(8, 2, 16, 64)
    c = vb.make_paged_cache(pool, pool)
    b = vb.make_paged_batch(z(3, dtype=I), z(2, dtype=I), z(2, 3, dtype=I), 5, 3, 40)
    m, q, row, seen, sel, mass = vb.make_paged_mask(1.0), z(5, 4, 64), z(5, dtype=I), z(5, 1, dtype=I), z(5, 2, 4, dtype=I), z(2, 2, 40)
    good = {"tree": lambda **k: vb.vla_paged_tree(c, b, k.get("parent", row), k.get("seen", seen), k.get("position", row)),
            "tree_attention": lambda **k: vb.vla_paged_tree_attention(c, b, m, k.get("seen", seen), k.get("q", q), k.get("out", q), k.get("lse"), z(9)),
            "accept": lambda **k: vb.vla_paged_accept(c, 1, 0, b, k.get("parent", row), k.get("ids", row), k.get("chosen", row), k.get("path", z(2, 3, dtype=I)), k.get("count", z(2, dtype=I)),
                                                      k.get("next"), k.get("new_len")),
            "bounds": lambda **k: vb.vla_paged_bounds(c, b, k.get("bounds", z(8, 2, 2, 64))),
            "select": lambda **k: vb.vla_paged_select(c, b, k.get("bounds", z(8, 2, 2, 64)), k.get("q", q), k.get("selected", sel), 1, 1, z(9)),
            "sparse": lambda **k: vb.vla_paged_sparse_attention(c, b, m, k.get("selected", sel), k.get("q", q), k.get("out", q), k.get("lse"), z(9)),
            "weights": lambda **k: vb.vla_paged_weights(c, b, k.get("mask", m), k.get("q", q), k.get("lse", z(5, 4)), k.get("mass", mass), z(9)),
            "evict": lambda **k: vb.vla_paged_evict(c, b, k.get("mass", mass), 0, 1, k.get("to", z(2, 2, dtype=I)), k.get("kept", z(2, 2, 20, dtype=I)), k.get("out", z(2, 2, 20)), k.get("new_len")),
            "append_at": lambda **k: vb.vla_paged_append_at(c, b, vb.make_rotary(), k.get("position", row), q, z(5, 2, 64), z(5, 2, 64), z(5, 4, 64))}
    bad = {"tree": [dict(parent=z(4, dtype=I)), dict(parent=z(5)), dict(seen=row), dict(seen=z(5, 2, dtype=I)[:, :1]), dict(position=z(6, dtype=I))],
           "tree_attention": [dict(seen=row), dict(seen=z(4, 1, dtype=I)), dict(q=z(4, 4, 64)), dict(q=q.bfloat16()), dict(out=z(5, 3, 64)), dict(lse=z(5, 3)), dict(q=z(5, 64, 4).transpose(1, 2))],
           "accept": [dict(parent=z(4, dtype=I)), dict(ids=z(5)), dict(chosen=z(5, dtype=torch.int64)), dict(path=z(2, 4, dtype=I)), dict(count=z(3, dtype=I)), dict(next=z(2)), dict(new_len=z(1, dtype=I))],
           "bounds": [dict(bounds=z(8, 2, 2, 64).bfloat16()), dict(bounds=z(8, 2, 64, 2)), dict(bounds=z(8, 2, 2, 65)[..., :64])],
           "select": [dict(bounds=z(7, 2, 2, 64)), dict(q=q.bfloat16()), dict(selected=z(5, 4, 4, dtype=I)), dict(selected=z(5, 8, dtype=I)), dict(selected=sel.long())],
           "sparse": [dict(selected=z(5, 4, 4, dtype=I)), dict(selected=sel.transpose(0, 2).contiguous().transpose(0, 2)), dict(out=q.bfloat16()), dict(lse=z(4, 4))],
           "weights": [dict(lse=z(5, 3)), dict(lse=z(5, 4).double()), dict(mass=z(2, 4, 40)), dict(mass=z(2, 80)), dict(q=q.bfloat16()), dict(mask=vb.make_paged_mask(1.0, slopes=z(3))),
                       dict(mask=vb.make_paged_mask(1.0, prefix_len=z(3, dtype=I)))],
           "evict": [dict(mass=z(2, 1, 40)), dict(to=z(3, 2, dtype=I)), dict(to=z(2, dtype=I)), dict(kept=z(2, 20, dtype=I)), dict(kept=z(2, 2, 20)), dict(out=z(2, 2, 20).double()), dict(new_len=z(3, dtype=I))],
           "append_at": [dict(position=z(4, dtype=I)), dict(position=z(5))]}
    for name, f in good.items():
        with pytest.raises(vb.VlaError, match="not all on the current GPU"):
            f()
        for k in bad[name]:
            with pytest.raises(vb.VlaError) as e:
                f(**k)
            assert "not all on" not in str(e.value), (name, k)


def test_outputs_that_overlap_inputs():
    """Workgroups that read an input while another writes it."""
    far = dict(path=P + 0x2000, count=P + 0x3000)
    for k in (dict(far, count=P), dict(far, path=P + 16), dict(far, path=P - 8)):
        assert call("accept", **k) == E and b"overlaps" in vb.lib().vla_last_error(), k
    c, b = cache(), batch()
    at, L = C.byref, vb.lib()
    for lens in (b.kv_len, b.row_start + 4):
        assert L.vla_paged_accept(at(c), 1, 0, at(b), P + 0x4000, P + 0x5000, P + 0x6000, P + 0x2000, P + 0x3000, None, lens, None) == E
    assert L.vla_paged_evict(at(c), at(b), P, 64, 32, 1, 1, P + 0x4000, 2, P + 0x5000, P + 0x100000, 32, b.kv_len, None) == E and b"overlaps" in L.vla_last_error()
    assert call("evict", mo=P + 4) == E and call("evict", mo=P - 4) == E


def test_too_many_layers_or_positions():
    assert call("accept", c=cache(n_kv_heads=1024, head_dim=16), layers=1025) == S
    most = batch(max_len=1 << 30, table_stride=1 << 26)
    assert call("evict", c=cache(head_dim=256, dtype=vb.VLA_DTYPE_F32), b=most, ms=1 << 30, keep=1 << 30, ts=1 << 26, mos=1 << 30) == S


def test_binding_refuses_layers_beyond_the_pools():
    pools = [z(3, 8, 2, 16, 64) for _ in range(2)]
    b = vb.make_paged_batch(z(3, dtype=I), z(2, dtype=I), z(2, 3, dtype=I), 5, 3, 40)
    row, each = z(5, dtype=I), pools[0][0].numel()
    call = lambda first, n, stride: vb.vla_paged_accept(vb.make_paged_cache(pools[0][first], pools[1][first]), n, stride, b, row, row, row, z(2, 3, dtype=I), z(2, dtype=I))
    for first, n, stride in ((0, 4, each), (1, 3, each), (0, 3, 2 * each)):
        with pytest.raises(vb.VlaError, match="beyond the pools"):
            call(first, n, stride)
    for first, n, stride in ((0, 3, each), (1, 2, each), (0, 2, 2 * each), (2, 1, 0)):
        with pytest.raises(vb.VlaError, match="not all on the current GPU"):
            call(first, n, stride)
