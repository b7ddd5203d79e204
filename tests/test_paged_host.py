"""Refusals of the paged cache's entry points and of the sampler, and their size queries: host code, no device."""
import ctypes as C

import pytest

from paper_2510_06710_amd import binding as vb

P = 0x1000


def cache(**k):
    c = vb.vla_paged_cache(P, P, vb.VLA_DTYPE_BF16, 8, 16, 2, 64)
    for name, v in k.items():
        setattr(c, name, v)
    return c


def batch(**k):
    b = vb.vla_paged_batch(2, 5, 3, 40, 3, P, P, P)
    for name, v in k.items():
        setattr(b, name, v)
    return b


BAD_BOTH = [(dict(dtype=5), {}, vb.VLA_EDTYPE), (dict(k=None), {}, vb.VLA_EINVAL), (dict(v=0x1008), {}, vb.VLA_EINVAL), (dict(n_pages=0), {}, vb.VLA_EINVAL),
            (dict(page_size=24), {}, vb.VLA_ESHAPE), (dict(page_size=8), {}, vb.VLA_ESHAPE), (dict(page_size=2048), {}, vb.VLA_ESHAPE),
            (dict(head_dim=72), {}, vb.VLA_ESHAPE), (dict(head_dim=272), {}, vb.VLA_ESHAPE), (dict(n_kv_heads=0), {}, vb.VLA_EINVAL),
            ({}, dict(n_seq=0), vb.VLA_EINVAL), ({}, dict(n_rows=-1), vb.VLA_EINVAL), ({}, dict(max_len=-1), vb.VLA_EINVAL), ({}, dict(row_start=None), vb.VLA_EINVAL),
            ({}, dict(kv_len=None), vb.VLA_EINVAL), ({}, dict(page_table=None), vb.VLA_EINVAL), ({}, dict(max_len=49), vb.VLA_ESHAPE),
            ({}, dict(max_len=2 ** 30 + 1, table_stride=2 ** 27), vb.VLA_ESHAPE), ({}, dict(n_seq=70000), vb.VLA_ESHAPE)]


def append(c=None, b=None, rot=None, **k):
    a = dict(q=P, k=P, v=P, dt=vb.VLA_DTYPE_F32, heads=4, qs=256, ks=128, vs=128, qo=P + 0x100000, os=256)
    a.update(k)
    c, b, rot = c or cache(), b or batch(), rot if rot is not None else vb.vla_rotary(P, 64, 0, 1.0, 1e-6, None, None)
    return vb.lib().vla_paged_append(C.byref(c), C.byref(b), C.byref(rot), a["q"], a["k"], a["v"], a["dt"], a["heads"], a["qs"], a["ks"], a["vs"], a["qo"], a["os"], None)


def attend(c=None, b=None, m=None, **k):
    a = dict(q=P, heads=4, qs=256, out=P, os=256, ws=P, n=1 << 40)
    a.update(k)
    c, b, m = c or cache(), b or batch(), m or vb.vla_paged_mask(0.125, 0.0, None, None, 0, 0)
    return vb.lib().vla_paged_attention(C.byref(c), C.byref(b), C.byref(m), a["q"], a["heads"], a["qs"], a["out"], a["os"], None, a["ws"], a["n"], None)


@pytest.mark.parametrize("c,b,code", BAD_BOTH)
def test_cache_and_batch(c, b, code):
    assert append(cache(**c), batch(**b)) == code
    assert attend(cache(**c), batch(**b)) == code
    assert vb.vla_last_error()


def test_append_refuses():
    for k, code in [(dict(k=None), vb.VLA_EINVAL), (dict(v=None), vb.VLA_EINVAL), (dict(q=None), vb.VLA_EINVAL), (dict(qo=None), vb.VLA_EINVAL), (dict(dt=3), vb.VLA_EDTYPE),
                    (dict(heads=0), vb.VLA_ESHAPE), (dict(qs=255), vb.VLA_ESHAPE), (dict(ks=127), vb.VLA_ESHAPE), (dict(vs=0), vb.VLA_ESHAPE), (dict(os=200), vb.VLA_ESHAPE),
                    (dict(qo=P), vb.VLA_EINVAL)]:                        # in place with another type
        assert append(**k) == code, k
    r = lambda *a: vb.vla_rotary(*a)
    assert append(rot=r(P, 63, 0, 1.0, 1e-6, None, None)) == vb.VLA_ESHAPE
    assert append(rot=r(P, 66, 0, 1.0, 1e-6, None, None)) == vb.VLA_ESHAPE
    assert append(rot=r(None, 64, 0, 1.0, 1e-6, None, None)) == vb.VLA_EINVAL
    assert append(rot=r(P, 64, 0, 1.0, -1.0, P, None)) == vb.VLA_EINVAL
    assert append(b=batch(n_rows=0)) == vb.VLA_OK                        # nothing to do, nothing launched


def test_attention_refuses():
    m = lambda *a: vb.vla_paged_mask(*a)
    for k, code in [(dict(q=None), vb.VLA_EINVAL), (dict(out=None), vb.VLA_EINVAL), (dict(ws=None), vb.VLA_EINVAL), (dict(ws=0x1004), vb.VLA_EINVAL), (dict(n=16), vb.VLA_EWORKSPACE),
                    (dict(heads=3), vb.VLA_ESHAPE), (dict(heads=0), vb.VLA_ESHAPE), (dict(qs=255), vb.VLA_ESHAPE), (dict(os=255), vb.VLA_ESHAPE)]:
        assert attend(**k) == code, k
    for mask, code in [(m(0.0, 0.0, None, None, 0, 0), vb.VLA_EINVAL), (m(float("nan"), 0.0, None, None, 0, 0), vb.VLA_EINVAL), (m(float("inf"), 0.0, None, None, 0, 0), vb.VLA_EINVAL),
                       (m(1.0, -1.0, None, None, 0, 0), vb.VLA_EINVAL), (m(1.0, 0.0, None, None, -1, 0), vb.VLA_EINVAL), (m(1.0, 0.0, None, None, 0, -16), vb.VLA_EINVAL),
                       (m(1.0, 0.0, None, None, 0, 8), vb.VLA_ESHAPE), (m(1.0, 0.0, None, None, 0, 48), vb.VLA_ESHAPE), (m(1.0, 0.0, None, None, 5, 16), vb.VLA_EINVAL)]:
        assert attend(m=mask) == code
    assert attend(b=batch(n_rows=0)) == vb.VLA_OK
    q = lambda **k: vb.lib().vla_paged_attention_workspace_bytes(C.byref(cache(**k)), C.byref(batch()), C.byref(m(1.0, 0.0, None, None, 0, 0)), 4)
    assert q() > 0 and q(dtype=9) == 0


def test_sampler_refuses():
    L, f = vb.lib(), vb.VLA_DTYPE_F32
    s = lambda z=P, dt=f, stride=100, n=4, v=100, tok=P, ws=P, size=1 << 40: L.vla_sample_logits(z, dt, stride, n, v, None, None, None, None, None, tok, None, None, None, ws, size, None)
    assert s(z=None) == s(tok=None) == s(ws=None) == s(n=0) == s(v=0) == vb.VLA_EINVAL
    assert s(dt=2) == vb.VLA_EDTYPE and s(stride=99) == s(v=262145, stride=300000) == vb.VLA_ESHAPE and s(size=1) == vb.VLA_EWORKSPACE
    assert vb.lib().vla_sample_logits_workspace_bytes(4, 100) > 0 == vb.lib().vla_sample_logits_workspace_bytes(0, 100)
    with pytest.raises(vb.VlaError):
        vb.vla_sample_logits_workspace_bytes(1, 0)


def test_binding_refuses_arrays_that_would_be_read_wrongly():
    import torch
    z, i32 = torch.zeros, torch.int32
    k = z(8, 2, 16, 64)
    c = vb.make_paged_cache(k, k.clone())
    good = lambda: vb.make_paged_batch(z(3, dtype=i32), z(2, dtype=i32), z(2, 3, dtype=i32), 5, 3, 40)
    for bad in (lambda: vb.make_paged_cache(k, z(8, 2, 16, 32)), lambda: vb.make_paged_cache(k.double(), k.double()), lambda: vb.make_paged_cache(k.transpose(1, 2), k.transpose(1, 2)),
                lambda: vb.make_paged_batch(z(3), z(2, dtype=i32), z(2, 3, dtype=i32), 5, 3, 40), lambda: vb.make_paged_batch(z(2, dtype=i32), z(2, dtype=i32), z(2, 3, dtype=i32), 5, 3, 40),
                lambda: vb.make_paged_batch(z(3, dtype=i32), z(2, dtype=i32), z(3, 3, dtype=i32), 5, 3, 40), lambda: vb.make_rotary(z(32)),
                lambda: vb.vla_paged_append(c, good(), vb.make_rotary(), z(5, 4, 64), z(5, 2, 64), z(5, 1, 64), z(5, 4, 64)),
                lambda: vb.vla_paged_append(c, good(), vb.make_rotary(), z(5, 4, 64), z(4, 2, 64), z(4, 2, 64), z(5, 4, 64)),
                lambda: vb.vla_paged_append(c, good(), vb.make_rotary(), z(5, 64, 4).transpose(1, 2), z(5, 2, 64), z(5, 2, 64), z(5, 4, 64)),
                lambda: vb.vla_paged_append(c, good(), vb.make_rotary(q_gain=z(63)), z(5, 4, 64), z(5, 2, 64), z(5, 2, 64), z(5, 4, 64)),
                lambda: vb.vla_paged_attention(c, good(), vb.make_paged_mask(1.0), z(5, 4, 64).bfloat16(), z(5, 4, 64)),
                lambda: vb.vla_paged_attention(c, good(), vb.make_paged_mask(1.0, slopes=z(3)), z(5, 4, 64), z(5, 4, 64)),
                lambda: vb.vla_sample_logits(z(4, 9).T, z(9, dtype=i32)), lambda: vb.vla_sample_logits(z(4, 9), z(4)), lambda: vb.vla_sample_logits(z(4, 9), z(4, dtype=i32), top_k=z(4))):
        with pytest.raises(vb.VlaError):
            bad()


def test_forward_paged_refuses():
    import vla_inputs as vi
    from test_abi_host import fake_model
    cfg = vb.make_config(vi.TINY, 8, 80)
    h, keep = fake_model(cfg)
    L = vb.lib()
    good = dict(dtype=vb.VLA_DTYPE_F32, n_kv_heads=4, head_dim=64)

    def f(c=good, b={}, model=h, stride=1 << 20, ids=P, patch=P, n_patch=4, shared=0, ws=P, size=1 << 40, hl=P, value=None):
        cc, bb = cache(**c), batch(**b)
        return L.vla_forward_paged(model, C.byref(cc), stride, C.byref(bb), ids, patch, n_patch, None, shared, ws, size, hl, None, value, None)

    assert f(model=None) == f(ids=None) == f(ws=None) == f(hl=None) == f(patch=None) == f(n_patch=-1) == f(value=P) == vb.VLA_EINVAL
    assert f(ws=P + 4) == f(stride=(1 << 20) + 1) == f(b=dict(n_rows=0)) == f(b=dict(max_rows=0)) == vb.VLA_EINVAL
    assert f(c=dict(good, dtype=vb.VLA_DTYPE_BF16)) == f(c=dict(good, n_kv_heads=2)) == f(c=dict(good, head_dim=48)) == f(stride=100) == vb.VLA_ESHAPE
    assert f(c=dict(good, page_size=24)) == f(b=dict(n_rows=1 << 30)) == vb.VLA_ESHAPE and f(size=1000) == vb.VLA_EWORKSPACE
    q = lambda **k: L.vla_forward_paged_workspace_bytes(C.byref(cfg), C.byref(cache(**dict(good, **k))), C.byref(batch()), 0)
    assert q() > 5 * 256 * 4 and q(head_dim=48) == 0
    vb.vla_destroy(h)


def test_binding_refuses_arrays_of_the_host():
    import torch
    z, i32 = torch.zeros, torch.int32
    c, b = vb.make_paged_cache(z(8, 2, 16, 64), z(8, 2, 16, 64)), vb.make_paged_batch(z(3, dtype=i32), z(2, dtype=i32), z(2, 3, dtype=i32), 5, 3, 40)
    for call in (lambda: vb.vla_paged_append(c, b, vb.make_rotary(), z(5, 4, 64), z(5, 2, 64), z(5, 2, 64), z(5, 4, 64)),
                 lambda: vb.vla_paged_attention(c, b, vb.make_paged_mask(1.0), z(5, 4, 64), z(5, 4, 64), ws=z(1 << 20)),
                 lambda: vb.vla_forward_paged(None, c, 0, b, z(5, dtype=i32), z(1 << 20), z(2, 128)),
                 lambda: vb.vla_sample_logits(z(4, 9), z(4, dtype=i32), ws=z(64))):
        with pytest.raises(vb.VlaError, match="not all on the current GPU"):
            call()
    for k in (dict(h_last=z(2, 64)), dict(patch=z(4, 64)), dict(patch=z(4, 128).bfloat16()), dict(value=z(3)), dict(logits=z(2, 255)), dict(prefix_len=z(2))):
        with pytest.raises(vb.VlaError, match="wanted|patch"):
            vb.vla_forward_paged(None, c, 0, b, z(5, dtype=i32), z(1 << 20), **{"h_last": z(2, 128), **k})
