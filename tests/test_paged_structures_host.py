"""Structures of the paged cache built by their own constructors, from addresses, go through the binding as those of make_* do."""
import pytest
import torch

from paper_2510_06710_amd import binding as vb

z = torch.zeros


def test_structures_from_addresses():
    k, v, i32 = z(8, 2, 16, 64), z(8, 2, 16, 64), torch.int32
    arrays = z(3, dtype=i32), z(2, dtype=i32), z(2, 3, dtype=i32)
    cache = vb.vla_paged_cache(k.data_ptr(), v.data_ptr(), vb.VLA_DTYPE_F32, 8, 16, 2, 64)
    batch = vb.vla_paged_batch(2, 5, 3, 40, 3, *[a.data_ptr() for a in arrays])
    for call in (lambda: vb.vla_paged_append(cache, batch, vb.vla_rotary(None, 0, 0, 1.0, 0.0, None, None), z(5, 4, 64), z(5, 2, 64), z(5, 2, 64), z(5, 4, 64)),
                 lambda: vb.vla_paged_attention(cache, batch, vb.vla_paged_mask(1.0, 0.0, None, None, 0, 0), z(5, 4, 64), z(5, 4, 64), ws=z(1 << 20)),
                 lambda: vb.vla_forward_paged(None, cache, 0, batch, z(5, dtype=i32), z(1 << 20), z(2, 128))):
        with pytest.raises(vb.VlaError, match="not all on the current GPU"):          # (these tensors are the host's)
            call()
