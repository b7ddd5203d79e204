"""Pages whose elements lie beyond 2^32 bytes and 2^31 elements of a cache: the same bits as from the same rows in its first pages."""
import pytest
import torch

from paged_ref import DEV, TYPES
from paper_2510_06710_amd import binding as vb

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,n_pages", [("bf16", 36000), ("f32", 18000)])
@pytest.mark.parametrize("rows,shared", [(1, 0), (60, 0), (1, 128), (40, 128)])
def test_far_pages(dtype, n_pages, rows, shared):
    kind, heads, kv, d, page, per = TYPES[dtype], 16, 8, 128, 64, 8
    pools = [torch.zeros(n_pages, kv, page, d, dtype=kind, device=DEV) for _ in range(2)]
    assert pools[0].numel() * pools[0].element_size() > 2 ** 32 and (dtype == "f32" or pools[0].numel() > 2 ** 31)
    g = torch.Generator().manual_seed(0)
    n, lens = 3, [500, 333, 412]
    fill = [torch.randn(n * per, kv, page, d, generator=g).to(kind).to(DEV) for _ in range(2)]
    qkv = torch.randn(n * rows, heads + 2 * kv, d, generator=g).to(DEV)
    freq = (10000.0 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))).to(DEV)
    results = []
    for first in (0, n_pages - n * per):
        table = first + torch.arange(n * per, dtype=torch.int32).view(n, per)
        table[:, :shared // page] = table[0, :shared // page]
        for p, f in zip(pools, fill):
            p[first:first + n * per] = f
        cache = vb.make_paged_cache(*pools)
        batch = vb.make_paged_batch(torch.arange(0, n * rows + 1, rows, dtype=torch.int32, device=DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), table.to(DEV),
                                    n * rows, rows, max(lens))
        mask = vb.make_paged_mask(d ** -0.5, shared_len=shared)
        q, out = torch.zeros(n * rows, heads, d, dtype=kind, device=DEV), torch.zeros(n * rows, heads, d, dtype=kind, device=DEV)
        ws = torch.empty(vb.vla_paged_attention_workspace_bytes(cache, batch, mask, heads), dtype=torch.uint8, device=DEV)
        vb.vla_paged_append(cache, batch, vb.make_rotary(freq), qkv[:, :heads], qkv[:, heads:heads + kv], qkv[:, heads + kv:], q)
        vb.vla_paged_attention(cache, batch, mask, q, out, None, ws)
        torch.cuda.synchronize()
        results.append((q, out, *[p[first:first + n * per].clone() for p in pools]))
        for p in pools:                                      # (nothing of the near pages may serve the far ones)
            p[first:first + n * per] = float("nan")
    assert all(torch.equal(a, b) for a, b in zip(*results)) and torch.isfinite(results[1][1]).all() and results[1][1].abs().max() > 0
