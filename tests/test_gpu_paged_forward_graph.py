"""vla_forward_paged in a captured graph: replayed with other ids, lengths and tables it gives what eager calls give."""
import pytest
import torch

from paper_2510_06710_amd import binding as vb
from test_gpu_paged_rollout import DEV, setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["f32", "bf16", "bf16_wide"])
@pytest.mark.parametrize("rows", [1, 37])
def test_replays(name, rows):
    run, obs, _, _ = setup(name, [(8, 3)])
    s, n, page, entries = run.shape, 3, 16, 12
    pools = [torch.zeros(s.n_layers, n * entries, s.n_heads, page, s.head_dim, dtype=s.torch_dtype, device=DEV) for _ in range(2)]
    cache = vb.make_paged_cache(pools[0][0], pools[1][0])
    start = torch.arange(0, n * rows + 1, rows, dtype=torch.int32, device=DEV)
    lens, table, ids = torch.ones(n, dtype=torch.int32, device=DEV), torch.zeros(n, entries, dtype=torch.int32, device=DEV), torch.zeros(n * rows, dtype=torch.int32, device=DEV)
    batch = vb.make_paged_batch(start, lens, table, n * rows, rows, entries * page)
    ws = torch.empty(vb.vla_forward_paged_workspace_bytes(run.cfg, cache, batch), dtype=torch.uint8, device=DEV)
    h, logits, value, patch = torch.zeros(n, s.hidden, device=DEV), torch.zeros(n, 256, device=DEV), torch.zeros(n, device=DEV), obs[0][0]

    def step():
        vb.vla_forward_paged(run.model.handle, cache, pools[0][0].numel(), batch, ids, ws, h, patch, None, 0, logits, value)

    def inputs(seed):
        g = torch.Generator().manual_seed(seed)
        lens.copy_(torch.randint(rows, entries * page + 1, (n,), generator=g))
        table.copy_(torch.randperm(n * entries, generator=g).view(n, entries))
        ids.copy_(torch.randint(-8, s.vocab, (n * rows,), generator=g))

    inputs(0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for seed in (1, 2, 3, 1):
        inputs(seed)
        fill = [torch.randn(p.shape, generator=torch.Generator().manual_seed(seed)).to(p.dtype).to(DEV) for p in pools]
        got = []
        for call in (graph.replay, step):
            for p, f in zip(pools, fill):
                p.copy_(f)
            ws.fill_(255)
            call()
            torch.cuda.synchronize()
            got.append([t.clone() for t in (h, logits, value, *pools)])
        assert all(torch.equal(a, b) for a, b in zip(*got)) and torch.isfinite(got[0][1]).all()
