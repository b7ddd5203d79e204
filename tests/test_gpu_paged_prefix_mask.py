"""The prefix mask through the decoder: environments whose patches see each other, against the oracle's layers under that mask, prefixes of several lengths in a batch."""
import numpy as np
import pytest
import torch

from oracle import vla_oracle as vo
from oracle.from_inputs import to_f64
from paper_2510_06710_amd.harness import PagedRollout
from parity import TOL
from test_gpu_paged_rollout import setup

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["f32", "bf16", "bf16_wide"])
@pytest.mark.parametrize("page", [16, 64])
def test_logits_and_value(name, page):
    run, obs, cfg, w = setup(name, [(33, 5), (7, 2), (0, 4), (48, 16), (100, 1), (64, 33)])
    _, logits, value = PagedRollout(run, 64, page).prefill([p for p, _ in obs], [t for _, t in obs], see_patches=True)
    torch.cuda.synchronize()
    tol = TOL["f32" if name == "f32" else "bf16"]
    for i, (patch, ids) in enumerate(obs):
        x = vo.embed_prefix(w, to_f64(patch.cpu())[None], ids.cpu().numpy().astype(np.int64)[None])
        n = x.shape[1]
        row, key = np.arange(n)[:, None], np.arange(n)
        x, _ = vo.decoder_layers(cfg, w, x, np.arange(n), (key <= row) | (key < patch.shape[0]), None)
        h = vo.rmsnorm(x[:, n - 1], w.final_norm, cfg.rms_eps)
        assert np.abs(logits[i].double().cpu().numpy() - vo.bin_logits(cfg, w, h)[0]).max() <= tol["logits"], i
        assert abs(value[i].item() - np.ravel(vo.value_head(cfg, w, h))[0]) <= tol["value"], i
