"""Windows near 2^31: those of rows that see everything before them.  Tolerances: those of test_gpu_paged_evict.py and test_gpu_paged_attention.py."""
import pytest

import test_gpu_paged_attention as attention
import test_gpu_paged_evict as evict
from paged_ref import Batch

pytestmark = pytest.mark.gpu
BOTH = pytest.mark.parametrize("dtype", ["bf16", "f32"])
WIDE = pytest.mark.parametrize("window", [2 ** 31 - 1, 2 ** 31 - 200, 2 ** 30])
BEFORE = [(5, 2), (1, 40), (3, 3), (6, 4)]                    # some rows lie at negative positions
MANY = [(40, 3), (33, 40), (70, 60), (100, 90)]


@BOTH
@WIDE
@pytest.mark.parametrize("spec", [evict.DECODE, evict.PROMPT, BEFORE, MANY])
def test_weights(dtype, window, spec):
    evict.weigh(Batch(spec, 16, padding=2), dtype, 4, 2, 64, window=window)
    evict.weigh(Batch(spec, 32), dtype, 4, 2, 64, window=window, prefix=[min(l, 7 * i) for i, (_, l) in enumerate(spec)], bias=True)
    evict.weigh(Batch(spec, 32), dtype, 8, 1, 128, window=window, cap=20.0)


@BOTH
def test_weights_of_long_prompts(dtype):
    evict.weigh(Batch([(300, 700), (2, 40)], 64, max_len=4000), dtype, 8, 2, 64, window=2 ** 31 - 1)


@BOTH
@WIDE
@pytest.mark.parametrize("spec", [attention.DECODE, attention.PROMPT, BEFORE, MANY])
def test_attention(dtype, window, spec):
    attention.run(Batch(spec, 16, padding=2), dtype, 4, 2, 64, window=window)
    attention.run(Batch(spec, 32), dtype, 4, 2, 64, window=window, prefix=[min(l, 7 * i) for i, (_, l) in enumerate(spec)], bias=True)
