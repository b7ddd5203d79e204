"""The forms of single-token attention that test_gpu_paged_attention.py does not reach, against the same reference with the same tolerance: shares of the key
tiles of more than 64 sequences, and a wave per sequence and key head that writes the output itself."""
import numpy as np
import pytest

from paged_ref import Batch
from test_gpu_paged_attention import BOTH, run

pytestmark = pytest.mark.gpu


def ragged(n, longest, seed, empty=7):
    """Sequences of up to `longest` positions, most of them short, one row each but for every `empty`th without."""
    r = np.random.default_rng(seed)
    spec = [(0 if s % empty == empty - 1 else 1, int(l)) for s, l in enumerate(r.integers(1, 60, n))]
    for s in r.choice(n, 5, replace=False):
        spec[s] = (1, int(r.integers(longest // 2, longest)))
    spec[int(r.integers(n))] = (1, longest)
    return spec


@BOTH
@pytest.mark.parametrize("n", [64, 65, 130, 2048])
def test_divided_among_many_sequences(dtype, n):
    run(Batch(ragged(n, 700, n), 16, padding=2), dtype, 2, 1, 32)
    run(Batch(ragged(n, 1300, n + 1), 64), dtype, 3, 1, 64, cap=5.0, bias=True)
    if n < 2000:
        run(Batch(ragged(n, 900, n + 2), 32), dtype, 4, 2, 128, window=170, layout="unaligned")
        spec = ragged(n, 900, n + 3)
        run(Batch(spec, 16), dtype, 4, 2, 64, prefix=[min(l, 5 * s % 97) for s, (_, l) in enumerate(spec)], window=33)


SHORT = [(1, 1), (1, 2), (0, 9), (1, 31), (1, 32), (1, 33), (1, 64), (1, 65), (1, 127), (1, 128)]


@BOTH
@pytest.mark.parametrize("heads,kv,d", [(4, 4, 64), (8, 1, 128), (7, 1, 128), (6, 2, 80), (16, 8, 256), (32, 1, 64)])
def test_undivided(dtype, heads, kv, d):
    run(Batch(SHORT, 16, padding=2), dtype, heads, kv, d)
    run(Batch(SHORT, 64), dtype, heads, kv, d, cap=3.0, bias=True, layout="unaligned")
    run(Batch(SHORT, 32), dtype, heads, kv, d, window=20)
    run(Batch(SHORT, 16), dtype, heads, kv, d, window=9, prefix=[min(l, 7 * i) for i, (_, l) in enumerate(SHORT)])
    run(Batch([(min(2, l), l) for _, l in SHORT], 16), dtype, heads // 2 if heads == 32 else heads, kv, d, prefix=[l // 2 for _, l in SHORT])


@BOTH
def test_undivided_where_the_pairs_fill_the_chip(dtype):
    run(Batch([(1, 294)] * 256, 16), dtype, 8, 8, 128)
    run(Batch(ragged(150, 500, 4), 16, padding=1), dtype, 16, 16, 64, bias=True)
    run(Batch(ragged(260, 1000, 5), 32), dtype, 32, 32, 16)
