"""CPU: the bars of tests/paged_bars.py let no such mistake pass on the shapes that the GPU tests
use (planted in the oracle), and the exact values rounded to bf16 pass."""
import math

import numpy as np
import pytest

from oracle import paged as OP
from paper_2606_07116_amd import inputs
from tests.paged_bars import Exact

# new tokens, positions before them, query heads, key/value heads, channels, rotated values
SHAPES = [
    ([1], [1500], 4, 1, 128, False), ([1], [1023], 4, 1, 128, True), ([1, 1, 1], [40, 37, 250], 8, 2, 64, False),
    ([1, 2], [9000, 31], 4, 1, 128, False), ([40], [1500], 4, 1, 128, False), ([40], [9000], 4, 1, 128, False),
    ([5], [100], 16, 2, 128, False), ([5, 5], [3000, 20], 16, 2, 128, True), ([5], [3000], 16, 2, 64, False),
    ([8, 8], [2500, 400], 16, 2, 64, True), ([7, 8], [60, 90], 8, 1, 64, False), ([6], [700], 32, 4, 128, False),
    ([90], [60], 4, 2, 128, True), ([300], [30], 4, 2, 128, False), ([200, 1, 0, 3], [300, 40, 9, 77], 8, 2, 64, True),
    ([70], [3000], 4, 2, 128, False), ([70], [3000], 4, 2, 64, True), ([65, 129], [0, 31], 8, 2, 128, False),
]


def operands(new, past, Hq, Hkv, D, seed, P=16):
    """(q, starts, lens, table, k codes, v codes, params) of random rows on scattered pages."""
    rng = np.random.default_rng(seed)
    lens = [n + p for n, p in zip(new, past)]
    need = [-(-n // P) for n in lens]
    perm = rng.permutation(sum(need) + 2).astype(np.int32)
    table = np.full((len(new), max(need) + 1), -1, np.int32)
    for b, n in enumerate(need):
        table[b, :n] = perm[sum(need[:b]):sum(need[:b]) + n]
    shape = (len(perm), Hkv, P)
    kc, vc = (rng.integers(0, 256, shape + (D // 2,), dtype=np.uint8) for _ in range(2))
    par = np.empty(shape + (4,), np.int16)
    par[..., ::2] = rng.uniform(0.05, 0.6, shape + (2,)).astype(np.float16).view(np.int16)
    par[..., 1::2] = rng.integers(3, 13, shape + (2,))
    q = inputs.round_to_bf16(rng.standard_normal((sum(new), Hq, D)).astype(np.float32))
    return q, np.concatenate([[0], np.cumsum(new)]).astype(np.int32), lens, table, kc, vc, par


@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_mistakes_do_not_pass(i):
    new, past, Hq, Hkv, D, v_had = SHAPES[i]
    args = (*operands(new, past, Hq, Hkv, D, i), 1 / math.sqrt(D), True, v_had)
    exact = Exact(*args)
    ref, _, _, _ = OP.attention(*args)
    assert np.abs(exact.out - ref).max() <= 1e-12 * np.abs(ref).max()
    assert exact.outside(inputs.round_to_bf16(exact.out.astype(np.float32)).astype(np.float64)) is None
    for mistake in ("zeros", "page", "scores", "weights"):
        assert exact.outside(Exact(*args, mistake=mistake).out) is not None, mistake
