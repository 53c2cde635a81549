"""GPU: attention of the paged cache within the mean-square bars of tests/paged_bars.py (that these
let no dropped page, no 5 % of a score and no weights of six bits pass is checked on the CPU), on
those shapes and in every form of the kernels that sizes and lengths reach."""
import math

import numpy as np
import pytest
import torch

import paper_2606_07116_amd as offq
from tests import parity as P
from tests.paged_bars import Exact
from tests.test_gpu_paged import _cache, _t
from tests.test_paged_bars import SHAPES, operands

pytestmark = pytest.mark.gpu


def _run(args, max_new, sm, k_had=True, v_had=False):
    q, starts, lens, table, *cache = args
    out = offq.offq_kv_attention_paged(
        P.to_dev_bf16(q), _t(starts), _t(np.array(lens, np.int32)), _t(table), _cache(*cache), max_new,
        sm_scale=sm, k_hadamard=k_had, v_hadamard=v_had)
    torch.cuda.synchronize()
    return P.host(out.float()).astype(np.float64)


def _check(new, past, Hq, Hkv, D, v_had=False, seed=0, k_had=True, heads=None, P_=16):
    args = operands(new, past, Hq, Hkv, D, seed, P_)
    sm = 1 / math.sqrt(D)
    got = _run(args, max(new), sm, k_had, v_had)
    exact = Exact(*args, sm, k_had, v_had, heads=heads)
    wrong = exact.outside(got)
    print(f"{exact.call:.2f}")
    assert wrong is None, wrong


@pytest.mark.parametrize("i", range(len(SHAPES)))
def test_shapes(i):
    new, past, Hq, Hkv, D, v_had = SHAPES[i]
    _check(new, past, Hq, Hkv, D, v_had, seed=i)


# the few-row kernel with three row tiles at 128 channels, three and four at 64, as one chunk (up to
# 512 positions of the page table) and as joined ones
@pytest.mark.parametrize("rows,D", [(33, 128), (40, 128), (48, 128), (40, 64), (48, 64), (49, 64), (64, 64)])
@pytest.mark.parametrize("past", [0, 77, 400, 1500])
@pytest.mark.parametrize("k_had,v_had", [(True, False), (False, True)])
def test_row_tiles(rows, D, past, k_had, v_had):
    G = next(g for g in (8, 7, 11, 3) if rows % g == 0)
    new = rows // G
    _check([new, 1, new - 1], [past, past // 2, 5], 2 * G, 2, D, v_had, seed=rows + past, k_had=k_had)


def test_more_than_64_sequences_of_three_row_tiles():
    rng = np.random.default_rng(3)
    new, past = rng.integers(0, 6, 70).tolist(), rng.integers(0, 300, 70).tolist()
    new[9], past[9] = 5, 1700
    for D in (64, 128):
        _check(new, past, 8, 1, D, seed=D)


def test_one_long_sequence_among_short_ones():
    """Chunks in several rounds: the long sequence's would else take 15 times the others'."""
    new = [1] * 61
    past = [9] * 61
    past[17] = 30000
    for D in (64, 128):
        _check(new, past, 8, 8, D, seed=D + 1, heads={(17, h) for h in (0, 3, 7)} | {(b, 5) for b in range(61)})


def test_chunks_of_more_than_4096_positions():
    """Each wave of a workgroup past the 1024 positions whose pages it knows at first."""
    _check([1, 2, 1], [25000, 24500, 23000], 32, 32, 128, seed=5, heads={(0, 0), (0, 31), (1, 7), (2, 16)})
    _check([1, 1], [40000, 39000], 48, 48, 64, seed=6, heads={(0, 0), (0, 47), (1, 20)})
