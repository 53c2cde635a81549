"""GPU: calls of the paged cache that its documentation allows: rows that share a buffer, the
smallest write, and every form of the kernels that a size reaches."""
import math

import numpy as np
import pytest
import torch

import paper_2606_07116_amd as offq
from oracle import paged as OP
from tests import parity as P
from tests.test_gpu_paged import (_attend, _back, _bf16, _cache, _check_rows, _host_cache, _mixed_call,
                                  _t)

pytestmark = pytest.mark.gpu

DEV = P.DEV


# ------------------------------------------------------------------ rows in one buffer
def test_attention_between_the_rows_of_its_queries():
    """Queries and outputs as two parts of one wider row."""
    torch.manual_seed(1)
    rng = np.random.default_rng(1)
    for new, past in (([1] * 3, [40, 0, 700]), ([90, 2], [100, 30])):
        q, *rest = _mixed_call(rng, len(new), new, past)
        M, Hq, D = q.shape
        both = torch.full((M, 2, Hq, D), 3.0, dtype=torch.bfloat16, device=DEV)
        for i in (0, 1):
            both[:, i] = q
            offq.offq_kv_attention_paged(both[:, i], *rest, max(new), out=both[:, 1 - i])
            want = offq.offq_kv_attention_paged(q, *rest, max(new))
            torch.cuda.synchronize()
            assert torch.equal(both[:, 1 - i], want) and torch.equal(both[:, i], q)
        with pytest.raises(offq.OffqError):  # a head in common
            wide = torch.zeros((M, 2 * Hq, D), dtype=torch.bfloat16, device=DEV)
            offq.offq_kv_attention_paged(wide[:, :Hq], *rest, max(new), out=wide[:, Hq - 1:2 * Hq - 1])


def test_write_between_the_rows_of_the_projection():
    torch.manual_seed(2)
    M, Hq, Hkv, D = 9, 4, 2, 64
    cols = (Hq + 2 * Hkv) * D
    wide = torch.randn((M, cols + Hq * D), device=DEV).bfloat16()
    pos = torch.arange(M, dtype=torch.int32, device=DEV)
    slots, f = torch.arange(M, device=DEV), offq.offq_rope_inv_freq(D, device=DEV)
    for x, out in ((wide[:, :cols], wide[:, cols:]), (wide[:, Hq * D:], wide[:, :Hq * D])):
        caches = [offq.paged_cache(2, Hkv, 16, D, device=DEV) for _ in range(2)]
        want = offq.offq_rope_kv_paged(x.clone(), Hq, pos, slots, caches[0], f)
        got = offq.offq_rope_kv_paged(x, Hq, pos, slots, caches[1], f, out=out.unflatten(1, (Hq, D)))
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        assert all(torch.equal(caches[0][n], caches[1][n]) for n in caches[0])
    with pytest.raises(offq.OffqError):
        offq.offq_rope_kv_paged(wide[:, :cols], Hq, pos, slots, caches[0], f,
                                out=wide[:, cols - 64:-64].unflatten(1, (Hq, D)))
