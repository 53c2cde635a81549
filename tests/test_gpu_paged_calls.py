"""GPU: calls of the paged cache that its documentation allows: rows that share a buffer, the
smallest write, and every form of the kernels that a size reaches."""
import math

import numpy as np
import pytest
import torch

import paper_2606_07116_amd as offq
from oracle import paged as OP
from tests import parity as P
from tests.test_gpu_paged import (_back, _bf16, _cache, _check_rows, _host_cache, _mixed_call,
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


# ------------------------------------------------------------------ the smallest write
@pytest.mark.parametrize("Hq,Hkv", [(4, 1), (5, 1), (32, 8), (40, 8), (3, 3)])
@pytest.mark.parametrize("D,rotary,pairs,norm,k_had,v_had", [
    (128, 128, False, True, True, False), (128, 64, True, False, True, True), (64, 64, False, False, True, False),
    (64, 32, False, True, False, True), (128, 0, False, False, False, False),
])
def test_one_token(Hq, Hkv, D, rotary, pairs, norm, k_had, v_had):
    """Its rows against the oracle (the bars of tests/test_gpu_paged.py), the rest of the cache as it
    was; without a slot, nothing is written."""
    rng = np.random.default_rng(Hq + D + rotary)
    x = _bf16(rng, 1, Hq + 2 * Hkv, D)
    pos, freq = np.array([70001], np.int32), OP.inv_freq(rotary, 500000.0).astype(np.float32) if rotary else None
    qw, kw = (_bf16(rng, D) if norm else None for _ in range(2))
    before = _host_cache(rng, 3, Hkv, 16, D)
    bf = lambda t: None if t is None else P.to_dev_bf16(t)  # noqa: E731

    def turned(t, w):
        t = OP.norm(t, w, 1e-6)
        return OP.rotate(t, pos, freq, pairs, 1.0) if rotary else t

    qr, kr, vr = turned(x[:, :Hq], qw), turned(x[:, Hq:Hq + Hkv], kw), np.float64(x[:, Hq + Hkv:])
    for slot in (0, 21, 47, -1, 48):
        cache = _cache(*before)
        q = offq.offq_rope_kv_paged(P.to_dev_bf16(x.reshape(1, -1)), Hq, _t(pos), _t(np.array([slot])), cache,
                                    None if freq is None else _t(freq), interleaved=pairs, q_weight=bf(qw),
                                    k_weight=bf(kw), k_hadamard=k_had, v_hadamard=v_had)
        torch.cuda.synchronize()
        big = np.abs(qr).max(-1, keepdims=True) + np.abs(OP.norm(x[:, :Hq], qw, 1e-6)).max(-1, keepdims=True)
        assert np.all(np.abs(P.host(q.float()) - qr) <= 2.0 ** -8 * np.abs(qr) + D * 2.0 ** -24 * big)
        after = _back(cache)
        held = 0 <= slot < 48
        if held:
            for value, codes, had, y0 in ((False, after[0], k_had, kr), (True, after[1], v_had, vr)):
                c, s, z = OP.rows(codes, after[2], [slot], value=value)
                mag = np.abs(y0)
                delta = (D + 16) * 2.0 ** -24 * (mag.sum(-1) / math.sqrt(D) if had else 2 * mag.max(-1))
                _check_rows(c, s, z, OP.hadamard_rows(y0, had), delta,
                            not had and (value or (not norm and not rotary)))
        for a, b in zip(after, before):
            same = (a == b).all(-1).transpose(0, 2, 1).reshape(48, Hkv).all(-1)
            assert not same[slot] if held and a.dtype == np.uint8 else same.sum() >= 48 - held
            assert np.delete(same, slot if held else []).all()


# ------------------------------------------------------------------ calls past the caches
@pytest.mark.parametrize("D,rotary,pairs", [(128, 128, False), (128, 64, False), (128, 128, True),
                                            (64, 64, False), (64, 32, True)])
def test_large_write_as_two_small_ones(D, rotary, pairs):
    """Queries above 32 MB bypass the caches; the same tokens in two calls do not."""
    torch.manual_seed(D + rotary)
    Hq, Hkv, P_ = 32, 2, 256
    M = (32 << 20) // (2 * Hq * D) + 77
    x = torch.randn((M, (Hq + 2 * Hkv) * D), device=DEV).bfloat16()
    pos, slots = torch.arange(M, dtype=torch.int32, device=DEV), torch.randperm(-(-M // P_) * P_, device=DEV)[:M]
    f = offq.offq_rope_inv_freq(rotary, device=DEV)
    w = torch.rand(D, device=DEV).bfloat16()
    caches = [offq.paged_cache(-(-M // P_), Hkv, P_, D, device=DEV) for _ in range(2)]

    def write(c, rows):
        return offq.offq_rope_kv_paged(x[rows], Hq, pos[rows], slots[rows], c, f, interleaved=pairs, q_weight=w)

    whole = write(caches[0], slice(0, M))
    parts = torch.cat([write(caches[1], slice(0, M // 2)), write(caches[1], slice(M // 2, M))])
    torch.cuda.synchronize()
    assert torch.equal(whole, parts) and whole.isfinite().all()
    assert all(torch.equal(caches[0][n], caches[1][n]) for n in caches[0])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("k_had,v_had", [(True, False), (False, True)])
def test_large_read_as_two_small_ones(D, k_had, v_had):
    rng = np.random.default_rng(D)
    Hkv, P_ = 8, 64
    M = (32 << 20) // (4 * Hkv * D) + 55
    cache = _cache(*_host_cache(rng, -(-M // P_), Hkv, P_, D))
    slots = _t(rng.permutation(-(-M // P_) * P_)[:M])
    whole = offq.offq_kv_dequantize_paged(cache, slots, k_had, v_had)
    parts = [offq.offq_kv_dequantize_paged(cache, s, k_had, v_had) for s in (slots[:M // 2], slots[M // 2:])]
    torch.cuda.synchronize()
    for i in (0, 1):
        assert torch.equal(whole[i], torch.cat([p[i] for p in parts])) and whole[i].any(-1).all()
