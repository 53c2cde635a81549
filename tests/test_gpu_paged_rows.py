"""GPU: rows of the paged attention (offq_kv_attention_paged) in the company that they keep, and
scores wherever they lie, against fp64 softmax over the values that the cache stands for.

A softmax does not change when a row's scores all move by the same amount, and a row's result does
not depend on positions that it does not see or on the rows beside it.
"""
import math

import numpy as np
import pytest
import torch

import paper_2606_07116_amd as offq
from oracle import paged as OP
from tests import parity as P
from tests.test_gpu_paged import _bf16, _cache, _host_cache, _t, _tables

pytestmark = pytest.mark.gpu

DEV = P.DEV


class Call:
    """Sequences of new[b] rows after past[b] positions over a cache of random rows; `cache` and
    `queries` change them before the call."""

    def __init__(self, new, past, Hq=4, Hkv=2, D=128, P_=16, seed=0, cache=None, queries=None):
        rng = np.random.default_rng(seed)
        self.new, self.lens = new, [n + p for n, p in zip(new, past)]
        self.table, pages = _tables(rng, self.lens, P_)
        self.host = _host_cache(rng, pages, Hkv, P_, D)
        self.starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        self.q = _bf16(rng, sum(new), Hq, D)
        if cache:
            cache(self)
        if queries:
            queries(self.q)

    def slot(self, b, j):
        P_ = self.host[2].shape[2]
        return self.table[b, j // P_], j % P_

    def run(self, sm, k_had=True, v_had=False):
        out = offq.offq_kv_attention_paged(
            P.to_dev_bf16(self.q), _t(self.starts), _t(np.array(self.lens, np.int32)), _t(self.table),
            _cache(*self.host), max(self.new), sm_scale=sm, k_hadamard=k_had, v_hadamard=v_had)
        torch.cuda.synchronize()
        return P.host(out.float()).astype(np.float64)

    def exact(self, sm, k_had=True, v_had=False):
        """fp64, all rows of a sequence at once."""
        kc, vc, par = self.host
        qr = OP.hadamard_rows(self.q, k_had)
        out = np.zeros_like(qr)
        G = qr.shape[1] // par.shape[1]
        for b, n in enumerate(self.new):
            slots = OP.sequence_slots(self.table[b], self.lens[b], par.shape[2], par.shape[0])
            at = np.flatnonzero(slots >= 0)
            if not n or not len(at):
                continue
            K = OP.dequantize(kc, par, slots[at])
            V = OP.dequantize(vc, par, slots[at], value=True)
            see = at <= self.lens[b] - n + np.arange(n)[:, None]
            rows = slice(self.starts[b], self.starts[b + 1])
            for h in range(qr.shape[1]):
                s = np.where(see, sm * (qr[rows, h] @ K[:, h // G].T), -np.inf)
                top = s.max(-1, keepdims=True)
                p = np.where(see, np.exp(s - np.where(np.isfinite(top), top, 0)), 0)
                out[rows, h] = (p / np.maximum(p.sum(-1, keepdims=True), 1e-300)) @ \
                    np.where(see.any(0)[:, None], V[:, h // G], 0)
        return OP.hadamard_rows(out, v_had)


def _error(got, ref):
    """The error's norm over the output's."""
    return math.sqrt(((got - ref) ** 2).sum() / (ref ** 2).sum())


# ------------------------------------------------------------------ scores anywhere
# log2 of what every weight loses; sm_scale sk sqrt(D) q_0 log2(e) is 1/4 per step of the zero-point
DROPS = [0, 8, 12, 16, 18, 20, 22, 23, 24, 25, 26, 40]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new,past,absent", [
    ([300], [0], 0), ([150, 1, 64], [0, 90, 40], 0), ([70], [3000], 0), ([3, 40], [900, 1500], 0),
    ([90], [700], 9), ([5], [400], 2), ([1, 4], [1300, 20], 0),
])
def test_scores_below_zero(new, past, absent, D):
    """Keys moved along the first channel of the unrotated queries, which all rows share: every
    score of a row drops by the same amount and the outputs stay.  (The same errors to a half: the
    roundings of the scores' terms grow with the offset, 2^-11 of up to 40 / ln 2, those of the
    queries and codes that differ from row to row do not.)"""
    sm = 0.25 / (math.log2(math.e) * 0.125 * math.sqrt(D) * 2)

    def offset(by):
        def change(call):
            par = call.host[2]
            par[..., 0] = np.float16(0.125).view(np.int16)
            par[..., 1] = 7 + by
            call.table[:, :absent] = -1
        return change

    def first(q):
        q[..., 0] = 2.0

    errors = {}
    for drop in DROPS:
        call = Call(new, past, D=D, seed=sum(new) + D, cache=offset(4 * drop), queries=first)
        errors[drop] = _error(call.run(sm), call.exact(sm))
    print(" ".join(f"{d}: {e:.5f}" for d, e in errors.items()))
    # bf16 outputs alone leave between 2^-8 / 4 and 2^-8 / sqrt(3)
    assert errors[0] <= 2.0 ** -8
    assert max(errors.values()) <= 1.5 * errors[0], errors


# ------------------------------------------------------------------ values around an offset
@pytest.mark.parametrize("offset", [40, -300, 3000, -30000])
@pytest.mark.parametrize("new,past", [([300], [0]), ([70, 2], [1500, 300]), ([5], [300])])
@pytest.mark.parametrize("D", [64, 128])
def test_values_around_an_offset(offset, new, past, D):
    """Rotated values whose zero-points are far from their codes: the offset is channel 0's alone
    once the sum is rotated back, and the other channels keep their bits.  What they may lose: half
    a bf16 step and the weights' and codes' fp16 roundings (1.5 x 2^-8 of their norm in all), and
    the fp32 roundings of the offset, of the butterflies' L stages and the two steps before them:
    sqrt(L + 2) 2^-24 / sqrt(3) of channel 0 as a norm, twice that allowed and rounded up, 2^-22."""
    def shift(call):
        rng = np.random.default_rng(1)
        zero = call.host[2][..., 3]
        zero[...] = 7 + offset + rng.integers(-3, 4, zero.shape)

    call = Call(new, past, D=D, seed=abs(offset) + D, cache=shift)
    got, ref = (f(1 / math.sqrt(D), v_had=True) for f in (call.run, call.exact))
    off = np.linalg.norm((got - ref)[..., 1:])
    print(off / np.linalg.norm(ref[..., 1:]))
    assert off <= 1.5 * 2.0 ** -8 * np.linalg.norm(ref[..., 1:]) + 2.0 ** -22 * np.linalg.norm(ref[..., 0])
    assert np.linalg.norm((got - ref)[..., 0]) <= 2.0 ** -8 * np.linalg.norm(ref[..., 0])


# ------------------------------------------------------------------ rows not seen
def _last_position(key=None, value=None):
    """Parameters of each sequence's last position: (scale, zero-point) of its key, of its value."""
    def spoil(call):
        for b, n in enumerate(call.lens):
            page, at = call.slot(b, n - 1)
            for j, what in ((0, key), (2, value)):
                if what:
                    call.host[2][page, :, at, j] = np.float16(what[0]).view(np.int16)
                    call.host[2][page, :, at, j + 1] = what[1]
    return spoil


def _earlier_rows(new, past, spoil, D, one_sign=False, k_had=True):
    """The error of the rows that do not see their sequence's last position, with it spoilt, and the
    rows that do."""
    def positive(q):
        q[...] = np.abs(q)

    call = Call(new, past, D=D, seed=sum(new) + D, queries=positive if one_sign else None)
    ref = call.exact(1 / math.sqrt(D), k_had)
    spoil(call)
    got = call.run(1 / math.sqrt(D), k_had)
    early = np.ones(len(ref), bool)
    early[call.starts[1:] - 1] = False
    e = _error(got[early], ref[early])
    print(e)
    return e, got[~early]


@pytest.mark.parametrize("scale,zero", [(65504, 0), (65504, 15), (65504, 32767), (65504, -32768),
                                        (300, 5), (300, 32767)])
@pytest.mark.parametrize("one_sign", [False, True])
@pytest.mark.parametrize("new,past", [([100], [0]), ([70, 3], [1500, 300]), ([4], [300])])
@pytest.mark.parametrize("D", [64, 128])
def test_huge_rows_behind(scale, zero, one_sign, new, past, D):
    """A last token whose key and value have the largest scale that the quantizer writes (what an
    overflow before it leaves) and the rows before it, which do not see it.  Their scaled codes may
    become fp16 subnormals, 2^-8 of a step each: 2^-8 / sqrt(3) sm sk |q|, 0.001, in a score; with
    half a bf16 step and the other roundings 2^-8 of the outputs' norm holds."""
    assert _earlier_rows(new, past, _last_position((scale, zero), (scale, zero)), D, one_sign,
                         k_had=not one_sign)[0] <= 2.0 ** -8


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("side", ["key", "value", "both"])
@pytest.mark.parametrize("new,past", [([100], [0]), ([300], [30]), ([70, 3], [1500, 300]), ([4], [300])])
@pytest.mark.parametrize("D", [64, 128])
def test_rows_that_are_no_numbers_behind(value, side, new, past, D):
    """Parameters that are no numbers at the last position (a page that was never written) touch
    the one row that sees it and no other; that row is not a number."""
    p = (value, 7)
    spoil = _last_position(p if side != "value" else None, p if side != "key" else None)
    error, last = _earlier_rows(new, past, spoil, D)
    assert error <= 2.0 ** -8 and np.isnan(last).all()


@pytest.mark.parametrize("value", [3e4, 1e10, 1e30, 3e38])
@pytest.mark.parametrize("first", ["absent", "zero", "tiny", "as the others"])
@pytest.mark.parametrize("new,past", [([90], [200]), ([70, 3], [1500, 300]), ([5], [300])])
def test_huge_queries_beside(value, first, new, past):
    """One element of one query is huge and the first positions (64 and more) have no pages, no
    scale, or scales of 2^-24: the other rows stay as exact as they are (2^-8 of the outputs' norm)
    when later keys bring the scores of their size."""
    def start(call):
        for b in range(len(new)):
            for i in range(5):
                if first == "absent":
                    call.table[b, i] = -1
                elif first != "as the others":
                    call.host[2][call.table[b, i], ..., ::2] = first == "tiny"

    call = Call(new, past, seed=sum(new), cache=start)
    ref = call.exact(1 / math.sqrt(128))
    call.q[4, 1, 7] = value
    got = call.run(1 / math.sqrt(128))
    others = np.ones(ref.shape[:2], bool)
    others[4, 1] = False
    e = _error(got[others], ref[others])
    print(e)
    assert e <= 2.0 ** -8
