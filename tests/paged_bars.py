"""Bars on attention errors (offq_kv_attention_paged) in the mean square, from variances of roundings.

The worst case per element adds all roundings up; independent ones add in squares.  With
u = 2^-11 / sqrt(3) the rms of a rounding to fp16 and b = 2^-8 / sqrt(3) of one to bf16 (half a
step, at its largest), the error of channel d of a row's output o has in expectation at most
    b^2 o_d^2                                                              the output's
    u^2 sum_j p_j^2 v_jd^2                                                 weights
    u^2 sum_j p_j^2 sv_j^2 mean_d ((cv_jd - z')^2 + z'^2)                  scaled values, z' = zv in 0 .. 15
    u^2 sum_j p_j^2 (v_jd - o_d)^2 sm^2 sk_j^2 sum_e q_e^2 ((ck_je - zk_j)^2 + ck_je^2)   queries, scaled keys
    9 2^-48 / 3 |o|^2 / D                                                  fp32, log2 D + 2 butterflies and sums
where o and v are rotated back if the call does.  The mean over a call's channels of error^2 over
1.1^2 times the first and 1.5^2 times the others (their rms: a bf16 half-step is 0.73 of that on
average over a binade) may not pass 1, nor the mean over a row's 64 or 128 channels with 1.5^2 and
3^2 (its fp16 parts may come from one position).
"""
import numpy as np

from oracle import paged as OP

U2, B2 = 2.0 ** -22 / 3, 2.0 ** -16 / 3


def _six_bits(p):
    m, e = np.frexp(p)
    return np.ldexp(np.round(m * 64) / 64, e)


class Exact:
    """fp64 outputs `out` and the variances `bf16`, `fp16` [M, Hq, D]; `heads` (b, h) alone
    where given.  mistake: "page" leaves each sequence's first 16 positions out, "scores" makes
    scores 5 % larger, "weights" rounds weights to six bits, "zeros" gives zeros."""

    def __init__(self, q, starts, lens, table, kc, vc, par, sm, k_had=True, v_had=False, heads=None,
                 mistake=None):
        qr = OP.hadamard_rows(q, k_had)
        M, Hq, D = qr.shape
        G = Hq // par.shape[1]
        self.out, self.fp16 = np.zeros_like(qr), np.zeros_like(qr)
        self.some = np.zeros((M, Hq), bool)
        for b, length in enumerate(lens):
            rows = slice(starts[b], starts[b + 1])
            n = starts[b + 1] - starts[b]
            slots = OP.sequence_slots(table[b], length, par.shape[2], par.shape[0])
            at = np.flatnonzero(slots >= 0)
            todo = [h for h in range(Hq) if heads is None or (b, h) in heads]
            if not n or not todo:
                continue
            self.some[rows, todo] = True
            if not len(at):
                continue
            see = at <= length - n + np.arange(n)[:, None]
            if mistake == "page":
                see &= at >= 16
            pages = slots[at] // par.shape[2], slots[at] % par.shape[2]
            for k in sorted({h // G for h in todo}):
                one = lambda t: np.ascontiguousarray(t[pages[0], k, pages[1]])[:, None, None]  # noqa: E731
                p1 = one(par)
                where = np.arange(len(at))
                ck, sk, zk = (t[:, 0] for t in OP.rows(one(kc), p1, where))
                cv, sv, zv = (t[:, 0] for t in OP.rows(one(vc), p1, where, value=True))
                K, V = sk[:, None] * (ck - zk[:, None]), sv[:, None] * (cv - zv[:, None])
                z = np.clip(zv, 0, 15)[:, None]
                near = sv ** 2 * ((cv - z) ** 2 + z ** 2).mean(-1)
                far = (ck - zk[:, None]) ** 2 + ck ** 2
                V = OP.hadamard_rows(V, v_had)
                for h in todo:
                    if h // G != k:
                        continue
                    x = qr[rows, h]
                    s = np.where(see, sm * (1.05 if mistake == "scores" else 1) * (x @ K.T), -np.inf)
                    top = s.max(-1, keepdims=True)
                    p = np.where(see, np.exp(s - np.where(np.isfinite(top), top, 0)), 0)
                    total = np.maximum(p.sum(-1, keepdims=True), 1e-300)
                    o = (_six_bits(p) if mistake == "weights" else p) @ V / total
                    p2 = (p / total) ** 2
                    r = p2 * (sm ** 2 * sk ** 2 * ((x ** 2) @ far.T))
                    apart = r @ V ** 2 - 2 * o * (r @ V) + r.sum(-1, keepdims=True) * o ** 2
                    self.out[rows, h] = 0 if mistake == "zeros" else o
                    self.fp16[rows, h] = U2 * (p2 @ V ** 2 + (p2 @ near)[:, None] + np.maximum(apart, 0))
        self.bf16 = B2 * self.out ** 2
        self.fp16 += 3 * 2.0 ** -48 * (self.out ** 2).mean(-1, keepdims=True)

    def outside(self, got):
        """What of `got` is outside the bars: a text, or None."""
        def ratio(a, b):
            e2 = (got - self.out)[self.some] ** 2
            return (e2 / np.maximum(a * a * self.bf16 + b * b * self.fp16, 1e-300)[self.some]).mean(-1)

        self.call = ratio(1.1, 1.5).mean()
        rows = ratio(1.5, 3)
        if not self.call <= 1:
            return f"call: {self.call:.2f}"
        if not (rows <= 1).all():
            return f"{(~(rows <= 1)).sum()} of {rows.size} rows, {rows.max():.2f}"
        return None
