"""The paged 4-bit key/value cache (oracle; test-only): the rows that a QKV projection's output
leaves in it, rows read back, and causal attention of packed new tokens over the pages.

The cache is codes [pages, Hkv, P, D/2] of keys and of values and params int16 [pages, Hkv, P, 4]
(key scale bits, key zero-point, value scale bits, value zero-point); slot = page * P + offset.
Everything here is fp64 on the dequantized values, row by row.
"""

import numpy as np

from . import hadamard, quantizer


def inv_freq(rotary, base, factor=1.0, low_turns=1.0, high_turns=4.0, original_len=0.0):
    """fp64 frequencies: plain, interpolated, or interpolated by the turns over original_len."""
    f = np.array([base ** (-2.0 * i / rotary) for i in range(rotary // 2)])
    if factor == 1.0:
        return f
    if not original_len:
        return f / factor
    turns = original_len * f / (2 * np.pi)
    keep = np.clip((turns - low_turns) / (high_turns - low_turns), 0, 1)
    return f * keep + (1 - keep) * f / factor


def norm(x, w, eps):
    """x / sqrt(mean x^2 + eps) * w over the last axis (x itself without w)."""
    x = np.asarray(x, dtype=np.float64)
    if w is None:
        return x
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(w, np.float64)


def rotate(x, positions, freq, interleaved, amplitude):
    """[M, H, D] rows: the first 2 len(freq) channels turned by positions[m] * freq[i]."""
    x = np.array(x, dtype=np.float64)
    r = 2 * len(freq)
    t = np.asarray(positions, np.float64)[:, None] * np.asarray(freq, np.float64)
    cos, sin = amplitude * np.cos(t)[:, None], amplitude * np.sin(t)[:, None]
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if interleaved else (x[..., :r // 2], x[..., r // 2:r])
    a, b = a * cos - b * sin, b * cos + a * sin
    if interleaved:
        x[..., 0:r:2], x[..., 1:r:2] = a, b
    else:
        x[..., :r // 2], x[..., r // 2:r] = a, b
    return x


def hadamard_rows(x, yes):
    return hadamard.rotate(x, x.shape[-1]) if yes else np.asarray(x, np.float64)


def rows(codes, params, slots, value=False):
    """(codes [M, Hkv, D], scale [M, Hkv], zero [M, Hkv]) of the rows at `slots`, as fp64."""
    P = params.shape[2]
    slots = np.asarray(slots, np.int64)
    page, at = slots // P, slots % P
    c = quantizer.unpack_nibbles(codes[page, :, at]).astype(np.float64)
    w = np.ascontiguousarray(params[page, :, at])
    j = 2 if value else 0
    return c, w.view(np.float16)[..., j].astype(np.float64), w[..., j + 1].astype(np.float64)


def dequantize(codes, params, slots, value=False, undo=False):
    c, s, z = rows(codes, params, slots, value)
    return hadamard_rows(s[..., None] * (c - z[..., None]), undo)


def sequence_slots(table, length, P, pages):
    """The slots of positions 0 .. length - 1, -1 for those that are not seen."""
    j = np.arange(max(0, min(length, len(table) * P)))
    page = np.asarray(table, np.int64)[j // P]
    return np.where((page >= 0) & (page < pages), page * P + j % P, -1)


def attention(q, q_starts, seq_lens, table, k_codes, v_codes, params, sm_scale, k_hadamard=True,
              v_hadamard=False, max_new=None):
    """(out, E, eta, written) for q [M, Hq, D]: the outputs (fp64), and per (row, head) the
    magnitudes that error bounds are stated in,
        E   = sum_j p_j sv_j (|zv_j| + max_d |cv_j[d] - zv_j|),
        eta = sm_scale (max_j sk_j sum_d |q_r[d]| (ck_j[d] + |ck_j[d] - zk_j|)
                        + 2^-4 max_j sk_j sum_d |q_r[d]|);
    `written` marks the rows of some sequence."""
    q = np.asarray(q, np.float64)
    M, Hq, D = q.shape
    pages, Hkv, P, _ = params.shape
    G = Hq // Hkv
    out, E, eta = np.zeros_like(q), np.zeros((M, Hq, 1)), np.zeros((M, Hq, 1))
    written = np.zeros(M, bool)
    qr = hadamard_rows(q, k_hadamard)
    for b, length in enumerate(np.asarray(seq_lens).tolist()):
        lo, hi = int(q_starts[b]), int(q_starts[b + 1])
        n = hi - lo
        if n <= 0:
            continue
        slots = sequence_slots(table[b], length, P, pages)
        at = np.flatnonzero(slots >= 0)
        ck, sk, zk = rows(k_codes, params, slots[at])
        cv, sv, zv = rows(v_codes, params, slots[at], value=True)
        K, V = sk[..., None] * (ck - zk[..., None]), sv[..., None] * (cv - zv[..., None])
        kmag = sk[..., None] * (ck + np.abs(ck - zk[..., None]))
        vmag = sv * (np.abs(zv) + np.abs(cv - zv[..., None]).max(-1))
        for i in range(n if max_new is None else min(n, max_new)):
            m = lo + i
            written[m] = True
            see = at <= length - n + i
            if not see.any():
                continue
            for h in range(Hq):
                k = h // G
                s = sm_scale * (K[see, k] @ qr[m, h])
                p = np.exp(s - s.max())
                p /= p.sum()
                out[m, h] = p @ V[see, k]
                E[m, h] = p @ vmag[see, k]
                a = np.abs(qr[m, h])
                eta[m, h] = sm_scale * ((kmag[see, k] @ a).max() + sk[see, k].max() * a.sum() / 16)
    return hadamard_rows(out, v_hadamard), E, eta, written
