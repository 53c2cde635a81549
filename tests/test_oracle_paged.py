"""Pins of the paged-cache oracle (CPU), and the host-side rules of the paged entry points: the
rotary frequencies and every refusal, which validation gives before a device is touched."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import attention as OA
from oracle import layer as OL
from oracle import paged as OP
from paper_2606_07116_amd import _lib, inputs

SM = 1 / math.sqrt(128)


def _pages_of(kc, ks, kz, vc, vs, vz, P):
    """A contiguous cache [B, H, S, ...] as pages of P positions (S a multiple of P)."""
    B, H, S = ks.shape
    par = np.stack([ks.view(np.int16), kz, vs.view(np.int16), vz], -1)

    def pages(t):
        return np.ascontiguousarray(
            t.reshape(B, H, S // P, P, -1).transpose(0, 2, 1, 3, 4)).reshape(B * S // P, H, P, -1)

    return pages(kc), pages(vc), pages(par)


def test_attention_equals_the_contiguous_oracle():
    B, H, S, P, T, past = 2, 2, 64, 16, 5, 40
    kc, ks, kz = inputs.kv4_cache(B, H, S, 128, seed=1)
    vc, vs, vz = inputs.kv4_cache(B, H, S, 128, seed=2)
    q = inputs.queries(B * T, 4, 128, seed=3)
    ref = OA.prefill_attention(q.reshape(B, T, 4, 128), kc, ks, kz, vc, vs, vz, past, SM,
                               v_hadamard=True)
    pk, pv, par = _pages_of(kc, ks, kz, vc, vs, vz, P)
    table = np.arange(B * S // P).reshape(B, -1)
    out, E, eta, written = OP.attention(q, [0, T, 2 * T], [past + T] * B, table, pk, pv, par, SM,
                                        v_hadamard=True)
    assert written.all()
    # the contiguous oracle rounds the rotated query to bf16: scores off by 2^-8 of their terms
    assert np.all(np.abs(out.reshape(ref.shape) - ref).max(-1, keepdims=True)
                  <= 2 * 2.0 ** -8 * (eta * E).reshape(B, T, 4, 1) * math.sqrt(128))


def test_attention_equals_torch_and_skips_absent_pages():
    rng = np.random.default_rng(5)
    D, P, pages, H = 64, 16, 7, 2
    kc, vc = (rng.integers(0, 256, (pages, H, P, D // 2), dtype=np.uint8) for _ in range(2))
    par = np.empty((pages, H, P, 4), np.int16)
    par[..., ::2] = rng.uniform(0.05, 0.6, (pages, H, P, 2)).astype(np.float16).view(np.int16)
    par[..., 1::2] = rng.integers(-40, 40, (pages, H, P, 2))
    q = rng.standard_normal((3, 4, D))
    table = np.array([[5, -1, 2]])
    out, _, _, _ = OP.attention(q, [0, 3], [45], table, kc, vc, par, 0.2, k_hadamard=False)
    slots = OP.sequence_slots(table[0], 45, P, pages)
    seen = slots >= 0
    assert seen.sum() == 16 + 13 and not seen[16:32].any()
    k, v = (torch.from_numpy(OP.dequantize(c, par, slots.clip(0), value=i).transpose(1, 0, 2))
            for i, c in ((False, kc), (True, vc)))
    mask = torch.from_numpy(seen[None] & (np.arange(45) <= 42 + np.arange(3)[:, None]))
    ref = torch.nn.functional.scaled_dot_product_attention(
        torch.from_numpy(q.transpose(1, 0, 2)).reshape(1, 4, 3, D),
        k.repeat_interleave(2, 0)[None], v.repeat_interleave(2, 0)[None], attn_mask=mask, scale=0.2)
    assert np.allclose(out, ref[0].numpy().transpose(1, 0, 2), rtol=1e-10, atol=1e-12)


def test_attention_rows_that_see_nothing():
    par = np.zeros((2, 1, 16, 4), np.int16)
    par[..., 0] = par[..., 2] = np.float16(1).view(np.int16)
    codes = np.full((2, 1, 16, 32), 0x55, np.uint8)
    out, _, _, written = OP.attention(np.ones((6, 1, 64)), [0, 3, 5, 5], [2, 0, 9],
                                      [[0], [1], [1]], codes, codes, par, 1.0)
    # three rows on two positions: the first sits before the sequence; then an empty sequence
    assert not out[0].any() and out[1].any() and out[2].any() and not out[3:].any()
    assert written.tolist() == [True] * 5 + [False]


def test_rotation():
    x = inputs.queries(4, 3, 128, seed=9)
    pos = np.array([0, 1, 7, 300])
    f = OP.inv_freq(128, 500000.0).astype(np.float32)
    got = OP.rotate(x, pos, f, False, 1.0)
    ref = OL.rope(x, pos[:, None], 500000.0)
    # the layer's angles are rounded to fp32 (2^-24 of at most 300)
    assert np.all(np.abs(got - ref) <= 300 * 2.0 ** -23 * np.abs(x).max())
    # interleaved: the half layout of the channels taken in the other order
    perm = np.arange(128).reshape(64, 2).T.reshape(-1)
    assert np.allclose(OP.rotate(x, pos, f, True, 2.0)[..., perm],
                       2 * OP.rotate(x[..., perm], pos, f, False, 1.0), atol=1e-12)
    part = OP.rotate(x, pos, f[:16], False, 1.0)
    assert np.array_equal(part[..., 32:], x[..., 32:])
    assert np.allclose((part ** 2).sum(-1), (np.float64(x) ** 2).sum(-1))


def _freq(*args):
    out = (ctypes.c_float * 64)()
    assert _lib.offq_rope_inv_freq_raw(*args, out) == _lib.OFFQ_OK, _lib.last_error()
    return np.array(out[:args[0] // 2], np.float64)


@pytest.mark.parametrize("args", [
    (128, 500000.0, 1.0, 1.0, 4.0, 0.0), (64, 10000.0, 8.0, 1.0, 4.0, 0.0),
    (128, 500000.0, 8.0, 1.0, 4.0, 8192.0), (32, 10000.0, 40.0, 1.0, 32.0, 4096.0),
    (2, 10000.0, 1.0, 0.0, 0.0, 0.0),
])
def test_rope_inv_freq(args):
    got, ref = _freq(*args), OP.inv_freq(*args)
    assert np.all(np.abs(got - ref) <= 2.0 ** -24 * (1 + 1e-6) * ref)
    if args[5]:
        plain = OP.inv_freq(args[0], args[1])
        turns = args[5] * plain / (2 * np.pi)
        assert np.allclose(got[turns >= args[4]], plain[turns >= args[4]], rtol=1e-6)
        assert np.allclose(got[turns <= args[3]], plain[turns <= args[3]] / args[2], rtol=1e-6)


@pytest.mark.parametrize("args", [
    (0, 1e4, 1.0, 1.0, 4.0, 0.0), (7, 1e4, 1.0, 1.0, 4.0, 0.0), (64, 1.0, 1.0, 1.0, 4.0, 0.0),
    (64, float("nan"), 1.0, 1.0, 4.0, 0.0), (64, 1e4, 0.5, 1.0, 4.0, 0.0),
    (64, 1e4, 8.0, 4.0, 4.0, 8192.0), (64, 1e4, 8.0, -1.0, 4.0, 8192.0),
    (64, 1e4, 8.0, 1.0, 4.0, -5.0), (64, 1e4, 8.0, 1.0, float("inf"), 8192.0),
])
def test_rope_inv_freq_refusals(args):
    out = (ctypes.c_float * 64)()
    assert _lib.offq_rope_inv_freq_raw(*args, out) == _lib.OFFQ_ERR_INVALID
    assert _lib.offq_rope_inv_freq_raw(64, 1e4, 1.0, 1.0, 4.0, 0.0, None) == _lib.OFFQ_ERR_INVALID


A = 0x100000  # fake aligned addresses, far enough apart: validation fails before any is used
BAD, UNS, OK = _lib.OFFQ_ERR_INVALID, _lib.OFFQ_ERR_UNSUPPORTED, _lib.OFFQ_OK

WRITE = dict(qkv=A, ldq=6 * 128, M=4, Hq=4, Hkv=1, head_dim=128, q_weight=None, k_weight=None,
             eps=1e-6, positions=A, rotary_dim=128, interleaved=0, inv_freq=A, amplitude=1.0,
             k_hadamard=1, v_hadamard=0, q_out=4 * A, ldo=512, slots=A, k_codes=A, v_codes=A,
             kv_params=A, num_pages=8, page_size=16, stream=None)


@pytest.mark.parametrize("change,expect", [
    (dict(M=-1), BAD), (dict(Hq=0), BAD), (dict(Hkv=0), BAD), (dict(num_pages=0), BAD),
    (dict(head_dim=96), UNS), (dict(head_dim=256), UNS), (dict(page_size=24), BAD),
    (dict(page_size=8), UNS), (dict(page_size=8192), UNS), (dict(k_hadamard=2), BAD),
    (dict(v_hadamard=-1), BAD), (dict(ldq=760), BAD), (dict(ldq=772), BAD), (dict(ldo=504), BAD),
    (dict(ldo=516), BAD), (dict(rotary_dim=24), BAD), (dict(rotary_dim=144), BAD),
    (dict(rotary_dim=-16), BAD), (dict(interleaved=2), BAD), (dict(eps=-1.0), BAD),
    (dict(eps=float("nan")), BAD), (dict(amplitude=float("inf")), BAD), (dict(qkv=None), BAD),
    (dict(qkv=A + 8), BAD), (dict(positions=None), BAD), (dict(slots=None), BAD),
    (dict(slots=A + 4), BAD), (dict(q_out=None), BAD), (dict(q_out=4 * A + 2), BAD),
    (dict(q_weight=A + 2), BAD), (dict(k_weight=A + 8), BAD), (dict(inv_freq=None), BAD),
    (dict(k_codes=None), BAD), (dict(v_codes=A + 4), BAD), (dict(kv_params=A + 4), BAD),
    (dict(q_out=A + 64), BAD), (dict(M=1 << 31), UNS), (dict(num_pages=1 << 37), UNS),
    (dict(Hq=1 << 17, ldq=1 << 30, ldo=1 << 30), UNS), (dict(M=0, qkv=None, slots=None), OK),
])
def test_rope_kv_paged_refusals(change, expect):
    st = _lib.offq_rope_kv_paged_raw(*{**WRITE, **change}.values())
    assert st == expect, _lib.last_error()
    assert st == OK or _lib.last_error()


READ = dict(k_codes=A, v_codes=A, kv_params=A, num_pages=8, page_size=16, Hkv=2, head_dim=64,
            slots=A, M=5, k_hadamard=1, v_hadamard=0, k_out=2 * A, ldk=128, v_out=4 * A, ldv=128,
            stream=None)


@pytest.mark.parametrize("change,expect", [
    (dict(M=-1), BAD), (dict(Hkv=0), BAD), (dict(num_pages=-1), BAD), (dict(head_dim=32), UNS),
    (dict(page_size=0), BAD), (dict(page_size=4), UNS), (dict(k_hadamard=3), BAD),
    (dict(ldk=120), BAD), (dict(ldv=132), BAD), (dict(slots=None), BAD), (dict(slots=A + 4), BAD),
    (dict(k_out=None, v_out=None), BAD), (dict(k_out=2 * A + 8), BAD), (dict(v_codes=None), BAD),
    (dict(v_out=2 * A), BAD), (dict(v_out=2 * A + 256, ldk=256, ldv=248), BAD),
    (dict(v_out=2 * A + 128, ldk=256, ldv=256), BAD), (dict(M=1 << 31), UNS),
    (dict(M=0, slots=None, k_out=None, v_out=None), OK),
])
def test_kv_dequantize_paged_refusals(change, expect):
    st = _lib.offq_kv_dequantize_paged_raw(*{**READ, **change}.values())
    assert st == expect, _lib.last_error()


ATTEND = dict(q=2 * A, ldq=512, M=6, Hq=4, Hkv=2, head_dim=128, q_starts=A, seq_lens=A, B=3,
              max_new=4, page_table=A, max_pages=9, k_codes=A, v_codes=A, kv_params=A, num_pages=8,
              page_size=16, sm_scale=0.1, k_hadamard=1, v_hadamard=0, out=4 * A, ldo=512,
              workspace=A, workspace_bytes=1 << 40, stream=None)


@pytest.mark.parametrize("change,expect", [
    (dict(M=-1), BAD), (dict(B=-1), BAD), (dict(max_new=-1), BAD), (dict(max_pages=0), BAD),
    (dict(Hq=5), BAD), (dict(Hq=0), BAD), (dict(head_dim=80), UNS), (dict(page_size=48), BAD),
    (dict(page_size=1 << 13), UNS), (dict(sm_scale=0.0), BAD), (dict(sm_scale=float("nan")), BAD),
    (dict(sm_scale=float("inf")), BAD), (dict(ldq=504), BAD), (dict(ldo=516), BAD),
    (dict(q=None), BAD), (dict(q=2 * A + 8), BAD), (dict(q_starts=None), BAD),
    (dict(seq_lens=A + 2), BAD), (dict(page_table=None), BAD), (dict(out=None), BAD),
    (dict(out=2 * A + 1024), BAD), (dict(v_codes=A + 8), BAD), (dict(kv_params=None), BAD),
    (dict(workspace=A + 4), BAD), (dict(M=1 << 25), UNS), (dict(B=1 << 21), UNS),
    (dict(max_pages=1 << 27), UNS), (dict(num_pages=1 << 33), UNS),
    (dict(M=0, q=None, out=None, workspace=None, workspace_bytes=0), OK),
    (dict(B=0, q_starts=None, workspace=None, workspace_bytes=0), OK),
    (dict(max_new=0, workspace=None, workspace_bytes=0), OK),
])
def test_kv_attention_paged_refusals(change, expect):
    st = _lib.offq_kv_attention_paged_raw(*{**ATTEND, **change}.values())
    assert st == expect, _lib.last_error()


def test_workspace_bytes():
    f = _lib.offq_kv_attention_paged_workspace_bytes
    assert f(0, 4, 8, 8, 128, 1) == 0 and f(4, 0, 8, 8, 128, 1) == 0
    assert f(4, 4, 8, 3, 128, 1) == 0 and f(4, 4, 8, 8, 96, 1) == 0 and f(-1, 4, 8, 8, 128, 1) == 0
    need = f(6, 3, 4, 2, 128, 4)
    assert need >= 0 and need % 4 == 0
    if need:
        for short in (dict(workspace_bytes=need - 1), dict(workspace=None)):
            assert _lib.offq_kv_attention_paged_raw(*{**ATTEND, **short}.values()) == BAD
            assert "workspace" in _lib.last_error()


def test_more_threads_than_a_launch_has():
    """A wave per token, head_dim / 8 lanes per row, a workgroup per joined row: under 2^32 threads."""
    assert _lib.offq_rope_kv_paged_raw(*{**WRITE, "M": (1 << 26) - 3, "q_out": 1 << 45}.values()) == UNS
    for change in (dict(M=1 << 28, Hkv=2, head_dim=64), dict(M=1 << 24, Hkv=16, head_dim=128)):
        D = change["head_dim"] * change["Hkv"]
        big = {**READ, **change, "k_out": 1 << 44, "v_out": 1 << 46, "ldk": D, "ldv": D}
        assert _lib.offq_kv_dequantize_paged_raw(*big.values()) == UNS
    f = _lib.offq_kv_attention_paged_workspace_bytes
    many = dict(B=1 << 17, Hkv=2)
    assert f(1 << 17, many["B"], 4, many["Hkv"], 128, 1) == 0
    assert _lib.offq_kv_attention_paged_raw(*{**ATTEND, **many}.values()) == UNS
    assert f(1 << 16, 1 << 16, 4, 2, 128, 1) > 0
