"""Host-side checks of the paged entry points' row strides (no device: validation comes first)."""
import pytest

from paper_2606_07116_amd import _lib
from tests.test_oracle_paged import ATTEND, READ, UNS, WRITE


@pytest.mark.parametrize("ld", [1 << 40, 1 << 36, 3 << 38])
@pytest.mark.parametrize("raw,good,rows,strides", [
    ("offq_rope_kv_paged_raw", {**WRITE, "q_out": 1 << 45}, [(1 << 26) - 4, 1 << 25], ("ldq", "ldo")),
    ("offq_kv_dequantize_paged_raw", {**READ, "v_out": 1 << 45}, [(1 << 28) - 1, 1 << 23], ("ldk", "ldv")),
    ("offq_kv_attention_paged_raw", {**ATTEND, "out": 1 << 45, "workspace_bytes": 1 << 60},
     [1 << 24, 1 << 22], ("ldq", "ldo")),
])
def test_rows_beyond_any_memory(raw, good, rows, strides, ld):
    """Rows that end past 2^40 elements are refused before their ends are computed in 64 bits."""
    for M in rows:
        for s in (strides[:1], strides[1:], strides):
            st = getattr(_lib, raw)(*{**good, "M": M, **{n: ld for n in s}}.values())
            assert st == UNS and "too large" in _lib.last_error(), (M, s, st, _lib.last_error())


def test_long_rows_of_few_tokens_pass():
    """(a NULL pointer is found after the sizes)"""
    for raw, good, what in (("offq_rope_kv_paged_raw", {**WRITE, "ldq": 1 << 30, "ldo": 1 << 37}, "slots"),
                            ("offq_kv_dequantize_paged_raw", {**READ, "ldk": 1 << 37}, "slots"),
                            ("offq_kv_attention_paged_raw", {**ATTEND, "ldq": 1 << 37}, "q_starts")):
        assert getattr(_lib, raw)(*{**good, what: None}.values()) == _lib.OFFQ_ERR_INVALID
        assert "null" in _lib.last_error()
