"""Shapes beyond what a launch can have are refused by the checks: no GPU needed."""
import pytest

import paper_2511_16047_amd as amskv

A = 1 << 20          # an address that is never followed: every call here ends in the checks


@pytest.mark.parametrize("shape", [dict(batch=1 << 16, heads=256, kv_heads=256, q_tokens=97), dict(batch=1 << 20, heads=16, kv_heads=16, q_tokens=128),
                                   dict(batch=1 << 9, heads=1, kv_heads=1, q_tokens=1 << 22), dict(batch=1 << 10, heads=256, kv_heads=1, q_tokens=1 << 13)],
                         ids=str)
def test_cross_attention_of_more_rows_than_a_launch_has(shape):
    """2^26 blocks of 32 rows, one wave each (less 8, by which a grid may be rounded up)."""
    big = 1 << 36
    x = amskv.Cross(head_dim=64, dtype=amskv.AMSKV_DTYPE_BF16, kv_tokens=40, q=amskv.Strides(0, 0, 64), k=amskv.Strides(0, 0, 64), v=amskv.Strides(0, 0, 64),
                    o=amskv.Strides(big, 1 << 28, 64), **shape)
    rows = shape["heads"] // shape["kv_heads"] * shape["q_tokens"]
    assert shape["batch"] * shape["kv_heads"] * -(-rows // 32) > (1 << 26) - 8
    for call in (lambda: amskv.amskv_cross_workspace_bytes(x), lambda: amskv.amskv_cross_attend(x, A, A, A, 2 * A)):
        with pytest.raises(amskv.AmskvError) as e:
            call()
        assert e.value.status == amskv.AMSKV_ERR_INVALID_ARG
