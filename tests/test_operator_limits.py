"""Shapes beyond what a launch can have are refused by the checks: no GPU needed."""
import pytest
import torch

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


# ---------------------------------------------------------------- one tensor in two roles
SAME = [  # Q, Q_out, K, V; refused where the scale is copied into the cache, refused where it is read in place
    ((1, 2, 3, 4), False, False), ((1, 1, 3, 4), False, False), ((None, None, 3, 4), False, False),
    ((1, 3, 3, 4), True, True), ((1, 4, 3, 4), True, True), ((3, 3, 3, 4), True, True), ((4, 4, 3, 4), True, True), ((1, 3, 3, 3), True, True),
    ((1, 2, 3, 3), False, True), ((None, None, 3, 3), False, True), ((3, 2, 3, 4), False, True), ((4, 2, 3, 4), False, False)]


@pytest.mark.parametrize("tensors,copied,in_place", SAME, ids=str)
@pytest.mark.parametrize("dtype,how", [(t, h) for t in (amskv.AMSKV_DTYPE_F32, amskv.AMSKV_DTYPE_BF16, amskv.AMSKV_DTYPE_BF16_KV8)
                                       for h in ({}, dict(borrow_unretained=True), dict(fuse_append=True))
                                       if not (t == amskv.AMSKV_DTYPE_BF16_KV8 and h.get("fuse_append"))], ids=str)
def test_rotary_append_of_one_tensor_in_two_roles(tensors, copied, in_place, dtype, how):
    """A tensor that the launch turns is none that it also reads: the queries' place is not K or V, and K that is turned in its own buffer
    is neither V nor what the queries are read from.  The arena's address is never followed: what is not refused here ends at the launch,
    for want of a device."""
    h = amskv.amskv_cache_create(1, 2, 64, (1, 2), (1, 2), 1, dtype, [(0, 1, False)], arena=A, arena_bytes=A, **how)
    try:
        q, q_out, k, v = (None if t is None else 2 * A * t for t in tensors)
        last = how.get("borrow_unretained", False)                 # the last scale of all is read by no later step
        if last:
            amskv.amskv_append_scale(h, 0, 0)
        refused = in_place if how else copied
        if refused or not torch.cuda.is_available():
            with pytest.raises(amskv.AmskvError) as e:
                amskv.amskv_append_scale_rotary(h, 0, int(last), amskv.Rope(rot_dim=64), A, q, 0, q_out, k, v, stream=0)
            assert (e.value.status == amskv.AMSKV_ERR_INVALID_ARG) == refused
    finally:
        amskv.amskv_cache_destroy(h)
