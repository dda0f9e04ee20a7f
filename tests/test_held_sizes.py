"""Held tensors of another size than the call's shape says are refused, before anything is launched: no GPU needed."""
import pytest
import torch

import paper_2511_16047_amd as amskv
from paper_2511_16047_amd import binding

A = 1 << 20          # an address that is never followed: every call here ends in the checks
SMALL, INVALID = amskv.AMSKV_ERR_ARENA_TOO_SMALL, amskv.AMSKV_ERR_INVALID_ARG


def _cross(**k):
    s, kv = amskv.Strides(6 * 64 * 7, 64 * 7, 64), amskv.Strides(3 * 64 * 11, 64, 3 * 64)
    return amskv.Cross(**dict(dict(batch=2, heads=6, kv_heads=3, head_dim=64, dtype=amskv.AMSKV_DTYPE_BF16_KV4, q_tokens=7, kv_tokens=11, kv_rows=20,
                                   q=s, k=kv, v=kv, o=s), **k))


def _calls(cross, k, v, where):
    yield amskv.amskv_cross_hold, (cross, A, 2 * A, k, v), where
    yield amskv.amskv_cross_export, (cross, k, v, A, 2 * A), where
    yield amskv.amskv_cross_attend, (cross, A, k, v, 2 * A), where


def _refused(status, cross, k, v, where):
    for call, a, kw in _calls(cross, k, v, where):
        with pytest.raises(amskv.AmskvError) as e:
            call(*a, **kw)
        assert e.value.status == status, call.__name__


@pytest.fixture(params=["extension", "ctypes"], autouse=True)
def way(request, monkeypatch):
    amskv.amskv_cross_held_bytes(_cross())        # (the library is loaded)
    if request.param == "ctypes":
        for name in ("_hold", "_export", "_cross"):
            monkeypatch.setattr(binding, name, binding._not_built)


@pytest.mark.parametrize("where", [{}, {"lengths": A}, {"offsets": A}], ids=lambda x: "".join(x))
@pytest.mark.parametrize("by,status", [(-1, SMALL), (1, INVALID)])
def test_one_of_the_two(where, by, status):
    need = amskv.amskv_cross_held_bytes(_cross(), packed="offsets" in where)
    right, wrong = torch.empty(need, dtype=torch.uint8), torch.empty(need + by, dtype=torch.uint8)
    _refused(status, _cross(), wrong, right, where)
    _refused(status, _cross(), right, wrong, where)


def test_held_with_another_shape():
    """Another batch, capacity or number of heads, padded for packed: their powers of two would be looked for elsewhere."""
    held = [torch.empty(amskv.amskv_cross_held_bytes(_cross()), dtype=torch.uint8) for _ in range(2)]
    _refused(INVALID, _cross(batch=1), *held, {})
    _refused(SMALL, _cross(batch=3), *held, {})
    _refused(INVALID, _cross(kv_tokens=10), *held, {})
    _refused(INVALID, _cross(heads=2, kv_heads=2), *held, {})
    _refused(SMALL, _cross(head_dim=128), *held, {})
    _refused(INVALID, _cross(), *held, {"offsets": A})


def test_bytes_count_not_elements():
    need = amskv.amskv_cross_held_bytes(_cross())
    _refused(INVALID, _cross(), *(torch.empty(need, dtype=torch.int16) for _ in range(2)), {})
    _refused(SMALL, _cross(), *(torch.empty(need // 4 - 1, dtype=torch.float32) for _ in range(2)), {})
