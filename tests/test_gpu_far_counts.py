"""Counts of (b,h) next to the largest that the calls of the rotary, 8-bit and cross-attention operators take."""
import math

import pytest
import torch

import paper_2511_16047_amd as amskv
import plain_operators as plain

pytestmark = pytest.mark.gpu


def _normal(*shape, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16)


@pytest.mark.parametrize("B,Tk", [(1 << 19, 2048), (1 << 20, 40)])
def test_cross_attention_of_very_many_units(B, Tk):
    """One query each of 2^23 and 2^24 (b,h) to states that all batch elements share."""
    H, D = 16, 64
    q = _normal(B, H, 1, D, seed=1)
    k, v = _normal(Tk, H, D, seed=2), _normal(Tk, H, D, seed=3)
    out = torch.full_like(q, 9.0)
    qs, st = amskv.Strides(H * D, D, D), amskv.Strides(0, D, H * D)
    x = amskv.Cross(batch=B, heads=H, kv_heads=H, head_dim=D, dtype=amskv.AMSKV_DTYPE_BF16, q_tokens=1, kv_tokens=Tk, q=qs, k=st, v=st, o=qs)
    amskv.amskv_cross_attend(x, q, k, v, out)
    assert not bool((out == 9.0).all(dim=-1).any())
    for b in (0, 1, B // 2 - 1, B // 2, B - 1):
        want, bound = plain.attention(q[b], k.transpose(0, 1), v.transpose(0, 1), 1 / math.sqrt(D))
        assert bool(((out[b].double() - want).abs() <= bound).all())
