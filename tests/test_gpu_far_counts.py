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


class Cache8:
    """One layer of 8 bits over scales of single rows."""

    def __init__(self, B, H, D, tokens, pol, **kw):
        args = (1, H, D, (1,) * len(tokens), tokens, B, amskv.AMSKV_DTYPE_BF16_KV8, [pol])
        self.arena = torch.empty(amskv.amskv_cache_required_bytes(*args, **kw), dtype=torch.uint8, device="cuda").fill_(0xFF)
        self.h = amskv.amskv_cache_create(*args, arena=self.arena, **kw)

    def __enter__(self):
        return self.h

    def __exit__(self, *a):
        torch.cuda.synchronize()
        amskv.amskv_cache_destroy(self.h)


@pytest.mark.parametrize("B", [1 << 18, 1 << 20])
def test_compaction_of_very_many_units(B):
    """2^22 and 2^24 (b,h): the scale that stays slides to the front, step after step."""
    H, D, tokens = 16, 64, (1, 1, 2, 1)
    some = [slice(0, 3), slice(B // 2 - 2, B // 2 + 2), slice(B - 3, B)]
    with Cache8(B, H, D, tokens, (0, 1, False)) as h:
        kept = []
        for s, t in enumerate(tokens):
            q, k, v = (_normal(B, H, t, D, seed=10 * s + i) for i in range(3))
            o = torch.full_like(q, 9.0)
            amskv.amskv_append_scale(h, 0, s, k, v)
            amskv.amskv_attend(h, 0, s, q, o)
            kept = kept[-1:] + [[(plain.held(k[x]), plain.held(v[x])) for x in some]]
            n = sum(tokens[s - 1: s + 1]) if s else tokens[0]
            ko, vo = (torch.full((B, H, n, D), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            amskv.amskv_cache_export(h, 0, ko, vo)
            for i, x in enumerate(some):
                kk, vv = (torch.cat([step[i][j] for step in kept], dim=2) for j in range(2))
                assert torch.equal(ko[x].double(), kk) and torch.equal(vo[x].double(), vv)
                want, bound = plain.attention(q[x], kk, vv, 1 / math.sqrt(D))
                assert bool(((o[x].double() - want).abs() <= bound).all())
            assert not bool((ko == 9.0).all(dim=-1).any()) and not bool((vo == 9.0).all(dim=-1).any())


def test_a_read_back_of_very_many_units():
    """2^24 (b,h), the most a cache may have, of one token each: appended, attended, read back."""
    B, H, D = 1 << 20, 16, 64
    with Cache8(B, H, D, (1,), (0, 0, True)) as h:
        q, k, v = (_normal(B, H, 1, D, seed=i) for i in range(3))
        o, ko, vo = (torch.full((B, H, 1, D), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(3))
        amskv.amskv_append_scale(h, 0, 0, k, v)
        amskv.amskv_attend(h, 0, 0, q, o)
        amskv.amskv_cache_export(h, 0, ko, vo)
        for x in (slice(0, 5), slice(B // 2 - 3, B // 2 + 3), slice(B - 5, B)):
            assert torch.equal(ko[x].double(), plain.held(k[x])) and torch.equal(vo[x].double(), plain.held(v[x]))
            assert torch.equal(o[x], vo[x])                       # one key: its value
        assert torch.equal(o, vo) and not bool((ko == 9.0).all(dim=-1).any())


def test_cross_attention_to_the_most_states():
    """2^26 states of one (b,h), K and V of 2^33 bytes each, by queries that look at single ones: four times a key has nearly all the weight."""
    n, D = 1 << 26, 64
    k, v = (torch.empty(n, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for i, x in enumerate((k, v)):
        for j, part in enumerate(x.split(1 << 23)):
            part.copy_(_normal(*part.shape, seed=100 * i + j))
    aims = [n - 1, n - 33, n // 2, n // 2 - 1, (1 << 25) + 5, 31, 0]
    q = 4 * k[aims][None, None]
    qs, st = amskv.Strides(0, 0, D), amskv.Strides(0, 0, D)
    x = amskv.Cross(batch=1, heads=1, kv_heads=1, head_dim=D, dtype=amskv.AMSKV_DTYPE_BF16, q_tokens=len(aims), kv_tokens=n, q=qs, k=st, v=st, o=qs)
    need = amskv.amskv_cross_workspace_bytes(x)
    assert need > 0
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    # the definition, some states at a time: sums of exp(s - top), top being the aimed-at key's score or above it by rounding
    s_top = (q[0, 0].double() * k[aims].double()).sum(dim=-1) / math.sqrt(D) + 4
    total, o, size, largest = 0.0, 0.0, 0.0, 0.0
    for kk, vv in zip(k.split(1 << 21), v.split(1 << 21)):
        p = torch.exp(q[0, 0].double() @ kk.double().T / math.sqrt(D) - s_top[:, None])
        pieces, values = p.view(len(aims), 256, -1).transpose(0, 1).contiguous(), vv.double().view(256, -1, D)
        total, o, size = total + p.sum(dim=1), o + (pieces @ values).sum(dim=0), size + (pieces @ values.abs()).sum(dim=0)
        largest = max(largest, float(kk.abs().amax()))
    want, size = o / total[:, None], size / total[:, None]
    err = (D + 2) * plain.F32 * q[0, 0].double().abs().sum(dim=-1, keepdim=True) * largest / math.sqrt(D) + 2.0 ** -16
    bound = size * (plain.BF16 * 1.004 + 2 * err) + want.abs() * 2.004 * plain.BF16
    for space in (ws, None):
        out = torch.full_like(q, 9.0)
        amskv.amskv_cross_attend(x, q, k, v, out, workspace=space)
        assert bool(((out[0, 0].double() - want).abs() <= bound).all())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Tq", [3, 200])
def test_states_at_the_widest_strides(D, Tq):
    """K and V rows 2^23 - 8 elements apart, in tiles of many rows."""
    T, far = 70, (1 << 23) - 8
    whole = torch.empty((T - 1) * far + 2 * D, dtype=torch.bfloat16, device="cuda")
    k, v = (whole.as_strided((T, D), (far, 1), i * D) for i in range(2))
    k.copy_(_normal(T, D, seed=1)), v.copy_(_normal(T, D, seed=2))
    q = _normal(40, 2, Tq, D, seed=3)
    out = torch.full_like(q, 9.0)
    qs, st = amskv.Strides(2 * Tq * D, Tq * D, D), amskv.Strides(0, 0, far)
    x = amskv.Cross(batch=40, heads=2, kv_heads=2, head_dim=D, dtype=amskv.AMSKV_DTYPE_BF16, q_tokens=Tq, kv_tokens=T, q=qs, k=st, v=st, o=qs)
    amskv.amskv_cross_attend(x, q, k, v, out)
    want, bound = plain.attention(q, k, v, 1 / math.sqrt(D))
    assert bool(((out.double() - want).abs() <= bound).all())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [5, 100])
def test_tokens_at_the_widest_strides(D, T):
    """A scale read in place behind codes, its K and V rows 2^23 - 8 elements apart, and appended to an 8-bit cache from there."""
    H, far = 2, (1 << 23) - 8
    args = (1, H, D, (1, 1), (20, T), 1, amskv.AMSKV_DTYPE_BF16_KV8, [(0, 0, True)])
    for borrow in (False, True):
        kw = dict(borrow_unretained=borrow)
        arena = torch.empty(amskv.amskv_cache_required_bytes(*args, **kw), dtype=torch.uint8, device="cuda").fill_(0xFF)
        h = amskv.amskv_cache_create(*args, arena=arena, **kw)
        try:
            amskv.amskv_cache_set_io_layout(h, amskv.AMSKV_IO_TOKEN_MAJOR, H * D, far, H * D)
            kept = []
            for s, t in enumerate((20, T)):
                whole = torch.empty((t - 1) * far + 2 * H * D, dtype=torch.bfloat16, device="cuda")
                k, v = (whole.as_strided((t, H * D), (far, 1), i * H * D) for i in range(2))
                k.copy_(_normal(t, H * D, seed=s)), v.copy_(_normal(t, H * D, seed=s + 5))
                q = _normal(1, t, H * D, seed=s + 9)
                o = torch.full_like(q, 9.0)
                amskv.amskv_append_scale(h, 0, s, k, v)
                amskv.amskv_attend(h, 0, s, q, o)
                heads = lambda y: y.reshape(1, t, H, D).transpose(1, 2)
                hold = (lambda y: y.double()) if borrow and s == 1 else plain.held
                kept.append((hold(heads(k)), hold(heads(v))))
                kk, vv = (torch.cat([x[j] for x in kept], dim=2) for j in range(2))
                want, bound = plain.attention(heads(q), kk, vv, 1 / math.sqrt(D))
                assert bool(((heads(o).double() - want).abs() <= bound).all())
        finally:
            torch.cuda.synchronize()
            amskv.amskv_cache_destroy(h)
