"""Combinations of the operators' forms: K turned in its own buffer in every type, teams of eight waves over many tiles, and the far end of a
long cache by queries that look there."""
import math

import pytest
import torch

import paper_2511_16047_amd as amskv
import plain_operators as plain
from test_gpu_cache_in_8_bits import Cache, _drive, _normal
from test_gpu_rotary import KINDS, _run_cache

pytestmark = pytest.mark.gpu

BORROW = dict(borrow_unretained=True)
IN_PLACE = {"borrow": BORROW, "planned": dict(BORROW, layout=amskv.AMSKV_LAYOUT_PLANNED), "fuse": dict(fuse_append=True),
            "all": dict(BORROW, layout=amskv.AMSKV_LAYOUT_PLANNED, fuse_append=True), "budget": dict(budgets=[(20, 40, 5, 2.0)]),
            "window": dict(windows=[(30, 5)])}


@pytest.mark.parametrize("kind,how", [(k, h) for k in KINDS for h in IN_PLACE if k != "8 bits" or h in ("borrow", "planned")])
@pytest.mark.parametrize("D,rot,pairing", [(64, 64, "interleaved"), (128, 96, "half")])
@pytest.mark.parametrize("packed", ["", "in place", "apart"])
@pytest.mark.parametrize("policy", [(1, 1, False), (2, 0, False)], ids=["window", "condensed"])
def test_keys_turned_in_their_own_buffer(kind, how, D, rot, pairing, packed, policy):
    """What becomes of the caller's K, what the cache holds and what is attended.  A scale that no later step reads stays where it is
    (borrowed), all do (fused, the token modes), the others are copied and K is only read."""
    kw = IN_PLACE[how]
    if how in ("budget", "window") and policy[1] == 0:
        policy = (1, 1, False)     # (not read there)
    steps, segs, ko, vo = _run_cache(KINDS[kind], D, pairing, rot, bool(packed), policy, q_apart=packed == "apart", **dict(kw))
    dt = torch.float32 if kind == "f32" else torch.bfloat16
    c, w, _ = policy
    kept = {}
    for s, (turned, want_q, want_k, v, out, k_after, k, buffer) in enumerate(steps):
        later = s + 1 < len(steps) and (s < c or w > 0)
        here = bool(kw.get("fuse_append") or "budgets" in kw or "windows" in kw or (kw.get("borrow_unretained") and not later))
        assert torch.equal(turned, want_q.to(dt))
        assert torch.equal(k_after, want_k.to(dt) if here else k)
        if packed:
            assert torch.equal(buffer[:, :, 2].reshape(*v.transpose(1, 2).shape).transpose(1, 2), v)
        coded = kind == "8 bits" and not here
        kept[s] = (plain.held(want_k), plain.held(v)) if coded else (want_k.to(dt).double(), v.double())
        if "budgets" in kw or "windows" in kw:
            continue
        now = [i for i in range(s + 1) if i < c or s - i <= w]
        kk, vv = (torch.cat([kept[i][j] for i in now], dim=2) for j in range(2))
        o, bound = plain.attention(turned, kk, vv, 1 / math.sqrt(D))
        if kind == "f32":
            assert float((out.double() - o).abs().max()) <= 1e-4      # the fp32 contract
        else:
            assert bool(((out.double() - o).abs() <= bound).all())
    at = 0
    for scale, first, _, n in segs:
        assert torch.equal(ko[:, :, at:at + n].double(), kept[scale][0][:, :, first:first + n])
        assert torch.equal(vo[:, :, at:at + n].double(), kept[scale][1][:, :, first:first + n])
        at += n


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("before", [2500, 2528, 2560])
@pytest.mark.parametrize("borrow", [False, True])
def test_teams_of_eight_over_many_tiles(D, before, borrow):
    """39 to 44 tiles of codes, whole and not, the last ones codes too or rows read in place."""
    _drive([(1, before), (1, 256)], 10, 15, D, [(1, 0, False)], seed=before, borrow_unretained=borrow)


def test_queries_that_look_at_the_far_end():
    """45000 tokens of 384 (b,h), offsets beyond 2^31 bytes.  Each query is four times one key, whose weight is then above 0.99 (its score
    is near 4 * 128 / sqrt(128) = 45, the others' are a few times 4): a key that is lost or in another's place is seen."""
    B, H, D, T = 24, 16, 128, 45000
    aims = [T - 1, T - 2, T - 16, T - 17, T - 33, T - 65, T // 2, T // 2 + 1, 31, 32, 1, 0]
    with Cache([(1, T), (1, len(aims))], B, H, D, [(1, 0, False)]) as c:
        assert B * H * T * D > 2 ** 31
        g = torch.Generator(device="cuda")
        g.manual_seed(1)
        k = torch.empty(B, H, T, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        v = torch.empty(B, H, T, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        amskv.amskv_append_scale(c.h, 0, 0, k, v)
        q = 4 * k[:, :, aims].contiguous()
        k1, v1 = (_normal(B, H, len(aims), D, seed=i).bfloat16() for i in (1, 2))
        o = torch.empty_like(q)
        amskv.amskv_append_scale(c.h, 0, 1, k1, v1)
        amskv.amskv_attend(c.h, 0, 1, q, o)
        for b, h in ((0, 0), (0, H - 1), (11, 3), (B - 1, 0), (B - 1, H - 1)):
            kk, vv = (torch.cat([plain.held(x[b, h]), plain.held(y[b, h])], dim=0) for x, y in ((k, k1), (v, v1)))
            want, bound = plain.attention(q[b, h], kk, vv, 1 / math.sqrt(D))
            weight = torch.softmax(q[b, h].double() @ kk.T / math.sqrt(D), dim=-1)
            assert bool((weight[torch.arange(len(aims)), aims] > 0.99).all())
            assert bool(((o[b, h].double() - want).abs() <= bound).all())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H", [2, 40])
@pytest.mark.parametrize("long", [255, 512, 513, 1500, 5000])
def test_long_survivors_behind_short_scales(D, H, long):
    """Survivors that slide by one block in one pass and in many, in the launch of the append and in one of their own."""
    _drive([(1, 16), (1, long), (1, 5), (1, 40)], 1, H, D, [(0, 2, False), (0, 1, False)] if H == 2 else [(0, 2, False)], seed=long)
