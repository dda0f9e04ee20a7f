"""Rotary tables, turning tensors, and appending turned keys, against the formulas in 64 bits."""
import math

import pytest
import torch

import paper_2511_16047_amd as amskv
import plain_operators as plain

pytestmark = pytest.mark.gpu
F32 = plain.F32


def _normal(*shape, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda")


def _pairing(name):
    return amskv.AMSKV_ROPE_HALF if name == "half" else amskv.AMSKV_ROPE_INTERLEAVED


def _table(rope, where):
    t = torch.full((where.shape[0], rope.rot_dim // 2, 2), float("nan"), device="cuda")
    amskv.amskv_rope_table(rope, where, t)
    return t


@pytest.mark.parametrize("rot,axes,n", [(16, 1, 1), (64, 1, 257), (48, 2, 100), (128, 2, 4096), (128, 1, 7), (80, 2, 33)])
@pytest.mark.parametrize("long", [{}, dict(factor=4.0), dict(factor=8.0, original=4096.0, low=1.0, high=32.0, amplitude=1.2)], ids=["as trained", "linear", "by parts"])
def test_table(rot, axes, n, long):
    """Within half a step of fp32, and what fp64 angles leave: positions up to 1e6 times a frequency, 2^-52 each of 1e6."""
    where = (_normal(n, axes, seed=n) * 1e5).double().round() + torch.tensor([0.25] * axes, device="cuda").double()
    where[0] = 0
    got = _table(amskv.Rope(rot_dim=rot, axes=axes, **long), where)
    k = dict(long)
    want = plain.table(where, rot, amplitude=k.pop("amplitude", 1.0), **k)
    assert float((got.double() - want).abs().max()) <= 1.2 * F32 + 1e6 * 2.0 ** -50


def _turned_bound(x, tab, pairing, half_step):
    """Per element: the table's rounding, two products and a sum (2^-24 each of the magnitudes), the type's half step."""
    size = plain.turn(x.double().abs(), torch.stack((tab[..., 0].abs(), -tab[..., 1].abs()), dim=-1), pairing).abs()
    size = torch.maximum(size, plain.turn(x.double().abs(), tab.abs(), pairing).abs())
    return 4 * F32 * size + half_step * size


SHAPES = [  # B, H, T, D, rot
    (1, 1, 1, 64, 64), (3, 5, 1, 128, 128), (2, 17, 2, 64, 48), (2, 3, 4, 128, 16), (1, 9, 8, 64, 32), (2, 4, 9, 128, 96), (1, 2, 16, 64, 16),
    (2, 7, 17, 64, 64), (1, 3, 100, 128, 64), (2, 30, 169, 64, 64), (5, 33, 25, 128, 128), (40, 24, 36, 64, 64)]


@pytest.mark.parametrize("B,H,T,D,rot", SHAPES)
@pytest.mark.parametrize("pairing", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rotate(B, H, T, D, rot, pairing, dtype):
    """Every layout of the two tensors, one table and one per batch element, there and back; the rest of the row and what lies
    around it stay."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    rope = amskv.Rope(rot_dim=rot, pairing=_pairing(pairing))
    x = (_normal(B, H, T, D, seed=T) * torch.exp(_normal(H, 1, D, seed=1))).to(dt)
    for each in (False, True):
        where = (_normal(B if each else 1, T, 1, seed=3) * 1000).double()
        tab = _table(rope, where.flatten(0, 1)).view(-1, T, rot // 2, 2)
        row = T * rot if each else 0
        per_head = tab[:, None]
        bound = _turned_bound(x, per_head.double(), pairing, plain.BF16 if dtype == "bf16" else 0.0)
        for back in (False, True):
            want = plain.turn(x.double(), per_head.double(), pairing, back)
            bits = plain.turn(x.float(), per_head, pairing, back).to(dt)   # the same formula in fp32: the same bits
            def check(out):
                assert bool(((out.double() - want).abs() <= bound).all())
                assert torch.equal(out, bits)
            out = torch.empty_like(x)
            xs = amskv.Strides(H * T * D, T * D, D)
            args = (rope, amskv.AMSKV_DTYPE_BF16 if dtype == "bf16" else amskv.AMSKV_DTYPE_F32, D, B, H, T, tab, row)
            amskv.amskv_rotate(*args, x, xs, out, xs, inverse=back)
            check(out)
            # out of a projection output [B][T][3][H][D], into [B][T][H][D] with a margin that must stay
            qkv = torch.zeros(B, T, 3, H, D, dtype=dt, device="cuda")
            qkv[:, :, 1] = x.transpose(1, 2)
            wide = torch.full((B, T, H + 1, D), 7.0, dtype=dt, device="cuda")
            amskv.amskv_rotate(*args, qkv[:, :, 1], amskv.Strides(3 * T * H * D, D, 3 * H * D), wide, amskv.Strides(T * (H + 1) * D, D, (H + 1) * D),
                               inverse=back)
            check(wide[:, :, :H].transpose(1, 2).contiguous())
            assert bool((wide[:, :, H] == 7.0).all())
            # in place
            z = x.clone()
            amskv.amskv_rotate(*args, z, xs, z, xs, inverse=back)
            check(z)


@pytest.mark.parametrize("B,H,T", [(20001, 1, 17), (3001, 7, 1), (5, 5, 9000), (1, 1, 300001)])
def test_many_rows(B, H, T):
    """More blocks than waves that take one head each."""
    rope = amskv.Rope(rot_dim=32, pairing=amskv.AMSKV_ROPE_INTERLEAVED)
    tab = _table(rope, (_normal(T, 1, seed=3) * 1000).double())
    x = _normal(B, H, T, 64, seed=T).bfloat16()
    out, xs = torch.full_like(x, 7.0), amskv.Strides(H * T * 64, T * 64, 64)
    amskv.amskv_rotate(rope, amskv.AMSKV_DTYPE_BF16, 64, B, H, T, tab, 0, x, xs, out, xs)
    assert torch.equal(out, plain.turn(x.float(), tab, "interleaved").bfloat16())


def test_far_rows():
    """A tensor beyond 2^32 bytes, turned in place, with the most tokens it may have."""
    H, T, D = 9, 1 << 22, 64
    rope = amskv.Rope(rot_dim=16)
    tab = _table(rope, torch.arange(T, dtype=torch.float64, device="cuda")[:, None])
    x = torch.empty(1, H, T, D, dtype=torch.bfloat16, device="cuda").fill_(0.5)
    x[..., :16] = _normal(16, seed=1).bfloat16()
    want = plain.turn(x[0, 0].float(), tab, "half").bfloat16()
    xs = amskv.Strides(0, T * D, D)
    amskv.amskv_rotate(rope, amskv.AMSKV_DTYPE_BF16, D, 1, H, T, tab, 0, x, xs, x, xs)
    for h in range(H):
        assert torch.equal(x[0, h], want)


def test_a_head_for_all():
    """A tensor that repeats is read with stride 0."""
    B, H, T, D = 2, 6, 20, 64
    rope = amskv.Rope(rot_dim=64)
    tab = _table(rope, torch.arange(T, dtype=torch.float64, device="cuda")[:, None])
    x = _normal(B, 1, T, D).bfloat16()
    out = torch.empty(B, H, T, D, dtype=torch.bfloat16, device="cuda")
    amskv.amskv_rotate(rope, amskv.AMSKV_DTYPE_BF16, D, B, H, T, tab, 0, x, amskv.Strides(T * D, 0, D), out, amskv.Strides(H * T * D, T * D, D))
    assert torch.equal(out, plain.turn(x.float(), tab, "half").bfloat16().expand(B, H, T, D))


@pytest.mark.parametrize("pairing", ["half", "interleaved"])
def test_back_is_the_gradient(pairing):
    """<turn(x), g> = <x, back(g)>, against differences of the formula in 64 bits and autograd's own."""
    B, H, T, D, rot = 2, 3, 10, 64, 48
    rope = amskv.Rope(rot_dim=rot, pairing=_pairing(pairing), amplitude=1.3)
    tab = _table(rope, (_normal(T, 1) * 50).double())
    x, g = _normal(B, H, T, D, seed=1), _normal(B, H, T, D, seed=2)
    got = torch.empty_like(g)
    s = amskv.Strides(H * T * D, T * D, D)
    amskv.amskv_rotate(rope, amskv.AMSKV_DTYPE_F32, D, B, H, T, tab, 0, g, s, got, s, inverse=True)
    f = lambda z: (plain.turn(z, tab.double(), pairing) * g.double()).sum()
    z = x.double().requires_grad_(True)
    want, = torch.autograd.grad(f(z), z)
    assert float((got.double() - want).abs().max()) <= 1e-5
    step = torch.zeros_like(z)
    step[1, 2, 3, 5] = step[0, 1, 9, 40] = 1e-3
    slope = (f(x.double() + step) - f(x.double() - step)) / 2
    assert abs(float(slope) - 1e-3 * float(got[1, 2, 3, 5] + got[0, 1, 9, 40])) <= 1e-8


def test_far_positions_keep_their_angles():
    """Differences of positions near 2^30 turn like small ones: the products of turned rows agree."""
    T, D = 8, 64
    rope = amskv.Rope(rot_dim=D)
    near = torch.arange(T, dtype=torch.float64, device="cuda")[:, None]
    q, k = _normal(1, 1, T, D, seed=1), _normal(1, 1, T, D, seed=2)
    s = amskv.Strides(T * D, T * D, D)
    scores = []
    for first in (0.0, float(2 ** 30)):
        tab = _table(rope, near + first)
        outs = []
        for x in (q, k):
            o = torch.empty_like(x)
            amskv.amskv_rotate(rope, amskv.AMSKV_DTYPE_F32, D, 1, 1, T, tab, 0, x, s, o, s)
            outs.append(o.double())
        scores.append(outs[0] @ outs[1].transpose(-1, -2))
    size = q.double().abs() @ k.double().abs().transpose(-1, -2)
    # per product: two turned factors, each off by 4 * 2^-24, twice; and 2^30 * 2^-53 * 2 pi of angle
    assert bool(((scores[0] - scores[1]).abs() <= size.amax() * (32 * F32 + 2.0 ** -20)).all())


SIDES = (1, 2, 3, 5, 7)


def _run_cache(dtype, D, pairing, rot, packed, policy, B=2, H=3, seed=0, q_apart=False, **kw):
    """One layer through the schedule with turned appends and attention; yields per step (turned q, k as the cache should hold them, v, out,
    what is left of K's buffer) and at the end the read-back cache."""
    dt = torch.float32 if dtype == amskv.AMSKV_DTYPE_F32 else torch.bfloat16
    mode = {x: kw.pop(x) for x in ("budgets", "windows") if x in kw}
    args = (1, H, D, SIDES, SIDES, B, dtype, None if mode else [policy])
    arena = torch.empty(amskv.amskv_cache_required_bytes(*args, **kw, **mode), dtype=torch.uint8, device="cuda").fill_(0xFF)
    h = amskv.amskv_cache_create(*args, arena=arena, **kw, **mode)
    rope = amskv.Rope(rot_dim=rot, pairing=_pairing(pairing), axes=2)
    width = H * D
    steps = []
    try:
        if packed:
            amskv.amskv_cache_set_io_layout(h, amskv.AMSKV_IO_TOKEN_MAJOR, width if q_apart else 3 * width, 3 * width, width)
        for s, side in enumerate(SIDES):
            T = side * side
            t = torch.arange(T, device="cuda")
            tab = _table(rope, torch.stack((t // side, t % side), dim=1).double() * (SIDES[-1] / side))
            q, k, v = (_normal(B, H, T, D, seed=seed + 10 * s + i).to(dt) for i in range(3))
            want_q, want_k = (plain.turn(x.float(), tab, pairing) for x in (q, k))
            if packed:
                x = torch.stack((q, k, v)).permute(1, 3, 0, 2, 4).reshape(B, T, 3, width).contiguous()
                qd, kd, vd = x[:, :, 0], x[:, :, 1], x[:, :, 2]
                out = torch.empty(B, T, width, dtype=dt, device="cuda")
                turned = torch.empty(B, T, width, dtype=dt, device="cuda") if q_apart else qd
                amskv.amskv_append_scale_rotary(h, 0, s, rope, tab, qd, 3 * width if q_apart else 0, turned, kd, vd)
                amskv.amskv_attend(h, 0, s, turned, out)
                heads = lambda y: y.reshape(B, T, H, D).transpose(1, 2)
                steps.append((heads(turned).clone(), want_q, want_k, v, heads(out), heads(kd).clone(), k, x))
            else:
                kd, out, turned = k.clone(), torch.empty_like(q), torch.empty_like(q)
                amskv.amskv_append_scale_rotary(h, 0, s, rope, tab, q, 0, turned, kd, v)
                amskv.amskv_attend(h, 0, s, turned, out)
                steps.append((turned, want_q, want_k, v, out, kd.clone(), k, kd))
        segs = amskv.amskv_cache_segments(h, 0)
        n = sum(x[3] for x in segs)
        ko, vo = (torch.empty(B, H, n, D, dtype=dt, device="cuda") for _ in range(2))
        amskv.amskv_cache_export(h, 0, ko, vo)
        torch.cuda.synchronize()
    finally:
        amskv.amskv_cache_destroy(h)
    return steps, segs, ko, vo


KINDS = {"f32": amskv.AMSKV_DTYPE_F32, "bf16": amskv.AMSKV_DTYPE_BF16, "8 bits": amskv.AMSKV_DTYPE_BF16_KV8}


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("D,rot", [(64, 64), (128, 96), (64, 16)])
@pytest.mark.parametrize("pairing", ["half", "interleaved"])
@pytest.mark.parametrize("packed", ["", "in place", "apart"])
@pytest.mark.parametrize("policy", [(2, 1, False), (0, 0, True)], ids=["window", "all"])
def test_append_copying(kind, D, rot, pairing, packed, policy):
    """Turned queries, the cache's contents and the attention over them; K's buffer stays."""
    steps, segs, ko, vo = _run_cache(KINDS[kind], D, pairing, rot, bool(packed), policy, q_apart=packed == "apart")
    as_held = plain.held if kind == "8 bits" else (lambda x: x.to(torch.float32 if kind == "f32" else torch.bfloat16).double())
    kept = {}
    for s, (turned, want_q, want_k, v, out, k_after, k, _) in enumerate(steps):
        assert torch.equal(turned, want_q.to(turned.dtype))
        assert torch.equal(k_after, k)
        kept[s] = as_held(want_k), as_held(v)
        c, w, everything = policy
        now = [i for i in range(s + 1) if everything or i < c or s - i <= w]
        kk, vv = (torch.cat([kept[i][j] for i in now], dim=2) for j in range(2))
        o, bound = plain.attention(turned, kk, vv, 1 / math.sqrt(D))
        if kind != "f32":
            assert bool(((out.double() - o).abs() <= bound).all())
        else:
            assert float((out.double() - o).abs().max()) <= 1e-4
    assert torch.equal(ko.double(), kk) and torch.equal(vo.double(), vv)


@pytest.mark.parametrize("kw", [dict(layout=amskv.AMSKV_LAYOUT_PLANNED, borrow_unretained=True, fuse_append=True),
                                dict(borrow_unretained=True), dict(fuse_append=True), dict(budgets=[(20, 40, 5, 2.0)]), dict(windows=[(30, 5)])],
                         ids=["all in place", "borrow", "fuse", "budget", "window"])
@pytest.mark.parametrize("packed", [False, True])
def test_append_in_place(kw, packed):
    """Where the scale is read in place K is turned in its own buffer; nothing else changes there."""
    steps, segs, ko, vo = _run_cache(amskv.AMSKV_DTYPE_BF16, 64, "half", 48, packed, (1, 1, False), **dict(kw))
    at = 0
    for s, (turned, want_q, want_k, v, out, k_after, k, buffer) in enumerate(steps):
        assert torch.equal(turned, want_q.bfloat16())
        in_place = bool(kw.get("fuse_append") or "budgets" in kw or "windows" in kw or (kw.get("borrow_unretained") and s == len(steps) - 1))
        assert torch.equal(k_after, want_k.bfloat16() if in_place else k)
        if packed:
            assert torch.equal(buffer[:, :, 2].reshape(*v.transpose(1, 2).shape).transpose(1, 2), v)
    for scale, first, _, n in segs:
        assert torch.equal(ko[:, :, at:at + n], steps[scale][2].bfloat16()[:, :, first:first + n])
        assert torch.equal(vo[:, :, at:at + n], steps[scale][3][:, :, first:first + n])
        at += n


def test_keys_only():
    B, H, D = 1, 2, 64
    args = (1, H, D, (3,), (4,), B, amskv.AMSKV_DTYPE_BF16_KV8, [(0, 0, True)])
    arena = torch.empty(amskv.amskv_cache_required_bytes(*args), dtype=torch.uint8, device="cuda")
    h = amskv.amskv_cache_create(*args, arena=arena)
    try:
        rope = amskv.Rope(rot_dim=64)
        tab = _table(rope, torch.arange(12, device="cuda").double()[:, None])
        k, v = _normal(B, H, 12, D, seed=1).bfloat16(), _normal(B, H, 12, D, seed=2).bfloat16()
        amskv.amskv_append_scale_rotary(h, 0, 0, rope, tab, None, 0, None, k, v)
        ko, vo = torch.empty_like(k), torch.empty_like(v)
        amskv.amskv_cache_export(h, 0, ko, vo)
        assert torch.equal(ko.double(), plain.held(plain.turn(k.float(), tab, "half"))) and torch.equal(vo.double(), plain.held(v))
    finally:
        amskv.amskv_cache_destroy(h)
