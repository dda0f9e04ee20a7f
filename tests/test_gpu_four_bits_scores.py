"""Scores of the attentions over K and V in 4 bits where they are hard to keep, in every form that a launch takes: the shapes
below reach all of them, which test_four_bits_scores_choice.py asks of the code that chooses."""
import math

import pytest
import torch

import paper_2511_16047_amd as amskv
import plain_four_bits as plain
import plain_operators
from test_gpu_cache_in_4_bits import EVEN, Cache, _normal
from test_gpu_held_states import Case

pytestmark = pytest.mark.gpu

# head dim -> (B, H, tokens before, queries) of a step over a cache
STEPS = {64: [(1, 4, 48, 3), (1, 4, 64, 60), (1, 4, 840, 60), (8, 16, 48, 225), (8, 16, 64, 257), (4, 16, 300, 520)],
         128: [(1, 4, 48, 3), (1, 4, 64, 60), (1, 4, 840, 60), (4, 16, 48, 257), (4, 16, 300, 400), (4, 16, 64, 520)]}
# head dim -> (B, kv heads, queries, states) of a call over held states
CALLS = {64: [(1, 1, 1, 20), (1, 4, 3, 150), (1, 4, 3, 1100), (2, 2, 1, 5000), (10, 15, 260, 600), (8, 16, 257, 557)],
         128: [(1, 1, 1, 20), (1, 4, 3, 150), (1, 4, 60, 600), (1, 4, 3, 1100), (4, 16, 260, 150), (8, 16, 257, 557)]}
steps = pytest.mark.parametrize("D,shape", [(d, x) for d in STEPS for x in STEPS[d]], ids=str)
calls = pytest.mark.parametrize("D,shape", [(d, x) for d in CALLS for x in CALLS[d]], ids=str)


def _coarse(*shape, seed):
    """Numbers of few bits."""
    return torch.round(_normal(*shape, seed=seed)).clamp(-2, 2)


def _lost(q, k):
    """Most that a score (of one head, q [Tq, D], k [Tk, D], times the scale still to come) may lose in launches of many rows.

    32 channels of Q with largest element m are numbers of 8 bits times 2^a, 224 * 2^a < m <= 448 * 2^a, in two parts of 4 significant
    bits: exact down to 2^-6 * 2^a, below off by 2^-14 * 2^a at most, which is less than 2^-21.8 m.  The products of 8 channels are cut to
    units of 2^-13 of the power of two of the largest.  Q's larger part is off by 2^-4 of q at most, so with P the largest |q k| the unit is at most U =
    2^-13 * 2^floor(log2(17/16 P)), and a product, of 4 + 2 bits, that is 32 U or more is a multiple of it: what is lost is at most min(U, 17/16
    |q k|) where 15/16 |q k| < 32 U.  The smaller part is at most 2^-4 q, its unit U / 16: 7 of those."""
    m = q.unflatten(-1, (-1, 32)).abs().amax(dim=-1, keepdim=True).expand(-1, -1, 32).flatten(-2)
    off = torch.where(q.abs() < m * (2.0 ** -6 / 224), m * 2.0 ** -21.8, torch.zeros_like(m)) @ k.abs().T
    for i in range(0, q.shape[-1], 8):
        p = (q[:, None, i:i + 8] * k[None, :, i:i + 8]).abs()
        unit = torch.exp2(torch.floor(torch.log2(p.amax(dim=-1, keepdim=True) * (17 / 16) + 1e-300)) - 13)
        off += torch.where(p * (15 / 16) < 32 * unit, torch.minimum(p * (17 / 16), unit), torch.zeros_like(p)).sum(dim=-1) + 7 / 16 * unit[..., 0]
    return off


def _check(out, q, k, v, scale, what=""):
    """[..., T, D] against the formula with Q as it is; scores may be off by _lost(), and weights of 2^-120 of the largest and less may
    vanish (plain_four_bits.attention).  With weights p_j e^d_j, |d_j| <= e_j, in both sums O is off by at most sum p_j |e^d_j - 1| |v_j - o| / sum
    p_j e^d_j <= e^max(e) sum p_j (e^e_j - 1) (|v_j| + |o|)."""
    out, q, k, v = (x.double().flatten(0, -3) for x in (out, q, k, v))
    for i in range(len(q)):
        o, bound = plain_operators.attention(q[i], k[i], v[i], scale)
        e = _lost(q[i], k[i]) * scale
        s = q[i] @ k[i].T * scale
        p, rel = torch.softmax(s, dim=-1), torch.exp(s - s.amax(dim=-1, keepdim=True))
        w = p * torch.expm1(e) * torch.exp(e.amax(dim=-1, keepdim=True))
        bound = bound * torch.exp(e.amax(dim=-1, keepdim=True)) + w @ v[i].abs() + w.sum(dim=-1, keepdim=True) * o.abs()
        bound = bound + torch.where(rel <= 1.01 * 2.0 ** -120, p, torch.zeros_like(p)) @ v[i].abs()
        off = (out[i] - o).abs()
        assert bool((off <= bound).all()), "%s, %d: %.3e of the bound" % (what, i, float((off / bound).nan_to_num(math.inf).max()))


def _step(D, B, H, before, queries, q, k, v, borrow, scale=0.0):
    """k, v: of both scales.  The second one's output, and K and V as its attention has them."""
    with Cache([(1, before), (1, queries)], B, H, D, [(0, 0, True)], borrow_unretained=borrow, softmax_scale=scale) as c:
        o = torch.full_like(q, 9.0)
        for s in range(2):
            amskv.amskv_append_scale(c.h, 0, s, k[s], v[s])
        amskv.amskv_attend(c.h, 0, 1, q, o)
        held = [[plain.held(x[0]), x[1].double() if borrow else plain.held(x[1])] for x in (k, v)]
        return o, held[0], held[1]


# ---------------------------------------------------------------- a reference that moves far
@steps
@pytest.mark.parametrize("far", [2.0 ** 10, 2.0 ** 30, 2.0 ** 60, 2.0 ** 100])
@pytest.mark.parametrize("borrow", [False, True])
def test_scores_behind_far_lower_ones(D, shape, far, borrow):
    """The first scale's scores are some -far^2; the second's come out as if alone.  (With queries of few bits.)"""
    B, H, before, queries = shape
    k = [_normal(B, H, n, D, seed=n).bfloat16() for n in (before, queries)]
    v = [_normal(B, H, n, D, seed=n + 1).bfloat16() for n in (before, queries)]
    q = _coarse(B, H, queries, D, seed=5).bfloat16()
    q[..., :32] = 0
    q[..., 0], k[0][..., 0], k[1][..., :32] = far, -far, 0
    o, kk, vv = _step(D, B, H, before, queries, q, k, v, borrow, EVEN)
    _check(o, q, kk[1], vv[1], EVEN, "far below")


@calls
@pytest.mark.parametrize("far", [2.0 ** 10, 2.0 ** 30, 2.0 ** 60, 2.0 ** 100])
def test_held_scores_behind_far_lower_ones(D, shape, far):
    """The same over held states: the first third of every length is far below."""
    B, H, queries, keys = shape
    lengths = [max(2, keys - 17 * b) for b in range(B)]
    c = Case(H, H, D, queries, keys, lengths, sharp=2.0, hold=False)
    c.q[..., :32] = 0
    c.q[..., 0] = far
    for b, n in enumerate(lengths):
        c.k[b, :n, :, :32] = 0
        c.k[b, :n // 3, :, 0] = -far
    c.hold()
    out = c.run()
    for b, n in enumerate(lengths):
        k, v = (plain.held(x[b, n // 3:n]).transpose(0, 1) for x in (c.k, c.v))
        _check(out[b], c.q[b], k, v, EVEN, "%d states" % n)


# ---------------------------------------------------------------- queries that are not finite
def _spoilt(q):
    """Rows with one channel that is NaN or infinite, and which they are."""
    q, spoilt = q.clone(), torch.zeros(q.shape[:-1], dtype=torch.bool, device="cuda")
    D, flat, rows = q.shape[-1], q.view(-1, q.shape[-1]), spoilt.view(-1)
    for i, x in enumerate((math.nan, math.inf, -math.inf)):
        for j, row in enumerate((i, len(flat) // 2 + i, len(flat) - 1 - i)):
            flat[row % len(flat), (7 * j + 33 * i) % D], rows[row % len(flat)] = x, True
    return q, spoilt


# The reference of a row moves when any row of its wave asks for it (a score more than 2^6 above it is taken as it is while the sum stays
# below 2^10), so the other rows need not be the same bits: they are as near to the formula as ever.
def _check_rest(out, rows, q, k, v):
    want, bound = plain.attention(q.masked_fill(rows[..., None], 0.0), k, v, 1 / math.sqrt(q.shape[-1]))
    assert bool(torch.isnan(out[rows]).all()) and bool(((out.double() - want).abs() <= bound)[~rows].all())


@steps
@pytest.mark.parametrize("borrow", [False, True])
def test_queries_that_are_not_finite(D, shape, borrow):
    """A row with a channel that is not finite comes out as NaN in every form, and no other row does."""
    B, H, before, queries = shape
    k, v = ([_normal(B, H, n, D, seed=n + i).bfloat16() for n in (before, queries)] for i in range(2))
    q, rows = _spoilt(_normal(B, H, queries, D, seed=5).bfloat16())
    out, k, v = _step(D, B, H, before, queries, q, k, v, borrow)
    _check_rest(out, rows, q, *(torch.cat(x, dim=2) for x in (k, v)))


@calls
def test_held_states_and_queries_that_are_not_finite(D, shape):
    B, H, queries, keys = shape
    c = Case(H, H, D, queries, keys, [max(1, keys - 17 * b) for b in range(B)])
    c.q, rows = _spoilt(c.q)
    out = c.run()
    for b, n in enumerate(c.lengths):
        _check_rest(out[b], rows[b], c.q[b], *(plain.held(x[b, :n]).transpose(0, 1) for x in c.kv))


# ---------------------------------------------------------------- queries as they come
def _queries(kind, *shape):
    """Q, and what K's channels are taken by: scores of a standard deviation of 20; a channel of Q 30 and 300 times the others, whose
    keys are as much smaller, scores of 8; channels of every size down to 2^-24, each with a random one in full."""
    x, D = _normal(*shape, seed=11), shape[-1]
    gain = torch.ones(D, device="cuda")
    if kind == "sharp":
        return (20 * x).bfloat16(), gain
    if kind.startswith("outlier"):
        gain[5], gain[D - 20] = float(kind[7:]), float(kind[7:])
        return (8 * x * gain).bfloat16(), 1 / gain
    size = 2.0 ** (-24 * torch.rand(*shape, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda"))
    return (x * size).bfloat16(), gain


KINDS = ["sharp", "outlier30", "outlier300", "wide"]


@steps
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("borrow", [False, True])
def test_queries_as_they_come(D, shape, kind, borrow):
    B, H, before, queries = shape
    q, by = _queries(kind, B, H, queries, D)
    k = [(_normal(B, H, n, D, seed=n) * by).bfloat16() for n in (before, queries)]
    v = [_normal(B, H, n, D, seed=n + 1).bfloat16() for n in (before, queries)]
    o, k, v = _step(D, B, H, before, queries, q, k, v, borrow)
    _check(o, q, torch.cat(k, dim=2), torch.cat(v, dim=2), 1 / math.sqrt(D), kind)


@calls
@pytest.mark.parametrize("kind", KINDS)
def test_held_states_and_queries_as_they_come(D, shape, kind):
    B, H, queries, keys = shape
    c = Case(H, H, D, queries, keys, [max(1, keys - 17 * b) for b in range(B)], spoil=False, hold=False)
    c.q, by = _queries(kind, B, H, queries, D)
    c.k *= by
    c.hold()
    out = c.run()
    for b, n in enumerate(c.lengths):
        k, v = (plain.held(x[b, :n]).transpose(0, 1) for x in (c.k, c.v))
        _check(out[b], c.q[b], k, v, 1 / math.sqrt(D), "%s, %d states" % (kind, n))


@pytest.mark.parametrize("D", [64, 128])
def test_a_row_is_the_same_in_every_form(D):
    """Rows of one query at a time (waves by themselves) and of all (teams): each within the bound of Q as it is."""
    B, H, queries, keys = (8, 16, 257, 557)
    c = Case(H, H, D, queries, keys, [keys] * B, spoil=False, hold=False)
    c.q, by = _queries("outlier300", B, H, queries, D)
    c.k *= by
    c.hold()
    many = c.run()
    q, c.x.q_tokens = c.q, 1
    few = torch.empty_like(q[:, :, :1])
    c.x.o = amskv.Strides(H * D, D, D)
    for row in (0, 100, 256):
        amskv.amskv_cross_attend(c.x, q[:, :, row:].data_ptr(), *c.held, few)
        k, v = (plain.held(x).transpose(1, 2) for x in (c.k, c.v))
        for o in (few, many[:, :, row:row + 1]):
            _check(o, q[:, :, row:row + 1], k, v, 1 / math.sqrt(D), "row %d" % row)
