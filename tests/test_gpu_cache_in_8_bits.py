"""The cache in 8 bits: what it holds, code by code, and the attention over it, against the definitions in 64 bits."""
import math

import pytest
import torch

import paper_2511_16047_amd as amskv
import plain_operators as plain

pytestmark = pytest.mark.gpu
COMPACT, PLANNED = amskv.AMSKV_LAYOUT_COMPACT, amskv.AMSKV_LAYOUT_PLANNED


def _normal(*shape, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda")


class Cache:
    def __init__(self, sides, B, H, D, pols, **kw):
        hs, ws = zip(*sides)
        args = (len(pols), H, D, hs, ws, B, amskv.AMSKV_DTYPE_BF16_KV8, pols)
        need = amskv.amskv_cache_required_bytes(*args, **kw)
        self.arena = torch.empty(need + 256, dtype=torch.uint8, device="cuda").fill_(0xFF)   # codes of NaN wherever nothing was put
        self.h = amskv.amskv_cache_create(*args, arena=self.arena, arena_bytes=need, **kw)
        self.B, self.H, self.D, self.need = B, H, D, need

    def __enter__(self):
        return self

    def __exit__(self, *a):
        torch.cuda.synchronize()
        assert bool((self.arena[self.need:] == 0xFF).all())
        amskv.amskv_cache_destroy(self.h)

    def read(self, layer):
        n = sum(x[2] for x in amskv.amskv_cache_layout(self.h, layer))
        k, v = (torch.full((self.B, self.H, n, self.D), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        amskv.amskv_cache_export(self.h, layer, k, v)
        return k, v


def _hold(x):
    """x [B, H, T, D] bf16 through a one-scale cache."""
    with Cache([(1, x.shape[2])], x.shape[0], x.shape[1], x.shape[3], [(0, 0, True)]) as c:
        amskv.amskv_append_scale(c.h, 0, 0, x, x.flip(-1).contiguous())
        k, v = c.read(0)
        assert torch.equal(v.flip(-1), k)      # a block's scale does not depend on the order of its channels
        return k


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T", [1, 2, 3, 5, 8, 9, 15, 16, 17, 31, 64, 100])
def test_held_values(D, T):
    x = (_normal(2, 5, T, D, seed=T) * torch.exp(3 * _normal(2, 5, T, 1, seed=1))).bfloat16()
    got = _hold(x)
    assert torch.equal(got.double(), plain.held(x))
    top = torch.stack([b.abs().amax(dim=(-1, -2)) for b in x.double().split(16, dim=2)], dim=2)          # 2^-4 of a value, 2^-18 of the block's largest
    top = top.repeat_interleave(16, dim=2)[:, :, :T, None]
    assert bool(((got.double() - x.double()).abs() <= 2.0 ** -4 * x.double().abs() + 2.0 ** -17 * top).all())


def test_every_code_and_every_midpoint():
    """All e4m3 numbers and the bf16 numbers at and beside the middle between two, under a largest element of 448."""
    n = torch.tensor(plain.e4m3_numbers(), dtype=torch.float64)
    mid = (n[1:] + n[:-1]) / 2
    x = torch.cat([n, mid, mid * (1 + 2.0 ** -7), mid * (1 - 2.0 ** -7), torch.tensor([448.0], dtype=torch.float64)])
    x = torch.cat([x, -x, torch.zeros(16 * 64 - 2 * len(x), dtype=torch.float64)]).bfloat16().cuda().view(1, 1, 16, 64)
    for e in (-90, -20, 0, 7, 100):
        y = (x.double() * 2.0 ** e).bfloat16()
        got = _hold(y)
        assert torch.equal(got.double(), plain.held(y))
        assert torch.equal(got.double()[y.double() == 448 * 2.0 ** e], y.double()[y.double() == 448 * 2.0 ** e])


def test_ends_of_the_range():
    """Blocks of zeros, of the smallest and of the largest bf16 numbers; largest elements at and just above 448 times a power."""
    big = torch.finfo(torch.bfloat16).max
    tops = [0.0, 2.0 ** -133, 2.0 ** -126, 2.0 ** -112, 2.0 ** -100, 448.0, 450.0, 1.75, 1.7578125, 2.0, 448 * 2.0 ** 90, big]
    x = torch.zeros(1, len(tops), 16, 64, dtype=torch.float64, device="cuda")
    for i, m in enumerate(tops):
        x[0, i] = m * torch.linspace(-1, 1, 16 * 64, dtype=torch.float64, device="cuda").view(16, 64)
        x[0, i, 3, 3] = m
    y = x.bfloat16()
    got = _hold(y).double()
    assert torch.equal(got, plain.held(y))
    assert bool((got[0, 0] == 0).all()) and bool((got[0, 1] == 0).all()) and bool(torch.isfinite(got[0, -2]).all())


def _attended(c, layer, steps, pol, borrow=False):
    """The steps of one layer: (q, k, v, out) per scale, checked against what the cache should hold."""
    held = {}
    for s, (q, k, v, out) in enumerate(steps):
        cpol, w, everything = pol
        now = [i for i in range(s + 1) if everything or i < cpol or s - i <= w]
        later = s + 1 < len(steps) and (everything or s < cpol or w > 0)
        held[s] = (k.double(), v.double()) if borrow and not later else (plain.held(k), plain.held(v))
        kk, vv = (torch.cat([held[i][j] for i in now], dim=2) for j in range(2))
        o, bound = plain.attention(q, kk, vv, 1 / math.sqrt(q.shape[-1]))
        off = (out.double() - o).abs()
        assert bool((off <= bound).all()), "scale %d, %d x %d: %.3e of %.3e" % (s, q.shape[2], kk.shape[2], float((off / bound).max()), 1.0)
    return kk, vv


def _drive(sides, B, H, D, pols, seed=0, packed=False, sharp=1.0, **kw):
    with Cache(sides, B, H, D, pols, **kw) as c:
        width = H * D
        if packed:
            amskv.amskv_cache_set_io_layout(c.h, amskv.AMSKV_IO_TOKEN_MAJOR, 3 * width, 3 * width, width)
        layers = [[] for _ in pols]
        alive = []
        for s, (a, b) in enumerate(sides):
            T = a * b
            for l in range(len(pols)):
                q, k, v = (_normal(B, H, T, D, seed=seed + 1000 * l + 10 * s + i) for i in range(3))
                q, k, v = (q * sharp).bfloat16(), (k * torch.exp(_normal(H, 1, D, seed=5))).bfloat16(), v.bfloat16()
                if packed:
                    x = torch.stack((q, k, v)).permute(1, 3, 0, 2, 4).reshape(B, T, 3, width).contiguous()
                    o = torch.full((B, T, width), 9.0, dtype=torch.bfloat16, device="cuda")
                    amskv.amskv_append_scale(c.h, l, s, x[:, :, 1], x[:, :, 2])
                    amskv.amskv_attend(c.h, l, s, x[:, :, 0], o)
                    o = o.view(B, T, H, D).transpose(1, 2)
                    alive.append(x)
                else:
                    o = torch.full((B, H, T, D), 9.0, dtype=torch.bfloat16, device="cuda")
                    amskv.amskv_append_scale(c.h, l, s, k, v)
                    amskv.amskv_attend(c.h, l, s, q, o)
                layers[l].append((q, k, v, o))
        for l, pol in enumerate(pols):
            kk, vv = _attended(c, l, layers[l], pol, kw.get("borrow_unretained", False))
            ko, vo = c.read(l)
            assert torch.equal(ko.double(), kk) and torch.equal(vo.double(), vv)


VAR = [(s, s) for s in (1, 2, 3, 4, 5, 6, 8, 10, 13, 16)]


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", [COMPACT, PLANNED], ids=["compact", "planned"])
@pytest.mark.parametrize("borrow", [False, True])
@pytest.mark.parametrize("packed", [False, True])
def test_ten_scales(D, layout, borrow, packed):
    _drive(VAR, 2, 3, D, [(2, 2, False), (0, 0, True), (1, 0, False)], packed=packed, layout=layout, borrow_unretained=borrow)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("queries", [1, 7, 31, 32, 33, 63, 64, 65, 128, 129, 255, 256, 257, 300, 520])
@pytest.mark.parametrize("before", [0, 1, 15, 16, 31, 33, 64, 500])
def test_lengths(D, queries, before):
    """Any number of queries behind any number of cached tokens, the step's own keys cached and read in place."""
    sides = ([(1, before)] if before else []) + [(1, queries)]
    for borrow in (False, True):
        _drive(sides, 1, 3, D, [(0, 0, True)], seed=queries + before, borrow_unretained=borrow)


@pytest.mark.parametrize("D", [64, 128])
def test_shrinking_and_odd_grids(D):
    _drive([(5, 7), (1, 1), (17, 3), (2, 2), (9, 31), (1, 1), (3, 1)], 2, 5, D, [(1, 2, False), (0, 1, False), (3, 1, False)])


@pytest.mark.parametrize("B,H", [(1, 1), (3, 11), (40, 17), (130, 16)])
def test_units(B, H):
    """From one (b,h) to more than the chip has places for."""
    _drive([(1, 1), (3, 3), (6, 6), (13, 13)], B, H, 64, [(1, 1, False)], borrow_unretained=True)
    _drive([(2, 2), (10, 10)], B, H, 128, [(0, 0, True)])


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,H,queries", [(10, 15, 65), (10, 15, 100), (10, 15, 128), (10, 15, 150), (10, 15, 225), (10, 15, 256), (13, 10, 257),
                                         (4, 15, 300), (5, 15, 500)])
@pytest.mark.parametrize("before", [0, 1, 16, 30, 33, 64, 95, 200])
def test_many_units_of_many_rows(D, B, H, queries, before):
    """Enough rows for waves that share K and V: any number of tiles of codes, of rows, of both, and rows left over in each."""
    sides = ([(1, before)] if before else []) + [(1, queries)]
    for borrow in (False, True):
        _drive(sides, B, H, D, [(0, 0, True)], seed=queries + before, borrow_unretained=borrow)
    if before:
        _drive(sides, B, H, D, [(1, 0, False)], seed=queries, borrow_unretained=True)      # codes, then rows read in place


@pytest.mark.parametrize("before", [799, 831, 840])
def test_many_units_over_many_tokens(before):
    for borrow in (False, True):
        _drive([(1, before), (1, 225)], 17, 16, 128, [(1, 0, False)], seed=before, borrow_unretained=borrow)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", [COMPACT, PLANNED], ids=["compact", "planned"])
@pytest.mark.parametrize("packed", [False, True])
def test_many_units_of_short_segments(D, layout, packed):
    _drive([(1, 1), (1, 2), (1, 3), (4, 4), (1, 5), (1, 1), (6, 6), (9, 20), (15, 20)], 10, 15, D, [(3, 3, False), (0, 6, False)], packed=packed,
           layout=layout, borrow_unretained=True)


@pytest.mark.parametrize("sharp", [0.0, 20.0, 300.0])
def test_sharp_scores_of_many_units(sharp):
    _drive([(4, 4), (10, 10), (16, 16)], 10, 15, 64, [(0, 0, True)], sharp=sharp)
    _drive([(4, 4), (10, 10), (16, 16)], 10, 15, 128, [(2, 0, False)], sharp=sharp, borrow_unretained=True)


@pytest.mark.parametrize("sharp", [0.0, 20.0, 300.0])
def test_flat_and_sharp_scores(sharp):
    """Uniform weights; a few keys that take everything, at the start and the end of long key runs."""
    _drive([(4, 4), (10, 10), (16, 16)], 1, 4, 64, [(0, 0, True)], sharp=sharp)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,queries", [(2, 5), (16, 60), (150, 100), (150, 256)])
@pytest.mark.parametrize("first", [32, 48, 64])
def test_scores_beyond_fp32_weigh_nothing(D, H, queries, first):
    """A whole scale whose scores are -inf in fp32 (2^100 times -2^100), then keys as if alone: codes, and rows read in place."""
    for borrow in (False, True):
        with Cache([(1, first), (1, queries)], 1, H, D, [(0, 0, True)], borrow_unretained=borrow) as c:
            k0, v0 = (_normal(1, H, first, D, seed=i).bfloat16() for i in (1, 2))
            q, k, v = (_normal(1, H, queries, D, seed=i).bfloat16() for i in (3, 4, 5))
            q[..., 0], k0[..., 0], k[..., 0] = 2.0 ** 100, -2.0 ** 100, 0
            o = torch.empty_like(q)
            amskv.amskv_append_scale(c.h, 0, 0, k0, v0)
            amskv.amskv_append_scale(c.h, 0, 1, k, v)
            amskv.amskv_attend(c.h, 0, 1, q, o)
            kk, vv = (x.double() if borrow else plain.held(x) for x in (k, v))
            want, bound = plain.attention(q, kk, vv, 1 / math.sqrt(D))
            assert bool(((o.double() - want).abs() <= bound).all())


def test_many_tokens():
    """Offsets of codes and of a layer's regions beyond 2^31 bytes."""
    B, H, D, T = 24, 16, 128, 45000
    with Cache([(1, T), (1, 3)], B, H, D, [(1, 0, False)]) as c:
        assert B * H * T * D > 2 ** 31
        g = torch.Generator(device="cuda")
        g.manual_seed(1)
        k = torch.empty(B, H, T, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        v = torch.empty(B, H, T, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
        amskv.amskv_append_scale(c.h, 0, 0, k, v)
        q, k1, v1 = (_normal(B, H, 3, D, seed=i).bfloat16() for i in range(3))
        o = torch.empty_like(q)
        amskv.amskv_append_scale(c.h, 0, 1, k1, v1)
        amskv.amskv_attend(c.h, 0, 1, q, o)
        for b, h in ((0, 0), (11, 3), (B - 1, H - 1)):
            kk, vv = (torch.cat([plain.held(x[b, h]), plain.held(y[b, h])], dim=0) for x, y in ((k, k1), (v, v1)))
            want, bound = plain.attention(q[b, h], kk, vv, 1 / math.sqrt(D))
            assert bool(((o[b, h].double() - want).abs() <= bound).all())


def test_same_bits_again():
    """Two caches, filled and attended in turn on two streams, give the same bits as one after the other."""
    sides, B, H, D = [(4, 4), (9, 9), (16, 16)], 3, 8, 64
    data = [[_normal(B, H, a * b, D, seed=10 * s + i).bfloat16() for i in range(3)] for s, (a, b) in enumerate(sides)]
    outs = []
    streams = [torch.cuda.Stream() for _ in range(2)]
    with Cache(sides, B, H, D, [(1, 1, False)]) as one, Cache(sides, B, H, D, [(1, 1, False)]) as two:
        torch.cuda.synchronize()
        for s, (q, k, v) in enumerate(data):
            for c, st in zip((one, two), streams):
                o = torch.empty_like(q)
                torch.cuda.synchronize()
                amskv.amskv_append_scale(c.h, 0, s, k, v, stream=st)
                amskv.amskv_attend(c.h, 0, s, q, o, stream=st)
                outs.append(o)
        torch.cuda.synchronize()
        for a, b in zip(outs[::2], outs[1::2]):
            assert torch.equal(a, b)


@pytest.mark.parametrize("layout", [COMPACT, PLANNED], ids=["compact", "planned"])
def test_a_captured_image(layout):
    """Captured once, replayed with new inputs and eager work in between."""
    B, H, D, pols = 2, 4, 64, [(1, 1, False), (0, 0, True)]
    rope = amskv.Rope(rot_dim=32, axes=2)
    with Cache(VAR, B, H, D, pols, layout=layout) as c, Cache(VAR, B, H, D, pols, layout=layout) as eager:
        bufs = [[[torch.empty(B, H, a * b, D, dtype=torch.bfloat16, device="cuda") for _ in range(5)] for a, b in VAR] for _ in pols]
        tabs = []
        for a, b in VAR:
            t = torch.arange(a * b, device="cuda")
            tab = torch.empty(a * b, 16, 2, device="cuda")
            amskv.amskv_rope_table(rope, torch.stack((t // b, t % b), dim=1).double(), tab)
            tabs.append(tab)

        def image(h, out, stream=None):
            amskv.amskv_cache_reset(h)
            for s in range(len(VAR)):
                for l in range(len(pols)):
                    q, k, v, turned, o = bufs[l][s]
                    amskv.amskv_append_scale_rotary(h, l, s, rope, tabs[s], q, 0, turned, k, v, stream=stream)
                    amskv.amskv_attend(h, l, s, turned, out[l][s], stream=stream)

        def fill(seed):
            for l in range(len(pols)):
                for s in range(len(VAR)):
                    for i in range(3):
                        bufs[l][s][i].copy_(_normal(*bufs[l][s][i].shape, seed=seed + 100 * l + 10 * s + i))

        out = [[b[4] for b in layer] for layer in bufs]
        apart = [[torch.empty_like(b[4]) for b in layer] for layer in bufs]
        fill(1)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            image(c.h, out)
        for seed in (1, 5000, 9000):
            fill(seed)
            for layer in out:
                for o in layer:
                    o.fill_(3.0)
            graph.replay()
            image(eager.h, apart)
            torch.cuda.synchronize()
            for a, b in zip(out, apart):
                assert all(torch.equal(x, y) for x, y in zip(a, b))
