"""Calls of the operators that really run at the same time: everything is enqueued on both streams while they wait behind one long piece of
work, and every result is that of the same calls one after the other."""
import pytest
import torch

import paper_2511_16047_amd as amskv
from test_gpu_cache_in_8_bits import Cache
from test_gpu_cross_attention import Case

pytestmark = pytest.mark.gpu


class Gate:
    """Work that other streams wait for: some 5 ms of products."""

    def __init__(self):
        self.stream = torch.cuda.Stream()
        self.a = torch.randn(8192, 8192, device="cuda")
        self.b = torch.empty_like(self.a)
        torch.mm(self.a, self.a, out=self.b)       # (the library settles before)
        torch.cuda.synchronize()

    def hold(self, *streams):
        done = torch.cuda.Event()
        with torch.cuda.stream(self.stream):
            torch.mm(self.a, self.a, out=self.b)
            done.record()
        for st in streams:
            st.wait_event(done)


def _normal(*shape, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16)


@pytest.mark.parametrize("Tq", [1, 60])
def test_shared_states_on_two_streams(Tq):
    """Two launches and a workspace a call, 24 calls on each stream, each stream with one workspace."""
    cases = [Case(8, 2, 128, Tq, 6000, n, seed=i) for i, n in enumerate(([6000, 10], [1, 5999]))]
    need = amskv.amskv_cross_workspace_bytes(cases[0].x)
    assert need > 0 and need == amskv.amskv_cross_workspace_bytes(cases[1].x)
    serial = [c.run() for c in cases]
    for c, o in zip(cases, serial):
        c.check(o)
    streams = [torch.cuda.Stream() for _ in cases]
    spaces = [torch.empty(need, dtype=torch.uint8, device="cuda").fill_(0xFF) for _ in cases]
    outs = [[torch.full_like(c.q, 9.0) for _ in range(24)] for c in cases]
    gate = Gate()
    torch.cuda.synchronize()
    gate.hold(*streams)
    for i in range(24):
        for c, st, ws, o in zip(cases, streams, spaces, outs):
            amskv.amskv_cross_attend(c.x, c.q, c.k, c.v, o[i], workspace=ws, stream=st, **c.kw)
    torch.cuda.synchronize()
    for o, want in zip(outs, serial):
        assert all(torch.equal(x, want) for x in o)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,H", [(3, 8), (40, 10)])
def test_two_caches_of_8_bits(B, H, D):
    """Two caches that compact, turned appends and attention, three images each: (b,h) few enough for one launch an append, and more."""
    sides, pols = [(1, 1), (4, 4), (3, 3), (9, 9), (2, 2), (12, 12)], [(0, 2, False), (1, 1, False)]
    rope = amskv.Rope(rot_dim=32, axes=2)
    tabs, data = [], []
    for s, (a, b) in enumerate(sides):
        t = torch.arange(a * b, device="cuda")
        tabs.append(torch.empty(a * b, 16, 2, device="cuda"))
        amskv.amskv_rope_table(rope, torch.stack((t // b, t % b), dim=1).double(), tabs[-1])
    images = range(3)
    for c in range(2):
        data.append([[[[_normal(B, H, a * b, D, seed=1000 * c + 300 * n + 30 * s + 3 * l + i) for i in range(3)] for l in range(len(pols))]
                      for s, (a, b) in enumerate(sides)] for n in images])

    def calls(h, given, outs, stream):
        """One call after the other, to be taken in turn with another cache's."""
        for n in images:
            amskv.amskv_cache_reset(h)
            for s in range(len(sides)):
                for l in range(len(pols)):
                    q, k, v = given[n][s][l]
                    turned, o = outs[n][s][l]
                    amskv.amskv_append_scale_rotary(h, l, s, rope, tabs[s], q, 0, turned, k, v, stream=stream)
                    yield
                    amskv.amskv_attend(h, l, s, turned, o, stream=stream)
                    yield

    def space():
        return [[[[torch.full_like(x[0], 9.0) for _ in range(2)] for x in step] for step in image] for image in data[0]]

    with Cache(sides, B, H, D, pols) as one, Cache(sides, B, H, D, pols) as two:
        serial, outs = [space(), space()], [space(), space()]
        for c, given, o in zip((one, two), data, serial):
            for _ in calls(c.h, given, o, None):
                pass
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        gate = Gate()
        torch.cuda.synchronize()
        gate.hold(*streams)
        for _ in zip(*(calls(c.h, given, o, st) for c, given, o, st in zip((one, two), data, outs, streams))):
            pass
        torch.cuda.synchronize()
        for a, b in zip(serial, outs):
            for x, y in zip(a, b):
                for u, w in zip(x, y):
                    assert all(torch.equal(p[0], r[0]) and torch.equal(p[1], r[1]) for p, r in zip(u, w))
