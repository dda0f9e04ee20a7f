"""Calls over K and V in 4 bits that really run at the same time: everything is enqueued on both streams while they wait behind one long
piece of work, and every result is that of the same calls one after the other."""
import pytest
import torch

import paper_2511_16047_amd as amskv
from test_gpu_cache_in_4_bits import Cache
from test_gpu_held_states import Case
from test_gpu_operators_overlap import Gate, _normal

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,Hkv,Tq,Tk,D", [(8, 2, 1, 6000, 128), (8, 2, 60, 6000, 128), (8, 8, 3, 77, 64), (40, 40, 260, 600, 64)])
def test_held_states_on_two_streams(H, Hkv, Tq, Tk, D):
    """States held, attended and read back, 12 times on each stream, each stream with buffers and a workspace of its own; between them they
    hold two prompts by turns."""
    B = 2 if H < 40 else 8
    prompts = [[Case(H, Hkv, D, Tq, Tk, [max(0, n - 11 * b) for b in range(B)], seed=10 * i + j, spoil=False, hold=False) for j, n in enumerate((Tk, Tk - 1))]
               for i in range(2)]
    for pair in prompts:
        for c in pair:        # (a pair's calls say the same shape and differ in their lengths)
            c.kw = {"lengths": torch.tensor(c.lengths, dtype=torch.int32, device="cuda")}
    need = amskv.amskv_cross_workspace_bytes(prompts[0][0].x)

    def buffers():
        c = prompts[0][0]
        return ([torch.full_like(x, 0xFF) for x in c.held], torch.empty(need, dtype=torch.uint8, device="cuda").fill_(0xFF) if need else None,
                [(torch.full_like(c.q, 9.0), torch.full_like(c.k, 9.0), torch.full_like(c.v, 9.0)) for _ in range(12)])

    def calls(pair, held, ws, outs, stream):
        for i, (o, k, v) in enumerate(outs):
            c = pair[i % 2]
            amskv.amskv_cross_hold(c.x, c.k, c.v, *held, stream=stream, **c.kw)
            yield
            amskv.amskv_cross_attend(c.x, c.q, *held, o, workspace=ws, stream=stream, **c.kw)
            yield
            amskv.amskv_cross_export(c.x, *held, k, v, stream=stream, **c.kw)
            yield

    serial, together = [buffers() for _ in prompts], [buffers() for _ in prompts]
    for pair, b in zip(prompts, serial):
        for _ in calls(pair, *b, None):
            pass
        for i in (0, 1):
            pair[i].check(b[2][i][0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in prompts]
    gate = Gate()
    torch.cuda.synchronize()
    gate.hold(*streams)
    for _ in zip(*(calls(pair, *b, st) for pair, b, st in zip(prompts, together, streams))):
        pass
    torch.cuda.synchronize()
    for a, b in zip(serial, together):
        for x, y in zip(a[2], b[2]):
            assert all(torch.equal(p, r) for p, r in zip(x, y))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,H", [(3, 8), (16, 10)])
def test_two_caches_of_4_bits(B, H, D):
    """Two caches that compact, turned appends, attention and read-back, three images each."""
    sides, pols = [(1, 1), (4, 4), (3, 3), (9, 9), (2, 2), (16, 17)], [(0, 2, False), (1, 1, False)]
    rope = amskv.Rope(rot_dim=32, axes=2)
    tabs = []
    for a, b in sides:
        t = torch.arange(a * b, device="cuda")
        tabs.append(torch.empty(a * b, 16, 2, device="cuda"))
        amskv.amskv_rope_table(rope, torch.stack((t // b, t % b), dim=1).double(), tabs[-1])
    images = range(3)
    data = [[[[[_normal(B, H, a * b, D, seed=1000 * c + 300 * n + 30 * s + 3 * l + i) for i in range(3)] for l in range(len(pols))]
              for s, (a, b) in enumerate(sides)] for n in images] for c in range(2)]

    def calls(h, given, outs, backs, stream):
        for n in images:
            amskv.amskv_cache_reset(h)
            for s in range(len(sides)):
                for l in range(len(pols)):
                    (q, k, v), (turned, o) = given[n][s][l], outs[n][s][l]
                    amskv.amskv_append_scale_rotary(h, l, s, rope, tabs[s], q, 0, turned, k, v, stream=stream)
                    yield
                    amskv.amskv_attend(h, l, s, turned, o, stream=stream)
                    yield
            for l in range(len(pols)):
                amskv.amskv_cache_export(h, l, *backs[n][l], stream=stream)
                yield

    with Cache(sides, B, H, D, pols) as one, Cache(sides, B, H, D, pols) as two:
        for s in range(len(sides)):       # (what stays of an image)
            for l in range(len(pols)):
                amskv.amskv_append_scale(one.h, l, s, *data[0][0][s][l][1:])
        kept = [sum(x[2] for x in amskv.amskv_cache_layout(one.h, l)) for l in range(len(pols))]

        def space():
            return ([[[[torch.full_like(x[0], 9.0) for _ in range(2)] for x in step] for step in image] for image in data[0]],
                    [[[torch.full((B, H, n, D), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)] for n in kept] for _ in images])

        serial, together = [space(), space()], [space(), space()]
        for c, given, x in zip((one, two), data, serial):
            for _ in calls(c.h, given, *x, None):
                pass
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in range(2)]
        gate = Gate()
        torch.cuda.synchronize()
        gate.hold(*streams)
        for _ in zip(*(calls(c.h, given, *x, st) for c, given, x, st in zip((one, two), data, together, streams))):
            pass
        torch.cuda.synchronize()

        def flat(x):
            return [x] if torch.is_tensor(x) else [t for y in x for t in flat(y)]

        assert all(torch.equal(a, b) for a, b in zip(flat(serial), flat(together))) and not any(bool((t == 9.0).all()) for t in flat(serial))
