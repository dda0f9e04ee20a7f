"""An encoder's states held in 4 bits: written, read back and attended, against the definitions in 64 bits."""
import math

import pytest
import torch

import paper_2511_16047_amd as amskv
import plain_four_bits as plain

pytestmark = pytest.mark.gpu
KV4 = amskv.AMSKV_DTYPE_BF16_KV4


def _normal(*shape, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda")


class Case:
    """Q, K, V of a call: `lengths` per batch element; layout of K and V: heads first, tokens first or packed."""

    def __init__(self, H, Hkv, D, Tq, Tk, lengths, layout="tokens", seed=0, sharp=1.0, spoil=True, hold=True):
        B = len(lengths)
        self.lengths, self.layout, self.D, self.G, self.B, self.Hkv = lengths, layout, D, H // Hkv, B, Hkv
        self.q = _normal(B, H, Tq, D, seed=seed)
        if sharp != 1.0:   # queries of few bits, which the products take as they are
            self.q = torch.round(self.q).clamp(-2, 2) * sharp
        self.scale = 1 / math.sqrt(D) if sharp == 1.0 else 0.125 * math.log(2)   # (under which they are taken as they are)
        self.q = self.q.bfloat16()
        k, v = ((_normal(B, Tk, Hkv, D, seed=seed + i) * torch.exp(0.5 * _normal(Hkv, D, seed=8))).bfloat16() for i in (1, 2))
        for b, n in enumerate(lengths):    # nobody may look behind a batch element's last state
            if spoil:
                k[b, n:], v[b, n:] = float("nan"), float("inf")
        self.kv = k, v
        kw, rows = {}, 0
        if layout == "packed":
            self.k, self.v = (torch.cat([x[b, :n] for b, n in enumerate(lengths)] + [torch.full((3, Hkv, D), float("nan"), dtype=torch.bfloat16,
                                                                                                device="cuda")]) for x in (k, v))
            st, rows = amskv.Strides(0, D, Hkv * D), sum(lengths) + 3
            ends = torch.tensor([0] + [sum(lengths[:b + 1]) for b in range(B)], dtype=torch.int32, device="cuda")
            kw = {"offsets": ends}
        elif layout == "tokens":
            self.k, self.v, st = k, v, amskv.Strides(Tk * Hkv * D, D, Hkv * D)
        else:
            self.k, self.v = (x.transpose(1, 2).contiguous() for x in (k, v))
            st = amskv.Strides(Hkv * Tk * D, Tk * D, D)
        if layout != "packed" and any(n != Tk for n in lengths):
            kw = {"lengths": torch.tensor(lengths, dtype=torch.int32, device="cuda")}
        self.kw = kw
        qs = amskv.Strides(H * Tq * D, Tq * D, D)
        self.x = amskv.Cross(batch=B, heads=H, kv_heads=Hkv, head_dim=D, dtype=KV4, q_tokens=Tq, kv_tokens=Tk, kv_rows=rows, q=qs, k=st, v=st, o=qs,
                             softmax_scale=0.0 if sharp == 1.0 else self.scale)
        need = amskv.amskv_cross_held_bytes(self.x, packed=layout == "packed")
        assert need == (Hkv * rows if layout == "packed" else B * Hkv * Tk) * (D // 2 + D // 32)
        self.need, self.buffers = need, [torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda") for _ in range(2)]
        self.held = [x[:need] for x in self.buffers]
        if hold:
            self.hold()

    def hold(self, **k):
        amskv.amskv_cross_hold(self.x, self.k, self.v, *self.held, **dict(self.kw, **k))

    def export(self, fill=9.0, **k):
        out = [torch.full_like(x, fill) for x in (self.k, self.v)]
        amskv.amskv_cross_export(self.x, *self.held, *out, **dict(self.kw, **k))
        return out

    def check_held(self, fill=9.0):
        """What is read back is what the states are held as; rows without states, and what lies behind the buffers, stay."""
        for got, x in zip(self.export(fill), self.kv):
            if self.layout == "packed":
                want = torch.cat([plain.held(x[b, :n]) for b, n in enumerate(self.lengths)] + [torch.full((3, *x.shape[2:]), fill, dtype=torch.float64,
                                                                                                        device="cuda")])
            else:
                want = torch.full(x.shape, fill, dtype=torch.float64, device="cuda")
                for b, n in enumerate(self.lengths):
                    want[b, :n] = plain.held(x[b, :n])
                if self.layout == "heads":
                    want = want.transpose(1, 2)
            assert torch.equal(got.double(), want)
        for x in self.buffers:
            assert bool((x[self.need:] == 0xFF).all())

    def run(self, workspace=True, out=None, **k):
        out = torch.full_like(self.q, 9.0) if out is None else out
        need = amskv.amskv_cross_workspace_bytes(self.x)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda").fill_(0xFF) if need and workspace else None
        amskv.amskv_cross_attend(self.x, self.q, *self.held, out, workspace=ws, **dict(self.kw, **k))
        return out

    def check(self, out):
        for b, n in enumerate(self.lengths):
            if n == 0:
                assert bool((out[b] == 0).all())
                continue
            k, v = (plain.held(x[b, :n]).transpose(0, 1).repeat_interleave(self.G, dim=0) for x in self.kv)
            want, bound = plain.attention(self.q[b], k, v, self.scale)
            off = (out[b].double() - want).abs()
            assert bool((off <= bound).all()), "batch element %d of %d states: %.3f of the bound" % (b, n, float((off / bound).max()))


@pytest.mark.parametrize("layout", ["tokens", "heads", "packed"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hkv", [1, 3])
@pytest.mark.parametrize("lengths", [[1], [5, 0, 31, 32, 33, 64, 65, 0], [128, 127, 129, 200], [0, 0], [1000, 3]], ids=str)
def test_written_and_read_back(layout, D, Hkv, lengths):
    Case(Hkv, Hkv, D, 1, max(lengths + [1]), lengths, layout).check_held()


@pytest.mark.parametrize("layout", ["tokens", "heads", "packed"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Hkv", [2, 4, 6, 8])
@pytest.mark.parametrize("lengths", [[1], [5, 0, 31, 32, 33, 64, 65, 0], [128, 127, 129, 200]], ids=str)
def test_heads_side_by_side(layout, D, Hkv, lengths):
    """Rows of two and four heads to a workgroup."""
    Case(Hkv, Hkv, D, 1, max(lengths), lengths, layout, seed=Hkv).check_held()


def test_held_with_no_lengths():
    """All rows of a padded tensor; K alone, V alone."""
    c = Case(2, 2, 64, 1, 70, [70, 70], hold=False)
    amskv.amskv_cross_hold(c.x, c.k, None, c.held[0], None)
    assert bool((c.held[1] == 0xFF).all())
    amskv.amskv_cross_hold(c.x, None, c.v, None, c.held[1])
    c.check_held()
    one = torch.empty_like(c.v)
    amskv.amskv_cross_export(c.x, None, c.held[1], None, one)
    assert torch.equal(one.double(), plain.held(c.v))


@pytest.mark.parametrize("D", [64, 128])
def test_held_in_other_orders(D):
    """K and V out of one tensor of states, and back into one; what lies around stays."""
    B, H, T = 3, 5, 90
    lengths = torch.tensor([90, 0, 41], dtype=torch.int32, device="cuda")
    kv = _normal(B, T, 2, H, D, seed=1).bfloat16()
    st = amskv.Strides(T * 2 * H * D, D, 2 * H * D)
    x = amskv.Cross(batch=B, heads=H, kv_heads=H, head_dim=D, dtype=KV4, q_tokens=1, kv_tokens=T, k=st, v=st)
    held = [torch.empty(amskv.amskv_cross_held_bytes(x), dtype=torch.uint8, device="cuda") for _ in range(2)]
    amskv.amskv_cross_hold(x, kv[:, :, 0], kv[:, :, 1], *held, lengths=lengths)
    out = torch.full((B, T, 3, H, D), 5.0, dtype=torch.bfloat16, device="cuda")
    x.k = x.v = amskv.Strides(T * 3 * H * D, D, 3 * H * D)
    amskv.amskv_cross_export(x, *held, out[:, :, 0], out[:, :, 2], lengths=lengths)
    for i, j in ((0, 0), (1, 2)):
        for b, n in enumerate(lengths.tolist()):
            assert torch.equal(out[b, :n, j].double(), plain.held(kv[b, :n, i])) and bool((out[b, n:, j] == 5.0).all())
    assert bool((out[:, :, 1] == 5.0).all())


@pytest.mark.parametrize("layout", ["tokens", "heads", "packed"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,Hkv", [(3, 3), (6, 2), (8, 1)])
@pytest.mark.parametrize("Tq", [1, 5, 33, 100, 129, 300])
def test_ragged(layout, D, H, Hkv, Tq):
    c = Case(H, Hkv, D, Tq, 77, [77, 0, 1, 31, 32, 33, 64, 65, 0], layout)
    c.check(c.run())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Tk", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255, 257, 1000])
@pytest.mark.parametrize("Tq", [1, 32, 64, 128, 256])
def test_lengths(D, Tk, Tq):
    c = Case(2, 2, D, Tq, Tk, [Tk, Tk])
    c.check(c.run())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("Tq,H,Hkv", [(1, 4, 4), (1, 8, 2), (3, 16, 2), (40, 2, 2), (130, 2, 1)])
@pytest.mark.parametrize("lengths", [[5000], [4096, 0, 1, 700, 4095]], ids=["one", "ragged"])
def test_shared_between_workgroups(D, Tq, H, Hkv, lengths):
    """Few rows over many states, with the workspace and without; runs of tiles that no state of a short batch element reaches."""
    c = Case(H, Hkv, D, Tq, max(lengths), lengths)
    assert amskv.amskv_cross_workspace_bytes(c.x) > 0
    a, b = c.run(), c.run(workspace=False)
    c.check(a), c.check(b)
    assert torch.equal(a, c.run())      # the order of the sums is fixed


@pytest.mark.parametrize("sharp", [0.0, 30.0, 300.0])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,Tq,Tk", [(4, 1, 3000), (4, 64, 500), (80, 260, 600)])
def test_flat_and_sharp_scores(sharp, D, H, Tq, Tk):
    c = Case(H, H // 2, D, Tq, Tk, [Tk, Tk // 2], sharp=sharp)
    c.check(c.run())


def test_many_units():
    c = Case(16, 16, 64, 20, 90, [(37 * b) % 91 for b in range(130)])
    c.check(c.run())
    c.check_held()


@pytest.mark.parametrize("layout", ["tokens", "heads", "packed"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,Hkv,Tq", [(10, 10, 100), (10, 10, 129), (20, 10, 150), (12, 12, 250), (14, 14, 257), (7, 7, 700)])
def test_many_units_of_many_rows(layout, D, H, Hkv, Tq):
    """Enough rows for waves that share K and V: any number of tiles, none, and states left over."""
    lengths = [200, 0, 1, 31, 32, 33, 63, 64, 65, 96, 97, 127, 128, 129, 199, 160]
    c = Case(H, Hkv, D, Tq, 200, lengths, layout)
    c.check(c.run())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,Tq", [(17, 260), (8, 500)])
def test_many_units_over_many_states(D, H, Tq):
    c = Case(H, H, D, Tq, 1100, [1100, 1099, 0, 1024, 1025, 513, 64, 1088, 3, 1100, 1056, 700, 1, 1087, 90, 1100])
    c.check(c.run())


def test_no_states_at_all():
    c = Case(4, 2, 64, 7, 0, [0, 0, 0], spoil=False)
    c.check(c.run())
    out = torch.full_like(c.q, 9.0)
    amskv.amskv_cross_attend(c.x, c.q, None, None, out)
    assert bool((out == 0).all())


@pytest.mark.parametrize("Tq", [1, 200])
def test_lengths_the_device_got_wrong(Tq):
    """Lengths and offsets outside the tensors are cut to what is there, in all three calls."""
    wrong = torch.tensor([1 << 30, -5, 51], dtype=torch.int32, device="cuda")
    c = Case(2, 2, 64, Tq, 50, [50, 0, 50], spoil=False, hold=False)
    c.hold(lengths=wrong)
    for got, x in zip(c.export(lengths=wrong), c.kv):
        assert torch.equal(got[::2].double(), plain.held(x[::2])) and bool((got[1] == 9.0).all())
    c.check(c.run(lengths=wrong))
    p = Case(2, 2, 64, Tq, 50, [20, 0, 30], "packed", spoil=False, hold=False)
    p.k[-3:], p.v[-3:] = 0, 0
    wrong = torch.tensor([-7, 20, 20, 1 << 30], dtype=torch.int32, device="cuda")
    p.hold(offsets=wrong)
    assert torch.equal(p.export(offsets=wrong)[0].double(), plain.held(p.k))
    p.x.kv_tokens = 30
    p.check(p.run(offsets=wrong[[0, 1, 2, 2]] + torch.tensor([0, 0, 0, 30], dtype=torch.int32, device="cuda")))


def test_far_rows():
    """Codes and states beyond 2^31 bytes."""
    H, D, T = 16, 128, 2500000
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    k, v = (torch.empty(T, H, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2))
    q = _normal(2, H, 2, D, seed=3).bfloat16()
    out = torch.empty_like(q)
    qs, st = amskv.Strides(H * 2 * D, 2 * D, D), amskv.Strides(0, D, H * D)
    x = amskv.Cross(batch=2, heads=H, kv_heads=H, head_dim=D, dtype=KV4, q_tokens=2, kv_tokens=500, kv_rows=T, q=qs, k=st, v=st, o=qs)
    held = [torch.empty(amskv.amskv_cross_held_bytes(x, packed=True), dtype=torch.uint8, device="cuda") for _ in range(2)]
    assert held[0].numel() > 2 ** 31 and k.numel() * 2 > 2 ** 32
    ends = [T - 700, T - 300, T]
    offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
    amskv.amskv_cross_hold(x, k, v, *held, offsets=offsets)
    amskv.amskv_cross_attend(x, q, *held, out, offsets=offsets)
    back = torch.full_like(k, 9.0)
    amskv.amskv_cross_export(x, held[0], None, back, None, offsets=offsets)
    assert torch.equal(back[ends[0]:].double(), plain.held(k[ends[0]:])) and bool((back[:ends[0]] == 9.0).all())
    for b in range(2):
        want, bound = plain.attention(q[b], *(plain.held(y[ends[b]:ends[b + 1]]).transpose(0, 1) for y in (k, v)), 1 / math.sqrt(D))
        assert bool(((out[b].double() - want).abs() <= bound).all())


def test_far_rows_of_one_head():
    """One unit whose codes pass 2^31 bytes: a batch element of nearly all rows, whose last 150 weigh some e^180 times the others, and one of 150."""
    D, T, n = 128, 34000000, 300
    q = torch.round(_normal(2, 1, 3, D, seed=3)).clamp(-1, 1).bfloat16()
    q[..., :64] = 1
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    k, v = (torch.empty(T, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2))
    k[:T - n, :64] = -32.0
    k[:T - n, 64:] = 0
    k[T - n:] *= 0.125
    out = torch.empty_like(q)
    qs, st = amskv.Strides(3 * D, 3 * D, D), amskv.Strides(0, D, D)
    x = amskv.Cross(batch=2, heads=1, kv_heads=1, head_dim=D, dtype=KV4, q_tokens=3, kv_tokens=T, kv_rows=T, q=qs, k=st, v=st, o=qs)
    held = [torch.empty(amskv.amskv_cross_held_bytes(x, packed=True), dtype=torch.uint8, device="cuda") for _ in range(2)]
    assert T * D // 2 > 2 ** 31
    offsets = torch.tensor([0, T - n // 2, T], dtype=torch.int32, device="cuda")
    ws = torch.empty(amskv.amskv_cross_workspace_bytes(x), dtype=torch.uint8, device="cuda")
    amskv.amskv_cross_hold(x, k, v, *held, offsets=offsets)
    amskv.amskv_cross_attend(x, q, *held, out, offsets=offsets, workspace=ws)
    for b, rows in ((0, slice(T - n, T - n // 2)), (1, slice(T - n // 2, T))):
        want, bound = plain.attention(q[b], *(plain.held(y[rows])[None] for y in (k, v)), 1 / math.sqrt(D))
        assert bool(((out[b].double() - want).abs() <= bound).all())
    v.fill_(9.0)
    amskv.amskv_cross_export(x, held[0], None, v, None, offsets=offsets)
    for i in range(0, T, 1 << 20):
        assert torch.equal(v[i:i + (1 << 20)].double(), plain.held(k[i:i + (1 << 20)]))


def test_captured_and_replayed():
    """Lengths are read when the graph runs, not when it is captured; new states are held, attended and read back in it; eager calls in
    between use buffers of their own."""
    for Tq, Tk in ((70, 200), (1, 4000)):
        c = Case(4, 4, 64, Tq, Tk, [Tk, Tk], spoil=False)
        need = amskv.amskv_cross_workspace_bytes(c.x)
        ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        held = [torch.empty_like(x) for x in c.held]
        lengths = torch.tensor([Tk, Tk], dtype=torch.int32, device="cuda")
        out, back = torch.empty_like(c.q), [torch.empty_like(c.k) for _ in range(2)]
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            amskv.amskv_cross_hold(c.x, c.k, c.v, *held, lengths=lengths)
            amskv.amskv_cross_attend(c.x, c.q, *held, out, lengths=lengths, workspace=ws if need else None)
            amskv.amskv_cross_export(c.x, *held, *back, lengths=lengths)
        for i, n in enumerate(([Tk, Tk], [3, Tk - 1], [0, 17])):
            for j, x in enumerate((c.k, c.v)):
                x.copy_(_normal(*x.shape, seed=50 + 2 * i + j))
            lengths.copy_(torch.tensor(n, dtype=torch.int32))
            out.fill_(9.0)
            for x in back:
                x.fill_(9.0)
            graph.replay()
            c.hold(lengths=lengths)
            eager = c.run(lengths=lengths)
            again = c.export(lengths=lengths)
            torch.cuda.synchronize()
            assert torch.equal(out, eager) and all(torch.equal(x, y) for x, y in zip(back, again))
            c.lengths = n
            c.check(out)


def test_two_streams_at_once():
    a, b = Case(8, 2, 128, 1, 6000, [6000, 10], seed=1, hold=False), Case(8, 2, 128, 1, 6000, [1, 5999], seed=7, hold=False)
    torch.cuda.synchronize()
    outs = []
    for c, st in ((a, torch.cuda.Stream()), (b, torch.cuda.Stream())):
        ws = torch.empty(amskv.amskv_cross_workspace_bytes(c.x), dtype=torch.uint8, device="cuda")
        out = torch.empty_like(c.q)
        torch.cuda.synchronize()
        c.hold(stream=st)
        amskv.amskv_cross_attend(c.x, c.q, *c.held, out, workspace=ws, stream=st, **c.kw)
        outs.append((c, out, ws))
    torch.cuda.synchronize()
    for c, out, _ in outs:
        c.check(out)


def test_steps_of_a_model():
    """A scale cache in 4 bits and a prompt held in 4 bits, layer behind layer: self attention, then cross attention to the prompt, whose
    output is the next layer's input; the cache is read back at the end."""
    B, H, D, sides, layers, lengths = 3, 4, 64, [1, 2, 4, 6], 3, [20, 0, 33]
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    w = [[torch.randn(D, D, generator=g, device="cuda") / 8 for _ in range(4)] for _ in range(layers)]
    prompt = [Case(H, 2, D, 1, 40, lengths, seed=20 + l) for l in range(layers)]
    args = (layers, H, D, sides, sides, B, amskv.AMSKV_DTYPE_BF16_KV4, [(1, 1, False)] * layers)
    arena = torch.empty(amskv.amskv_cache_required_bytes(*args), dtype=torch.uint8, device="cuda").fill_(0xFF)
    h = amskv.amskv_cache_create(*args, arena=arena)
    kept = [{} for _ in range(layers)]
    for s, side in enumerate(sides):
        T = side * side
        x = _normal(B, H, T, D, seed=40 + s).bfloat16()
        qs = amskv.Strides(H * T * D, T * D, D)
        for l in range(layers):
            q, k, v, cq = ((x.float() @ m).bfloat16() for m in w[l])
            o, y = torch.empty_like(x), torch.empty_like(x)
            amskv.amskv_append_scale(h, l, s, k, v)
            amskv.amskv_attend(h, l, s, q, o)
            kept[l] = {i: y for i, y in kept[l].items() if i == 0 or s - i <= 1}
            kept[l][s] = plain.held(k), plain.held(v)
            kk, vv = (torch.cat([kept[l][i][j] for i in sorted(kept[l])], dim=2) for j in range(2))
            want, bound = plain.attention(q, kk, vv, 1 / 8)
            assert bool(((o.double() - want).abs() <= bound).all())
            p = prompt[l]
            p.x.q_tokens, p.x.q, p.x.o, p.q = T, qs, qs, cq
            need = amskv.amskv_cross_workspace_bytes(p.x)
            ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
            amskv.amskv_cross_attend(p.x, cq, *p.held, y, workspace=ws, **p.kw)
            p.check(y)
            x = (x.float() + o.float() + y.float()).bfloat16()
    for l in range(layers):
        n = sum(i[2] for i in amskv.amskv_cache_layout(h, l))
        k, v = (torch.empty(B, H, n, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        amskv.amskv_cache_export(h, l, k, v)
        for got, j in ((k, 0), (v, 1)):
            assert torch.equal(got.double(), torch.cat([kept[l][i][j] for i in sorted(kept[l])], dim=2))
    torch.cuda.synchronize()
    amskv.amskv_cache_destroy(h)


def test_without_the_extension_module(monkeypatch):
    """Both directions through ctypes: the same values."""
    from paper_2511_16047_amd import binding
    c = Case(6, 3, 64, 5, 40, [40, 0, 33])
    want = c.export()
    for name in ("_hold", "_export", "_cross"):
        monkeypatch.setattr(binding, name, binding._not_built)
    for x in c.held:
        x.fill_(0xFF)
    c.hold()
    assert all(torch.equal(a, b) for a, b in zip(want, c.export()))
    c.check(c.run())
