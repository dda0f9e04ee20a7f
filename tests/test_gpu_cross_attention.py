"""Cross attention to states of other lengths, against the definition in 64 bits."""
import math

import pytest
import torch

import paper_2511_16047_amd as amskv
import plain_operators as plain

pytestmark = pytest.mark.gpu


def _normal(*shape, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda")


class Case:
    """Q, K, V of a call: `lengths` per batch element; layout of K and V: heads first, tokens first or packed."""

    def __init__(self, H, Hkv, D, Tq, Tk, lengths, layout="tokens", seed=0, sharp=1.0, spoil=True):
        B = len(lengths)
        self.lengths, self.layout, self.D, self.G = lengths, layout, D, H // Hkv
        self.q = (_normal(B, H, Tq, D, seed=seed) * sharp).bfloat16()
        k, v = (_normal(B, Tk, Hkv, D, seed=seed + i).bfloat16() for i in (1, 2))
        for b, n in enumerate(lengths):    # nobody may look behind a batch element's last state
            if spoil:
                k[b, n:], v[b, n:] = float("nan"), float("inf")
        self.kv = k, v
        kw, rows = {}, 0
        if layout == "packed":
            self.k, self.v = (torch.cat([x[b, :n] for b, n in enumerate(lengths)] + [torch.full((3, Hkv, D), float("nan"), dtype=torch.bfloat16,
                                                                                                device="cuda")]) for x in (k, v))
            st, rows = amskv.Strides(0, D, Hkv * D), sum(lengths)
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
        self.x = amskv.Cross(batch=B, heads=H, kv_heads=Hkv, head_dim=D, dtype=amskv.AMSKV_DTYPE_BF16, q_tokens=Tq, kv_tokens=Tk, kv_rows=rows, q=qs,
                             k=st, v=st, o=qs)

    def run(self, workspace=True, out=None, **k):
        out = torch.full_like(self.q, 9.0) if out is None else out
        need = amskv.amskv_cross_workspace_bytes(self.x)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda").fill_(0xFF) if need and workspace else None
        amskv.amskv_cross_attend(self.x, self.q, self.k, self.v, out, workspace=ws, **dict(self.kw, **k))
        return out

    def check(self, out):
        for b, n in enumerate(self.lengths):
            if n == 0:
                assert bool((out[b] == 0).all())
                continue
            k, v = (x[b, :n].transpose(0, 1).repeat_interleave(self.G, dim=0) for x in self.kv)
            want, bound = plain.attention(self.q[b], k, v, 1 / math.sqrt(self.D))
            off = (out[b].double() - want).abs()
            assert bool((off <= bound).all()), "batch element %d of %d states: %.3f of the bound" % (b, n, float((off / bound).max()))


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


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,Tq,Tk", [(2, 5, 90), (4, 40, 500), (2, 1, 5000), (80, 100, 300), (80, 500, 300), (200, 70, 200)])
@pytest.mark.parametrize("start,end", [(0, 40), (0, 64), (33, 75), (32, 80)])
def test_scores_beyond_fp32_weigh_nothing(D, H, Tq, Tk, start, end):
    """A channel of 2^100 times -2^100: -inf in fp32, at the first keys, whole blocks and parts of them; the other keys as if alone."""
    c = Case(H, H, D, Tq, Tk, [Tk])
    c.q[..., 0] = 2.0 ** 100
    for x in {id(y): y for y in (c.k, c.kv[0])}.values():
        x[..., 0] = 0
        x[:, start:end, :, 0] = -2.0 ** 100
    out = c.run()
    k, v = (torch.cat((x[0, :start], x[0, end:])).transpose(0, 1).clone() for x in c.kv)
    want, bound = plain.attention(c.q[0], k, v, 1 / math.sqrt(D))
    assert bool(((out[0].double() - want).abs() <= bound).all())


@pytest.mark.parametrize("sharp", [0.0, 30.0, 300.0])
@pytest.mark.parametrize("Tq,Tk", [(1, 3000), (64, 500)])
def test_flat_and_sharp_scores(sharp, Tq, Tk):
    c = Case(4, 2, 64, Tq, Tk, [Tk, Tk // 2], sharp=sharp)
    c.check(c.run())


def test_many_units():
    c = Case(16, 16, 64, 20, 90, [(37 * b) % 91 for b in range(130)])
    c.check(c.run())


@pytest.mark.parametrize("layout", ["tokens", "heads", "packed"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,Hkv,Tq", [(10, 10, 100), (10, 10, 129), (20, 10, 150), (12, 12, 250), (14, 14, 257), (7, 7, 700)])
def test_many_units_of_many_rows(layout, D, H, Hkv, Tq):
    """Enough rows for waves that share K and V: any number of tiles, none, and states left over."""
    lengths = [200, 0, 1, 31, 32, 33, 63, 64, 65, 96, 97, 127, 128, 129, 199, 160]
    c = Case(H, Hkv, D, Tq, 200, lengths, layout)
    c.check(c.run())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("sharp", [0.0, 1.0, 300.0])
@pytest.mark.parametrize("H,Tq", [(17, 260), (8, 500)])
def test_many_units_over_many_states(D, sharp, H, Tq):
    c = Case(H, H, D, Tq, 1100, [1100, 1099, 0, 1024, 1025, 513, 64, 1088, 3, 1100, 1056, 700, 1, 1087, 90, 1100], sharp=sharp)
    c.check(c.run())


def test_few_rows_over_states_that_do_not_fit_anywhere_else():
    """Hundreds of megabytes of states, read once by teams."""
    c = Case(32, 32, 64, 20, 4100, [4100] * 10 + [4000, 1] + [33] * 3 + [0])
    c.check(c.run())
    c = Case(32, 32, 128, 20, 4100, [4100, 4099, 64, 0, 33])
    c.check(c.run())


def test_no_states_at_all():
    c = Case(4, 2, 64, 7, 0, [0, 0, 0], spoil=False)
    c.check(c.run())
    out = torch.full_like(c.q, 9.0)
    amskv.amskv_cross_attend(c.x, c.q, None, None, out)
    assert bool((out == 0).all())


@pytest.mark.parametrize("Tq", [1, 200])
def test_lengths_the_device_got_wrong(Tq):
    """Lengths and offsets outside the tensors are cut to what is there."""
    c = Case(2, 2, 64, Tq, 50, [50, 0, 50], spoil=False)
    c.check(c.run(lengths=torch.tensor([1 << 30, -5, 51], dtype=torch.int32, device="cuda")))
    p = Case(2, 2, 64, Tq, 50, [20, 0, 30], "packed")
    p.check(p.run(offsets=torch.tensor([-7, 20, 20, 1 << 30], dtype=torch.int32, device="cuda")))
    p = Case(2, 2, 64, Tq, 50, [20, 0, 0], "packed")
    p.check(p.run(offsets=torch.tensor([0, 20, 3, -9], dtype=torch.int32, device="cuda")))


def test_a_longer_run_than_kv_tokens_is_cut():
    c = Case(2, 2, 64, 9, 64, [64, 64], "packed")
    c.x.kv_tokens = 40
    out = c.run()
    c.lengths = [40, 40]
    c.check(out)


@pytest.mark.parametrize("Tq,Tk", [(100, 90), (1, 4000)])
def test_tensors_in_other_orders(Tq, Tk):
    """Q and O token-major in wider rows, K and V inside one tensor of states; what lies around O stays."""
    B, H, D = 2, 4, 64
    c = Case(H, H, D, Tq, Tk, [Tk, Tk - 7])
    q = torch.zeros(B, Tq, 2, H, D, dtype=torch.bfloat16, device="cuda")
    q[:, :, 1] = c.q.transpose(1, 2)
    kv = torch.stack((c.k, c.v), dim=2).contiguous()        # [B, Tk, 2, H, D]
    out = torch.full((B, Tq, H + 2, D), 5.0, dtype=torch.bfloat16, device="cuda")
    st = amskv.Strides(Tk * 2 * H * D, D, 2 * H * D)
    c.x.q, c.x.o, c.x.k, c.x.v = amskv.Strides(Tq * 2 * H * D, D, 2 * H * D), amskv.Strides(Tq * (H + 2) * D, D, (H + 2) * D), st, st
    need = amskv.amskv_cross_workspace_bytes(c.x)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    amskv.amskv_cross_attend(c.x, q[:, :, 1], kv[:, :, 0], kv[:, :, 1], out[:, :, 1:], workspace=ws, **c.kw)
    c.check(out[:, :, 1:H + 1].transpose(1, 2))
    assert bool((out[:, :, 0] == 5.0).all()) and bool((out[:, :, H + 1] == 5.0).all())


def test_one_set_of_states_for_all():
    """Batch stride 0: every batch element reads the same states, each its own number of them."""
    c = Case(2, 1, 128, 10, 40, [40])
    x = amskv.Cross.from_buffer_copy(c.x)
    x.batch, x.k.batch, x.v.batch = 3, 0, 0
    q = _normal(3, 2, 10, 128, seed=9).bfloat16()
    out = torch.empty_like(q)
    n = [40, 0, 13]
    amskv.amskv_cross_attend(x, q, c.k, c.v, out, lengths=torch.tensor(n, dtype=torch.int32, device="cuda"))
    for b in range(3):
        if n[b]:
            k, v = (y[0, :n[b]].transpose(0, 1).expand(2, -1, -1) for y in c.kv)
            want, bound = plain.attention(q[b], k, v, 1 / math.sqrt(128))
            assert bool(((out[b].double() - want).abs() <= bound).all())
        else:
            assert bool((out[b] == 0).all())


def test_scale_of_the_callers():
    c = Case(2, 2, 64, 40, 60, [60])
    c.x.softmax_scale = 0.02
    k, v = (x[0].transpose(0, 1) for x in c.kv)
    want, bound = plain.attention(c.q[0], k, v, c.x.softmax_scale)
    assert bool(((c.run()[0].double() - want).abs() <= bound).all())


def test_far_rows():
    """K and V beyond 2^31 bytes."""
    H, D, T = 16, 128, 700000
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    k, v = (torch.empty(T, H, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2))
    assert k.numel() * 2 > 2 ** 31
    q = _normal(2, H, 2, D, seed=3).bfloat16()
    out = torch.empty_like(q)
    qs, st = amskv.Strides(H * 2 * D, 2 * D, D), amskv.Strides(0, D, H * D)
    x = amskv.Cross(batch=2, heads=H, kv_heads=H, head_dim=D, dtype=amskv.AMSKV_DTYPE_BF16, q_tokens=2, kv_tokens=500, kv_rows=T, q=qs, k=st, v=st, o=qs)
    ends = [T - 700, T - 300, T]
    amskv.amskv_cross_attend(x, q, k, v, out, offsets=torch.tensor(ends, dtype=torch.int32, device="cuda"))
    for b in range(2):
        want, bound = plain.attention(q[b], k[ends[b]:ends[b + 1]].transpose(0, 1), v[ends[b]:ends[b + 1]].transpose(0, 1), 1 / math.sqrt(D))
        assert bool(((out[b].double() - want).abs() <= bound).all())


def test_far_queries():
    """The most queries a head may have, of eight heads that share one: Q and O beyond 2^32 bytes."""
    H, D, Tq, Tk = 8, 64, 1 << 22, 33
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    q = torch.empty(1, H, Tq, D, dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    k, v = (_normal(1, Tk, 1, D, seed=i).bfloat16() for i in (1, 2))
    assert q.numel() * 2 >= 2 ** 32
    out = torch.full_like(q, 9.0)
    qs, st = amskv.Strides(0, Tq * D, D), amskv.Strides(0, 0, D)
    x = amskv.Cross(batch=1, heads=H, kv_heads=1, head_dim=D, dtype=amskv.AMSKV_DTYPE_BF16, q_tokens=Tq, kv_tokens=Tk, q=qs, k=st, v=st, o=qs)
    amskv.amskv_cross_attend(x, q, k, v, out)
    assert not bool((out[:, :, ::4097] == 9.0).all(dim=-1).any())
    for h in (0, 3, H - 1):
        for at in (0, 2 ** 21 - 50, Tq - 100):
            want, bound = plain.attention(q[0, h, at:at + 100], k[0, :, 0], v[0, :, 0], 1 / math.sqrt(D))
            assert bool(((out[0, h, at:at + 100].double() - want).abs() <= bound).all())


def test_captured_and_replayed():
    """Lengths are read when the graph runs, not when it is captured; eager calls in between use a workspace of their own."""
    for Tq, Tk in ((70, 200), (1, 4000)):
        c = Case(4, 4, 64, Tq, Tk, [Tk, Tk], spoil=False)
        need = amskv.amskv_cross_workspace_bytes(c.x)
        ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        lengths = torch.tensor([Tk, Tk], dtype=torch.int32, device="cuda")
        out = torch.empty_like(c.q)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            amskv.amskv_cross_attend(c.x, c.q, c.k, c.v, out, lengths=lengths, workspace=ws if need else None)
        for n in ([Tk, Tk], [3, Tk - 1], [0, 17]):
            lengths.copy_(torch.tensor(n, dtype=torch.int32))
            out.fill_(9.0)
            graph.replay()
            eager = c.run(lengths=lengths)
            torch.cuda.synchronize()
            assert torch.equal(out, eager)
            c.lengths = n
            c.check(out)


def test_two_streams_at_once():
    a, b = Case(8, 2, 128, 1, 6000, [6000, 10], seed=1), Case(8, 2, 128, 1, 6000, [1, 5999], seed=7)
    torch.cuda.synchronize()
    outs = []
    for c, st in ((a, torch.cuda.Stream()), (b, torch.cuda.Stream())):
        ws = torch.empty(amskv.amskv_cross_workspace_bytes(c.x), dtype=torch.uint8, device="cuda")
        out = torch.empty_like(c.q)
        torch.cuda.synchronize()
        amskv.amskv_cross_attend(c.x, c.q, c.k, c.v, out, workspace=ws, stream=st, **c.kw)
        outs.append((c, out, ws))
    torch.cuda.synchronize()
    for c, out, _ in outs:
        c.check(out)
