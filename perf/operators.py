"""Operators beside the attention over the scale cache, as cases that can be timed and compared: rotary positions, the cache
held in 8 bits, and cross attention to an encoder's states.

kind     rotate   one call that turns a tensor of queries or keys by the positions of its tokens (or back: the gradient)
         image    one image (batch): for every scale and layer append K and V -- with `rope` the keys and queries are turned
                  on the way --, then attend; with `export` the cache is read back at the end, as a snapshot is taken
         cross    one call of attention from a step's queries to an encoder's states of other lengths
dtype    of image: "kv8" bf16 tensors and a cache in 8 bits, "bf16", "f32"
sides    "HxW HxW ..." of the scales, coarse to fine
policy   "c w" for every layer (condensed scales, window), "all", or "ragged" (c and w drawn per layer)
fast     PLANNED slots, unretained scales read in place (where nothing is turned); else the compacting, copying form
packed   token-major tensors: Q, K, V are read from one projection output [B][T][3][H*D]
rope     "", or "pairing axes rot_dim" with pairing half or interleaved
stretch  long-context factor of the rotary frequencies (1: none); above 1 the fast pairs keep their frequency
"""
import math
import random

import torch

own = False
amskv = None

VAR = "1x1 2x2 3x3 4x4 5x5 6x6 8x8 10x10 13x13 16x16"
INFINITY = "1x1 2x2 4x4 6x6 8x8 12x12 16x16 20x20 24x24 32x32 40x40 48x48 64x64"
BASE = 10000.0
TRAINED = 4096.0   # positions the frequencies were trained on, where they are stretched
BLOCK = 16         # tokens that share a scale in the cache of 8 bits


def _rotate(name, **k):
    base = {"name": name, "kind": "rotate", "batch": 1, "heads": 16, "tokens": 1, "head_dim": 64, "dtype": "bf16",
            "rope": "half 1 64", "stretch": 1.0, "each": False, "far": 0, "packed": False, "inverse": False}
    base.update(k)
    return base


def _image(name, **k):
    base = {"name": name, "kind": "image", "sides": VAR, "layers": 1, "batch": 1, "heads": 16, "head_dim": 64,
            "dtype": "kv8", "policy": "2 2", "fast": False, "packed": False, "rope": "", "stretch": 1.0, "export": False}
    base.update(k)
    return base


def _cross(name, **k):
    base = {"name": name, "kind": "cross", "batch": 2, "heads": 16, "kv_heads": 16, "head_dim": 64, "queries": 1,
            "keys": 64, "lengths": "ragged", "packed": False}
    base.update(k)
    return base


def listed():
    return [
        # one new token of each of 32 requests, each at its own far position: all latency
        _rotate("rotate tokens of 32 requests", batch=32, tokens=1, head_dim=128, rope="half 1 128", stretch=8.0, each=True,
                far=1000000),
        # the queries of the last scale of 1024x1024 images, out of the fused projection, by row and column
        _rotate("rotate 64x64 grid", batch=8, tokens=4096, head_dim=128, rope="interleaved 2 128", packed=True),
        # gradient of turned keys in fp32, half the head turned, an odd grid
        _rotate("rotate back f32", batch=12, heads=30, tokens=169, dtype="f32", rope="half 2 32", inverse=True),
        # one layer on one image with the 8-bit cache: the smallest unit of work
        _image("8 bit layer b1"),
        # throughput sampling, the last scale read in place
        _image("8 bit d30 b128", layers=4, batch=128, heads=30, fast=True),
        # policies of different layers, copying and compacting, the head turned in part
        _image("8 bit d24 ragged b40 rotary", layers=6, batch=40, heads=24, policy="ragged", rope="half 1 48", stretch=4.0,
               export=True),
        # 1024x1024 images: matrix-bound attention over 8-bit keys, positions by row and column, fused projections
        _image("8 bit infinity b4 rotary", layers=2, batch=4, head_dim=128, sides=INFINITY, policy="3 1", packed=True,
               rope="interleaved 2 128"),
        # positions with the ordinary cache, as a stack of layers makes them
        _image("bf16 stack b16 rotary", layers=8, batch=16, dtype="bf16", policy="all", rope="half 2 64", export=True),
        # the first scale's queries to a short prompt
        _cross("cross first scale", keys=77),
        # a mid scale at a large batch, prompts of every length, some empty
        _cross("cross 10x10 b96", batch=96, queries=100, keys=250),
        # the last scale of 1024x1024 images to packed prompts
        _cross("cross 64x64 b8 packed", batch=8, head_dim=128, queries=4096, keys=512, packed=True),
        # one query per request to a long document, four query heads to a key head
        _cross("cross one query, long", batch=8, heads=32, kv_heads=8, head_dim=128, keys=16000, lengths="long"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_sides(rng, most):
    """Scales that grow to a grid of any side and aspect, in any number of steps."""
    n = rng.randint(4, 13)
    h, w = _log(rng, 6, most), _log(rng, 6, most)
    if max(h, w) > 3 * min(h, w):
        h = w
    bend = rng.uniform(1.0, 1.6)
    out = []
    for i in range(n):
        f = (i / (n - 1)) ** bend
        out.append((max(1, round(1 + (h - 1) * f)), max(1, round(1 + (w - 1) * f))))
    return " ".join("%dx%d" % x for x in out)


def draw(rng):
    dearest = max(_cost(c) for c in listed())
    while True:
        kind = rng.choice(["rotate", "image", "image", "cross", "cross"])
        dim = rng.choice([64, 128])
        rope = "%s %d %d" % (rng.choice(["half", "interleaved"]), rng.choice([1, 2]), 16 * rng.randint(1, dim // 16))
        stretch = rng.choice([1.0, 1.0, rng.uniform(1.5, 32.0)])
        if kind == "rotate":
            c = _rotate("", batch=_log(rng, 1, 128), heads=rng.randint(1, 32), tokens=_log(rng, 1, 4096), head_dim=dim,
                        dtype=rng.choice(["bf16", "bf16", "f32"]), rope=rope, stretch=stretch, each=rng.random() < 0.3,
                        far=rng.choice([0, 1000000]), packed=rng.random() < 0.4, inverse=rng.random() < 0.3)
        elif kind == "image":
            dtype = rng.choice(["kv8"] * 4 + ["bf16", "f32"])
            fast = dtype == "kv8" and rng.random() < 0.4
            c = _image("", sides=rng.choice([VAR, "", ""]) or _draw_sides(rng, 40), layers=_log(rng, 1, 12),
                       batch=_log(rng, 1, 128), heads=rng.randint(2, 32), head_dim=dim, dtype=dtype, fast=fast,
                       policy=rng.choice(["%d %d" % (rng.randint(1, 3), rng.randint(1, 4)), "ragged", "all"]),
                       packed=rng.random() < 0.4, export=rng.random() < 0.4)
            if dtype != "kv8" or (not fast and rng.random() < 0.6):
                c.update(rope=rope, stretch=stretch)
        else:
            kv = rng.randint(1, 16)
            c = _cross("", batch=_log(rng, 1, 128), heads=kv * rng.choice([1, 1, 1, 2, 4, 8]), kv_heads=kv, head_dim=dim,
                       queries=_log(rng, 1, 4096), keys=_log(rng, 1, 16000), lengths=rng.choice(["ragged", "ragged", "long", "full"]),
                       packed=rng.random() < 0.4)
        c.pop("name")
        if _cost(c) <= dearest and _elements(c) < 1.5e9:
            return c


# ---------------------------------------------------------------- what a case says
def _sides(case):
    return [tuple(int(x) for x in s.split("x")) for s in case["sides"].split()]


def _tokens(case):
    return [h * w for h, w in _sides(case)]


def _rope(case):
    """(pairing, axes, channels that turn) or None."""
    if not case["rope"]:
        return None
    pairing, axes, rot = case["rope"].split()
    return pairing, int(axes), int(rot)


def _policies(case):
    n, p = case["layers"], case["policy"]
    if p == "all":
        return [(0, 0, True)] * n
    if p == "ragged":
        r = random.Random(n)
        return [(r.randint(1, 3), r.randint(1, 4), False) for _ in range(n)]
    c, w = p.split()
    return [(int(c), int(w), False)] * n


def _kept(policy, s):
    c, w, everything = policy
    return [k for k in range(s + 1) if everything or k < c or s - k <= w]


def _in_place(case, policy, s):
    """A scale no later step reads is not stored where the caller lets it be read in place."""
    return case["fast"] and (s + 1 == len(_tokens(case)) or s not in _kept(policy, s + 1))


def _elements(case):
    """Elements of all inputs."""
    if case["kind"] == "rotate":
        return case["batch"] * case["heads"] * case["tokens"] * case["head_dim"] * (3 if case["packed"] else 1)
    if case["kind"] == "image":
        return 3 * case["layers"] * case["batch"] * case["heads"] * case["head_dim"] * sum(_tokens(case))
    return case["batch"] * case["head_dim"] * (case["heads"] * case["queries"] + 2 * case["kv_heads"] * case["keys"])


def _mean_length(case):
    return case["keys"] * {"ragged": 0.5, "long": 0.9, "full": 1.0}[case["lengths"]]


def work(case):
    B, H, D = case["batch"], case["heads"], case["head_dim"]
    if case["kind"] == "rotate":
        _, axes, rot = _rope(case)
        e = 2 if case["dtype"] == "bf16" else 4
        n = B * H * case["tokens"]
        return {"bytes": 2.0 * n * D * e + 4.0 * rot * case["tokens"] * (B if case["each"] else 1), "flops": 3.0 * n * rot}
    if case["kind"] == "cross":
        rows = B * _mean_length(case)
        return {"bytes": 2.0 * D * (2 * B * H * case["queries"] + 2 * case["kv_heads"] * rows),
                "flops": 4.0 * D * H * case["queries"] * rows}
    # every call's operands once: the new scale's K, V (and Q, where it is turned) in, their turned and cached forms out;
    # then Q and the kept keys and values in, O out
    unit, e = B * H * D, 4 if case["dtype"] == "f32" else 2
    held = 1 + 1.0 / (BLOCK * D) if case["dtype"] == "kv8" else e
    size = flops = 0.0
    t = _tokens(case)
    for policy in _policies(case):
        for s in range(len(t)):
            keys = _kept(policy, s)
            place = _in_place(case, policy, s)
            if not place:
                size += unit * t[s] * 2 * (e + held)
            if case["rope"]:
                size += unit * t[s] * 2 * e
            size += unit * 2 * (t[s] * e + sum(t[k] for k in keys[:-1]) * held + t[s] * (e if place else held))
            flops += 4.0 * unit * t[s] * sum(t[k] for k in keys)
        if case["export"]:
            size += unit * 2 * (held + e) * sum(t[k] for k in _kept(policy, len(t) - 1))
    return {"bytes": size, "flops": flops}


def _cost(case):
    w = work(case)
    calls = case["layers"] * len(_tokens(case)) if case["kind"] == "image" else 1
    return w["bytes"] / 4e12 + w["flops"] / 4e14 + 1e-5 * calls


# ---------------------------------------------------------------- inputs
def _dtype(case):
    return torch.float32 if case["dtype"] == "f32" else torch.bfloat16


def _gains(shape, g):
    """Channels of different strength, as keys have them."""
    return torch.exp(0.4 * torch.randn(shape, generator=g, device="cuda"))


def _positions(case, tokens, hw, first):
    """fp64 [tokens, axes]: along the sequence, or row and column on the grid of the last scale."""
    axes = _rope(case)[1]
    t = torch.arange(tokens, dtype=torch.float64, device="cuda")
    if axes == 1:
        return (first + t)[:, None]
    h, w, top_h, top_w = hw
    return torch.stack((torch.floor(t / w) * (top_h / h), torch.remainder(t, w) * (top_w / w)), dim=1)


def _grid(tokens):
    """The squarest grid of that many tokens."""
    h = next(x for x in range(int(math.isqrt(tokens)), 0, -1) if tokens % x == 0)
    return h, tokens // h, h, tokens // h


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    B, H, D = case["batch"], case["heads"], case["head_dim"]
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    if case["kind"] == "rotate":
        n = case["tokens"]
        x = normal(B, n, 3, H, D)[:, :, 1] if case["packed"] else normal(B, H, n, D) * _gains((H, 1, D), g)
        where = []
        for b in range(B if case["each"] else 1):
            first = int(torch.randint(0, case["far"] + 1, (1,), generator=g, device="cuda")) if case["far"] else 0
            where.append(_positions(case, n, _grid(n), float(first)) + (first if _rope(case)[1] == 2 else 0))
        if case["packed"]:   # the tensor a fused projection leaves; its keys are what is turned
            whole = torch.zeros(B, n, 3, H, D, device="cuda")
            whole[:, :, 1] = x
            x = whole
        return {"x": x.to(_dtype(case)), "where": torch.stack(where)}
    if case["kind"] == "cross":
        if case["lengths"] == "full":
            lengths = torch.full((B,), case["keys"], device="cuda")
        elif case["lengths"] == "long":
            lengths = torch.randint(case["keys"] - case["keys"] // 5, case["keys"] + 1, (B,), generator=g, device="cuda")
        else:
            lengths = torch.randint(0, case["keys"] + 1, (B,), generator=g, device="cuda")
        q = normal(B, H, case["queries"], D).to(torch.bfloat16)
        rows = int(lengths.sum()) if case["packed"] else B * case["keys"]
        k, v = ((normal(max(rows, 1), case["kv_heads"], D) * _gains((case["kv_heads"], D), g)).to(torch.bfloat16) for _ in range(2))
        if not case["packed"]:
            k, v = (x.view(B, case["keys"], case["kv_heads"], D) for x in (k, v))
        offsets = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
        offsets[1:] = torch.cumsum(lengths, 0)
        return {"q": q, "k": k, "v": v, "lengths": lengths.to(torch.int32), "offsets": offsets}
    layers = []
    for _ in range(case["layers"]):
        gk, q, k, v = _gains((H, 1, D), g), [], [], []
        for t in _tokens(case):
            x = torch.stack((normal(B, H, t, D), normal(B, H, t, D) * gk, normal(B, H, t, D)))
            if case["packed"]:
                x = x.permute(1, 3, 0, 2, 4).reshape(B, t, 3, H * D).to(_dtype(case)).contiguous()
                q.append(x[:, :, 0]), k.append(x[:, :, 1]), v.append(x[:, :, 2])
            else:
                x = x.to(_dtype(case))
                q.append(x[0]), k.append(x[1]), v.append(x[2])
        layers.append((q, k, v))
    where = []
    if case["rope"]:
        sides, first = _sides(case), 0
        for h, w in sides:
            where.append(_positions(case, h * w, (h, w) + sides[-1], float(first)))
            first += h * w
    return {"layers": layers, "where": where}


# ---------------------------------------------------------------- the plain forms
def _frequencies(case):
    """fp64, one per pair of an axis."""
    _, axes, rot = _rope(case)
    n = rot // 2 // axes
    f = BASE ** (-torch.arange(n, dtype=torch.float64, device="cuda") / n)
    if case["stretch"] > 1:
        turns = TRAINED * f / (2 * math.pi)
        keep = torch.clamp((turns - 1.0) / 31.0, 0.0, 1.0)
        f = f * (keep + (1 - keep) / case["stretch"])
    return f


def _amplitude(case):
    return 1.0 if case["stretch"] == 1 else 0.1 * math.log(case["stretch"]) + 1.0


def _plain_table(case, where):
    """[..., tokens, pairs, 2]: cosine and sine of every pair's angle, formed in 64 bits."""
    angles = (where[..., None] * _frequencies(case)).flatten(-2)
    return (_amplitude(case) * torch.stack((torch.cos(angles), torch.sin(angles)), dim=-1)).float()


def _turn(case, x, table, back=False):
    """x [..., tokens, D] in the type it is computed in; table [..., tokens, pairs, 2] broadcasts against it."""
    pairing, _, rot = _rope(case)
    c, s = table[..., 0], table[..., 1]
    if back:
        s = -s
    head, rest = x[..., :rot], x[..., rot:]
    if pairing == "half":
        a, b = head[..., : rot // 2], head[..., rot // 2:]
        return torch.cat((a * c - b * s, b * c + a * s, rest), dim=-1)
    a, b = head[..., 0::2], head[..., 1::2]
    return torch.cat((torch.stack((a * c - b * s, b * c + a * s), dim=-1).flatten(-2), rest), dim=-1)


def _power(e):
    """2^e in fp32, from its bits."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _e4m3(x):
    """The nearest e4m3 number (3 bits behind the point, least exponent -6, at most 448), ties to even."""
    _, e = torch.frexp(x)
    step = _power(torch.clamp(e - 1, min=-6) - 3)
    return torch.round(x / step) * step


def _held(x):
    """What a cache of 8 bits stands for, [B, H, t, D]: per 16 tokens and head e4m3 numbers times the least power of two that
    takes the largest of them."""
    B, H, t, D = x.shape
    pad = -t % BLOCK
    y = torch.cat((x, x.new_zeros(B, H, pad, D)), dim=2) if pad else x
    y = y.reshape(B, H, -1, BLOCK * D)
    m, e = torch.frexp(y.abs().amax(dim=-1, keepdim=True))
    e = torch.clamp(torch.where(m > 0.875, e - 8, e - 9), min=-100)
    scale = _power(e)
    return (_e4m3(y / scale) * scale).reshape(B, H, t + pad, D)[:, :, :t]


def _softmax_product(q, k, v, budget):
    """softmax(q k^T / sqrt(D)) v over [..., rows, D], a few units at a time so that the scores stay small."""
    units, t, d = q.shape
    out = torch.empty_like(q)
    step = max(1, budget // max(1, t * k.shape[1]))
    for i in range(0, units, step):
        x = torch.matmul(q[i:i + step], k[i:i + step].transpose(1, 2).contiguous()) * (1.0 / math.sqrt(d))
        x = torch.exp(x - x.amax(dim=-1, keepdim=True))
        out[i:i + step] = torch.matmul(x, v[i:i + step]) / x.sum(dim=-1, keepdim=True)
    return out


def _heads_first(case, x, t):
    """A scale's tensor as [B, H, t, D]."""
    if case["packed"]:
        return x.reshape(case["batch"], t, case["heads"], case["head_dim"]).permute(0, 2, 1, 3)
    return x


def _as_laid_out(case, x):
    """[..., B, H, t, D] as the caller's O is laid out."""
    if case["packed"]:
        return x.transpose(-3, -2).flatten(-2)
    return x


def _plain_image(case, state, tables, budget):
    B, H, D, dt = case["batch"], case["heads"], case["head_dim"], _dtype(case)
    t, n = _tokens(case), len(_tokens(case))
    outs = [[] for _ in t]
    snapshots = []
    for (q, k, v), policy in zip(state["layers"], _policies(case)):
        held = {}
        for s in range(n):
            qs, ks, vs = (_heads_first(case, x[s], t[s]).float() for x in (q, k, v))
            if case["rope"]:
                qs, ks = _turn(case, qs, tables[s]), _turn(case, ks, tables[s])
                qs = qs.to(dt).float()    # the turned queries are a tensor of the caller's
            if case["dtype"] == "kv8" and not _in_place(case, policy, s):
                ks, vs = _held(ks), _held(vs)
            elif case["dtype"] == "bf16":
                ks = ks.to(dt).float()    # and the cache holds 16 bits
            held = {i: held[i] for i in _kept(policy, s) if i < s}
            held[s] = (ks, vs)
            kk, vv = (torch.cat([held[i][j] for i in sorted(held)], dim=2).reshape(B * H, -1, D) for j in range(2))
            o = _softmax_product(qs.reshape(B * H, t[s], D), kk, vv, budget).view(B, H, t[s], D)
            outs[s].append(_as_laid_out(case, o))
        if case["export"]:
            snapshots.append(tuple(x.view(B, H, -1, D) for x in (kk, vv)))
    return {"o": [torch.stack(o) for o in outs], "held": snapshots}


def _plain_cross(case, state, budget):
    B, H, D, G, T = case["batch"], case["heads"], case["head_dim"], case["heads"] // case["kv_heads"], case["queries"]
    out = torch.zeros(state["q"].shape, dtype=torch.bfloat16, device="cuda")
    if case["packed"]:   # each request's rows by themselves
        first, last = state["starts"]
        for b in range(B):
            if first[b] == last[b]:
                continue   # no states: nothing is added
            k, v = (x[first[b]:last[b]].float().transpose(0, 1).contiguous() for x in (state["k"], state["v"]))
            q = state["q"][b].float().reshape(case["kv_heads"], G * T, D)
            out[b] = _softmax_product(q, k, v, budget).view(H, T, D).to(torch.bfloat16)
        return out
    step = max(1, budget // (H * T * case["keys"]))
    beyond = torch.arange(case["keys"], device="cuda") >= state["lengths"][:, None]
    for i in range(0, B, step):
        k, v = (x[i:i + step].float().transpose(1, 2).flatten(0, 1) for x in (state["k"], state["v"]))
        q = state["q"][i:i + step].float().reshape(-1, G * T, D)
        x = torch.matmul(q, k.transpose(1, 2).contiguous()) * (1.0 / math.sqrt(D))
        x = x.view(-1, case["kv_heads"], G * T, case["keys"]).masked_fill_(beyond[i:i + step, None, None], -math.inf)
        top = x.amax(dim=-1, keepdim=True)
        x = torch.exp(x - torch.where(top == -math.inf, 0.0, top))
        total = x.sum(dim=-1, keepdim=True)
        o = torch.matmul(x.flatten(0, 1), v).view_as(x[..., :1].expand(-1, -1, -1, D)) / torch.where(total == 0, 1.0, total)
        out[i:i + step] = o.view(-1, H, T, D).to(torch.bfloat16)
    return out


# ---------------------------------------------------------------- state and pass
class _Cache:
    """The handle a program keeps, and the arena it lives in."""

    def __init__(self, case):
        hs, ws = zip(*_sides(case))
        dtype = {"kv8": amskv.AMSKV_DTYPE_BF16_KV8, "bf16": amskv.AMSKV_DTYPE_BF16, "f32": amskv.AMSKV_DTYPE_F32}[case["dtype"]]
        args = (case["layers"], case["heads"], case["head_dim"], hs, ws, case["batch"], dtype, _policies(case))
        kw = {"layout": amskv.AMSKV_LAYOUT_PLANNED, "borrow_unretained": True} if case["fast"] else {}
        self.arena = torch.empty(amskv.amskv_cache_required_bytes(*args, **kw), dtype=torch.uint8, device="cuda")
        self.handle = amskv.amskv_cache_create(*args, arena=self.arena, **kw)
        if case["packed"]:
            width = case["heads"] * case["head_dim"]
            amskv.amskv_cache_set_io_layout(self.handle, amskv.AMSKV_IO_TOKEN_MAJOR, width if case["rope"] else 3 * width, 3 * width, width)

    def __del__(self):
        if getattr(self, "handle", None) and amskv and amskv.amskv_cache_destroy:   # (gone at interpreter exit)
            amskv.amskv_cache_destroy(self.handle)


def _own_rope(case):
    pairing, axes, rot = _rope(case)
    stretched = case["stretch"] > 1
    return amskv.Rope(rot_dim=rot, pairing=amskv.AMSKV_ROPE_HALF if pairing == "half" else amskv.AMSKV_ROPE_INTERLEAVED, axes=axes,
                      base=BASE, factor=case["stretch"], original=TRAINED, low=1.0 if stretched else 0.0,
                      high=32.0 if stretched else 0.0, amplitude=_amplitude(case))


def _table(case, where):
    if not own:
        return _plain_table(case, where)
    flat = where.reshape(-1, where.shape[-1]).contiguous()
    table = torch.empty(*where.shape[:-1], _rope(case)[2] // 2, 2, device="cuda")
    amskv.amskv_rope_table(_own_rope(case), flat, table)
    return table


def prepare(case, seed):
    global amskv
    if own and amskv is None:
        import paper_2511_16047_amd
        amskv = paper_2511_16047_amd
    state = dict(_inputs(case, seed), case=case)
    B, H, D = case["batch"], case["heads"], case["head_dim"]
    # a program keeps one table for each scale, or for the positions its requests stand at
    if case["kind"] == "rotate":
        state["table"] = _table(case, state["where"])
    elif case["kind"] == "image":
        state["tables"] = [_table(case, w) for w in state["where"]]
    else:   # where each request's states begin and end; a program that packs them knows it on the host as well
        lengths = state["lengths"].tolist()
        first = state["offsets"].tolist()[:-1]
        state["starts"] = first, [f + n for f, n in zip(first, lengths)]
    if not own:
        return state
    if case["kind"] == "rotate":
        state["rope"], state["out"] = _own_rope(case), torch.empty_like(state["x"][:, :, 1] if case["packed"] else state["x"],
                                                                        memory_format=torch.contiguous_format)
    elif case["kind"] == "cross":
        k = state["k"]
        rows = k.stride(0) if case["packed"] else k.stride(1)
        kv = amskv.Strides(0 if case["packed"] else k.stride(0), D, rows)
        head = amskv.Strides(H * case["queries"] * D, case["queries"] * D, D)
        state["cross"] = amskv.Cross(batch=B, heads=H, kv_heads=case["kv_heads"], head_dim=D, dtype=amskv.AMSKV_DTYPE_BF16,
                                     q_tokens=case["queries"], kv_tokens=case["keys"], kv_rows=k.shape[0] if case["packed"] else 0,
                                     q=head, k=kv, v=kv, o=head)
        state["out"] = torch.empty_like(state["q"])
        need = amskv.amskv_cross_workspace_bytes(state["cross"])
        state["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    else:
        L, t = case["layers"], _tokens(case)
        state["cache"] = _Cache(case)
        state["rope"] = _own_rope(case) if case["rope"] else None
        shape = (lambda x: (L, B, x, H * D)) if case["packed"] else (lambda x: (L, B, H, x, D))
        state["out"] = [torch.empty(shape(x), dtype=_dtype(case), device="cuda") for x in t]
        state["turned"] = [torch.empty(shape(x)[1:], dtype=_dtype(case), device="cuda") for x in t]
        state["held"] = [tuple(torch.empty(B, H, sum(t[k] for k in _kept(p, len(t) - 1)), D, dtype=_dtype(case), device="cuda")
                               for _ in range(2)) for p in _policies(case)] if case["export"] else []
    return state


def run(state):
    case = state["case"]
    return _run_own(case, state) if own else _run_plain(case, state)


def _run_plain(case, state):
    if case["kind"] == "rotate":
        x = state["x"][:, :, 1] if case["packed"] else state["x"]
        table = state["table"]                                           # [1 or B, tokens, pairs, 2]
        table = table[:, :, None] if case["packed"] else table[:, None]  # one for all heads
        return _turn(case, x.float(), table, case["inverse"]).to(_dtype(case))
    if case["kind"] == "cross":
        return _plain_cross(case, state, 2 ** 30)
    out = _plain_image(case, state, state["tables"], 2 ** 30)
    return {"o": [o.to(_dtype(case)) for o in out["o"]], "held": [tuple(x.to(_dtype(case)) for x in p) for p in out["held"]]}


def _run_own(case, state):
    B, H, D = case["batch"], case["heads"], case["head_dim"]
    if case["kind"] == "rotate":
        n, x = case["tokens"], state["x"]
        if case["packed"]:
            x = x[:, :, 1]
            xs, os = amskv.Strides(3 * n * H * D, D, 3 * H * D), amskv.Strides(n * H * D, D, H * D)
        else:
            xs = os = amskv.Strides(H * n * D, n * D, D)
        pairs = state["table"].shape[2]
        amskv.amskv_rotate(state["rope"], amskv.AMSKV_DTYPE_F32 if case["dtype"] == "f32" else amskv.AMSKV_DTYPE_BF16, D, B, H, n,
                           state["table"], n * pairs * 2 if case["each"] else 0, x, xs, state["out"], os, inverse=case["inverse"])
        return state["out"]
    if case["kind"] == "cross":
        amskv.amskv_cross_attend(state["cross"], state["q"], state["k"], state["v"], state["out"],
                                 lengths=None if case["packed"] or case["lengths"] == "full" else state["lengths"],
                                 offsets=state["offsets"] if case["packed"] else None, workspace=state["workspace"])
        return state["out"]
    handle, rope, turned, tables = state["cache"].handle, state["rope"], state["turned"], state["tables"]
    width = H * D
    amskv.amskv_cache_reset(handle)
    for s in range(len(turned)):
        for l, (q, k, v) in enumerate(state["layers"]):
            if rope is None:
                amskv.amskv_append_scale(handle, l, s, k[s], v[s])
                amskv.amskv_attend(handle, l, s, q[s], state["out"][s][l])
            else:
                amskv.amskv_append_scale_rotary(handle, l, s, rope, tables[s], q[s], 3 * width if case["packed"] else 0, turned[s], k[s], v[s])
                amskv.amskv_attend(handle, l, s, turned[s], state["out"][s][l])
    for l, (k, v) in enumerate(state["held"]):
        amskv.amskv_cache_export(handle, l, k, v)
    return {"o": state["out"], "held": state["held"]}


# ---------------------------------------------------------------- the definitions in 64 bits
def exact(case, seed):
    x = _inputs(case, seed)
    wide = torch.float64

    def turned(t, where, back):
        pairing, axes, rot = _rope(case)
        y = t.clone()
        n = rot // 2 // axes
        for i in range(rot // 2):   # pair by pair, as the definition has it
            f = BASE ** (-(i % n) / n)
            if case["stretch"] > 1:
                ramp = min(1.0, max(0.0, (TRAINED * f / (2 * math.pi) - 1.0) / 31.0))
                f = f * ramp + f / case["stretch"] * (1.0 - ramp)
            angle = where[..., i // n] * f
            c, s = _amplitude(case) * torch.cos(angle), _amplitude(case) * torch.sin(angle) * (-1.0 if back else 1.0)
            a, b = (i, i + rot // 2) if pairing == "half" else (2 * i, 2 * i + 1)
            y[..., a] = t[..., a] * c - t[..., b] * s
            y[..., b] = t[..., a] * s + t[..., b] * c
        return y

    def two(e):   # 2^e
        return ((e.long() + 1023) << 52).view(wide)

    def in_8_bits(t):
        B, H, n, D = t.shape
        y = torch.zeros(B, H, (n + BLOCK - 1) // BLOCK * BLOCK, D, dtype=wide, device=t.device)
        y[:, :, :n] = t
        y = y.view(B, H, -1, BLOCK, D)
        top = y.abs().amax(dim=(3, 4), keepdim=True)
        e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -300) / 448.0)).clamp(min=-100)
        e = torch.where(top > 448.0 * two(e), e + 1, e)             # log2 next to a power of two
        e = torch.where((top <= 448.0 * two(e - 1)) & (e > -100), e - 1, e)
        z = y / two(e)
        small = two(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))))
        small = torch.where(z.abs() < small, small / 2, torch.where(z.abs() >= 2 * small, 2 * small, small)).clamp(min=2.0 ** -6)
        z = torch.round(z * 8 / small) * small / 8
        return (z * two(e)).view(B, H, -1, D)[:, :, :n]

    def attention(q, k, v):
        out = torch.empty_like(q)
        step = max(1, 2 ** 28 // (q.shape[1] * k.shape[1]))
        for i in range(0, q.shape[0], step):
            s = torch.bmm(q[i:i + step], k[i:i + step].transpose(1, 2).contiguous()) / math.sqrt(q.shape[-1])
            p = torch.exp(s - s.max(dim=2, keepdim=True).values)
            out[i:i + step] = torch.bmm(p / p.sum(dim=2, keepdim=True), v[i:i + step])
        return out

    B, H, D = case["batch"], case["heads"], case["head_dim"]
    if case["kind"] == "rotate":
        if case["packed"]:
            return turned(x["x"][:, :, 1].to(wide), x["where"][:, :, None], case["inverse"])
        return turned(x["x"].to(wide), x["where"][:, None], case["inverse"])
    if case["kind"] == "cross":
        out = torch.zeros(x["q"].shape, dtype=wide, device="cuda")
        ends, lengths, share = x["offsets"].tolist(), x["lengths"].tolist(), H // case["kv_heads"]
        for b in range(B):
            n = lengths[b]
            if n:
                k, v = ((t[ends[b]:ends[b] + n] if case["packed"] else t[b, :n]).to(wide).permute(1, 0, 2) for t in (x["k"], x["v"]))
                of = torch.arange(H, device="cuda") // share
                for h in range(0, H, share):   # the heads that read one key head
                    one = slice(of[h].item(), of[h].item() + 1)
                    out[b, h:h + share] = attention(x["q"][b, h:h + share].to(wide).reshape(1, -1, D), k[one].contiguous(),
                                                    v[one].contiguous()).view(share, -1, D)
        return out
    t = _tokens(case)
    result = {"o": [torch.empty((case["layers"], B, n, H * D) if case["packed"] else (case["layers"], B, H, n, D), dtype=wide,
                                device="cuda") for n in t], "held": []}
    for l, ((q, k, v), policy) in enumerate(zip(x["layers"], _policies(case))):
        keys, values = {}, {}
        for s, n in enumerate(t):
            a, b, c = ((y[s].reshape(B, n, H, D).transpose(1, 2) if case["packed"] else y[s]).to(wide) for y in (q, k, v))
            if case["rope"]:
                a, b = turned(a, x["where"][s], False), turned(b, x["where"][s], False)
                a = a.to(_dtype(case)).to(wide)
            if case["dtype"] == "kv8" and not _in_place(case, policy, s):
                b, c = in_8_bits(b), in_8_bits(c)
            if case["dtype"] == "bf16":
                b = b.to(_dtype(case)).to(wide)
            keys[s], values[s] = b, c
            now = _kept(policy, s)
            for old in [i for i in keys if i not in now]:
                del keys[old], values[old]
            kk, vv = (torch.cat([d[i] for i in now], dim=2) for d in (keys, values))
            o = attention(a.reshape(B * H, n, D), kk.reshape(B * H, -1, D), vv.reshape(B * H, -1, D)).view(B, H, n, D)
            result["o"][s][l] = o.transpose(1, 2).reshape(B, n, H * D) if case["packed"] else o
        if case["export"]:
            result["held"].append((kk, vv))
    return result
