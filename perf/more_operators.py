"""K and V held in 4 bits, as cases that can be timed and compared: the scale cache written, attended and read back, and an
encoder's states, which every step of a model with cross attention reads again.

kind     image    one image (batch): for every scale and layer append K and V -- with `rope` the keys and queries are turned
                  on the way --, then attend; with `export` the cache is read back at the end, as a snapshot is taken
         hold     an encoder's K and V put into 4 bits, and read back
         cross    one call of attention from a step's queries to an encoder's states that are held in 4 bits
sides    "HxW HxW ..." of the scales, coarse to fine
policy   "c w" for every layer (condensed scales, window), "all", or "ragged" (c and w drawn per layer)
fast     PLANNED slots, unretained scales read in place (where nothing is turned); else the compacting, copying form
packed   image: token-major tensors, Q, K, V are read from one projection output [B][T][3][H*D]; hold, cross: the states of
         all batch elements back to back
rope     "", or "pairing axes rot_dim" with pairing half or interleaved
stretch  long-context factor of the rotary frequencies (1: none); above 1 the fast pairs keep their frequency
lengths  of the states: "ragged" (0 to the most), "long" (the last fifth), "full"
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
GROUP = 32         # channels of a token that share a power of two


def _image(name, **k):
    base = {"name": name, "kind": "image", "sides": VAR, "layers": 1, "batch": 1, "heads": 16, "head_dim": 64,
            "policy": "2 2", "fast": False, "packed": False, "rope": "", "stretch": 1.0, "export": False}
    base.update(k)
    return base


def _hold(name, **k):
    base = {"name": name, "kind": "hold", "batch": 2, "kv_heads": 16, "head_dim": 64, "keys": 64, "lengths": "ragged",
            "packed": False}
    base.update(k)
    return base


def _cross(name, **k):
    base = {"name": name, "kind": "cross", "batch": 2, "heads": 16, "kv_heads": 16, "head_dim": 64, "queries": 1,
            "keys": 64, "lengths": "ragged", "packed": False}
    base.update(k)
    return base


def listed():
    return [
        # one layer on one image: the smallest unit of work, all latency
        _image("4 bit layer b1"),
        # throughput sampling, the last scale read in place
        _image("4 bit d30 b128", layers=4, batch=128, heads=30, fast=True),
        # policies of different layers, copying and compacting, the head turned in part, a snapshot at the end
        _image("4 bit d24 ragged b40 rotary", layers=6, batch=40, heads=24, policy="ragged", rope="half 1 48", stretch=4.0,
               export=True),
        # 1024x1024 images: matrix-bound attention over 4-bit keys, positions by row and column, fused projections
        _image("4 bit infinity b4 rotary", layers=2, batch=4, head_dim=128, sides=INFINITY, policy="3 1", packed=True,
               rope="interleaved 2 128"),
        # a stack of layers that keep everything, one prompt's worth of images
        _image("4 bit stack b16", layers=8, batch=16, policy="all", export=True),
        # the states of a short prompt
        _hold("hold a short prompt", keys=77),
        # the prompts of a batch, back to back, some empty
        _hold("hold packed prompts b96", batch=96, keys=512, head_dim=128, packed=True),
        # long documents, eight key heads
        _hold("hold long documents", batch=8, kv_heads=8, head_dim=128, keys=16000, lengths="long"),
        # the first scale's queries to a short prompt
        _cross("4 bit cross first scale", keys=77),
        # a mid scale at a large batch, prompts of every length, some empty
        _cross("4 bit cross 10x10 b96", batch=96, queries=100, keys=250),
        # the last scale of 1024x1024 images to packed prompts
        _cross("4 bit cross 64x64 b8 packed", batch=8, head_dim=128, queries=4096, keys=512, packed=True),
        # one query per request to a long document, four query heads to a key head
        _cross("4 bit cross one query, long", batch=8, heads=32, kv_heads=8, head_dim=128, keys=16000, lengths="long"),
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
        kind = rng.choice(["image", "image", "image", "hold", "cross", "cross"])
        dim = rng.choice([64, 128])
        if kind == "image":
            fast = rng.random() < 0.4
            c = _image("", sides=rng.choice([VAR, "", ""]) or _draw_sides(rng, 40), layers=_log(rng, 1, 12),
                       batch=_log(rng, 1, 128), heads=rng.randint(2, 32), head_dim=dim, fast=fast,
                       policy=rng.choice(["%d %d" % (rng.randint(1, 3), rng.randint(1, 4)), "ragged", "all"]),
                       packed=rng.random() < 0.4, export=rng.random() < 0.4)
            if not fast and rng.random() < 0.6:
                c.update(rope="%s %d %d" % (rng.choice(["half", "interleaved"]), rng.choice([1, 2]), 16 * rng.randint(1, dim // 16)),
                         stretch=rng.choice([1.0, 1.0, rng.uniform(1.5, 32.0)]))
        else:
            kv = rng.randint(1, 16)
            shape = dict(batch=_log(rng, 1, 128), kv_heads=kv, head_dim=dim, keys=_log(rng, 1, 16000),
                         lengths=rng.choice(["ragged", "ragged", "long", "full"]), packed=rng.random() < 0.4)
            if kind == "hold":
                c = _hold("", **shape)
            else:
                c = _cross("", heads=kv * rng.choice([1, 1, 1, 2, 4, 8]), queries=_log(rng, 1, 4096), **shape)
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
    if case["kind"] == "image":
        return 3 * case["layers"] * case["batch"] * case["heads"] * case["head_dim"] * sum(_tokens(case))
    queries = case["heads"] * case["queries"] if case["kind"] == "cross" else 0
    return case["batch"] * case["head_dim"] * (queries + 2 * case["kv_heads"] * case["keys"])


def _mean_length(case):
    return case["keys"] * {"ragged": 0.5, "long": 0.9, "full": 1.0}[case["lengths"]]


def work(case):
    B, D = case["batch"], case["head_dim"]
    held = 0.5 + 1.0 / GROUP   # bytes of an element in 4 bits, with its share of a power of two
    if case["kind"] != "image":
        rows = B * _mean_length(case)
        kv = 2.0 * D * case["kv_heads"] * rows
        if case["kind"] == "hold":   # bf16 in, 4 bits out; 4 bits in, bf16 out
            return {"bytes": kv * 2 * (2 + held), "flops": 4.0 * kv}
        H = case["heads"]
        return {"bytes": 2.0 * D * 2 * B * H * case["queries"] + kv * held, "flops": 4.0 * D * H * case["queries"] * rows}
    # every call's operands once: the new scale's K, V (and Q, where it is turned) in, their turned and cached forms out;
    # then Q and the kept keys and values in, O out
    unit = B * case["heads"] * D
    size = flops = 0.0
    t = _tokens(case)
    for policy in _policies(case):
        for s in range(len(t)):
            keys = _kept(policy, s)
            place = _in_place(case, policy, s)
            if not place:
                size += unit * t[s] * 2 * (2 + held)
            if case["rope"]:
                size += unit * t[s] * 2 * 2
            size += unit * 2 * (t[s] * 2 + sum(t[k] for k in keys[:-1]) * held + t[s] * (2 if place else held))
            flops += 4.0 * unit * t[s] * sum(t[k] for k in keys)
        if case["export"]:
            size += unit * 2 * (held + 2) * sum(t[k] for k in _kept(policy, len(t) - 1))
    return {"bytes": size, "flops": flops}


def _cost(case):
    w = work(case)
    calls = case["layers"] * len(_tokens(case)) if case["kind"] == "image" else 1
    return w["bytes"] / 4e12 + w["flops"] / 4e14 + 1e-5 * calls


# ---------------------------------------------------------------- inputs
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


def _inputs(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    B, D = case["batch"], case["head_dim"]
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")
    if case["kind"] != "image":
        if case["lengths"] == "full":
            lengths = torch.full((B,), case["keys"], device="cuda")
        elif case["lengths"] == "long":
            lengths = torch.randint(case["keys"] - case["keys"] // 5, case["keys"] + 1, (B,), generator=g, device="cuda")
        else:
            lengths = torch.randint(0, case["keys"] + 1, (B,), generator=g, device="cuda")
        # (an axis of packed states is as long as it may have to be, or as its states)
        rows = int(lengths.sum()) if case["packed"] and case["kind"] == "cross" else B * case["keys"]
        k, v = ((normal(max(rows, 1), case["kv_heads"], D) * _gains((case["kv_heads"], D), g)).to(torch.bfloat16) for _ in range(2))
        if not case["packed"]:
            k, v = (x.view(B, case["keys"], case["kv_heads"], D) for x in (k, v))
        offsets = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
        offsets[1:] = torch.cumsum(lengths, 0)
        out = {"k": k, "v": v, "lengths": lengths.to(torch.int32), "offsets": offsets}
        if case["kind"] == "cross":
            out["q"] = normal(B, case["heads"], case["queries"], D).to(torch.bfloat16)
        return out
    H = case["heads"]
    layers = []
    for _ in range(case["layers"]):
        gk, q, k, v = _gains((H, 1, D), g), [], [], []
        for t in _tokens(case):
            x = torch.stack((normal(B, H, t, D), normal(B, H, t, D) * gk, normal(B, H, t, D)))
            if case["packed"]:
                x = x.permute(1, 3, 0, 2, 4).reshape(B, t, 3, H * D).to(torch.bfloat16).contiguous()
                q.append(x[:, :, 0]), k.append(x[:, :, 1]), v.append(x[:, :, 2])
            else:
                x = x.to(torch.bfloat16)
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


def _turn(case, x, table):
    """x [..., tokens, D] in the type it is computed in; table [..., tokens, pairs, 2] broadcasts against it."""
    pairing, _, rot = _rope(case)
    c, s = table[..., 0], table[..., 1]
    head, rest = x[..., :rot], x[..., rot:]
    if pairing == "half":
        a, b = head[..., : rot // 2], head[..., rot // 2:]
        return torch.cat((a * c - b * s, b * c + a * s, rest), dim=-1)
    a, b = head[..., 0::2], head[..., 1::2]
    return torch.cat((torch.stack((a * c - b * s, b * c + a * s), dim=-1).flatten(-2), rest), dim=-1)


def _power(e):
    """2^e in fp32, from its bits."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _e2m1(x):
    """The nearest e2m1 number (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives), ties to even."""
    _, e = torch.frexp(x)
    step = _power(torch.clamp(e - 1, min=0) - 1)
    return torch.clamp(torch.round(x / step) * step, -6.0, 6.0)


def _held(x):
    """What 4 bits stand for, [..., D] in fp32: per row and 32 channels e2m1 numbers times the least power of two that takes the
    largest of them to 7 or less (what lies between 6 and 7 is next to 6)."""
    y = x.unflatten(-1, (-1, GROUP))
    m, e = torch.frexp(y.abs().amax(dim=-1, keepdim=True))
    scale = _power(torch.clamp(torch.where(m > 0.875, e - 2, e - 3), min=-100, max=125))
    return (_e2m1(y / scale) * scale).flatten(-2)


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
    B, H, D = case["batch"], case["heads"], case["head_dim"]
    t, n = _tokens(case), len(_tokens(case))
    outs = [[] for _ in t]
    snapshots = []
    for (q, k, v), policy in zip(state["layers"], _policies(case)):
        held = {}
        for s in range(n):
            qs, ks, vs = (_heads_first(case, x[s], t[s]).float() for x in (q, k, v))
            if case["rope"]:
                qs, ks = _turn(case, qs, tables[s]), _turn(case, ks, tables[s])
                qs = qs.to(torch.bfloat16).float()    # the turned queries are a tensor of the caller's
            if not _in_place(case, policy, s):
                ks, vs = _held(ks), _held(vs)
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
        args = (case["layers"], case["heads"], case["head_dim"], hs, ws, case["batch"], amskv.AMSKV_DTYPE_BF16_KV4, _policies(case))
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
    B, D = case["batch"], case["head_dim"]
    if case["kind"] == "image":   # a program keeps one table for each scale
        state["tables"] = [_table(case, w) for w in state["where"]]
    else:   # where each request's states begin and end; a program that packs them knows it on the host as well
        lengths = state["lengths"].tolist()
        first = state["offsets"].tolist()[:-1]
        state["starts"] = first, [f + n for f, n in zip(first, lengths)]
    if not own:
        if case["kind"] == "cross":   # 4 bits' worth of values, which bf16 numbers are
            state["k"], state["v"] = (_held(state[i].float()).to(torch.bfloat16) for i in "kv")
        return state
    if case["kind"] != "image":
        k = state["k"]
        kv = amskv.Strides(0 if case["packed"] else k.stride(0), D, k.stride(0) if case["packed"] else k.stride(1))
        H, T = (case["heads"], case["queries"]) if case["kind"] == "cross" else (case["kv_heads"], 0)
        head = amskv.Strides(H * T * D, T * D, D)
        state["cross"] = cross = amskv.Cross(batch=B, heads=H, kv_heads=case["kv_heads"], head_dim=D, dtype=amskv.AMSKV_DTYPE_BF16_KV4,
                                             q_tokens=T, kv_tokens=case["keys"], kv_rows=k.shape[0] if case["packed"] else 0,
                                             q=head, k=kv, v=kv, o=head)
        state["where"] = {"offsets": state["offsets"]} if case["packed"] else {"lengths": None if case["lengths"] == "full" else state["lengths"]}
        need = amskv.amskv_cross_held_bytes(cross, packed=case["packed"])
        state["held"] = tuple(torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(2))
        if case["kind"] == "hold":
            state["out"] = tuple(torch.zeros_like(state[i]) for i in "kv")
            return state
        amskv.amskv_cross_hold(cross, state["k"], state["v"], *state["held"], **state["where"])   # once, for all steps
        state["out"] = torch.empty_like(state["q"])
        need = amskv.amskv_cross_workspace_bytes(cross)
        state["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    else:
        L, H, t = case["layers"], case["heads"], _tokens(case)
        state["cache"] = _Cache(case)
        state["rope"] = _own_rope(case) if case["rope"] else None
        shape = (lambda x: (L, B, x, H * D)) if case["packed"] else (lambda x: (L, B, H, x, D))
        state["out"] = [torch.empty(shape(x), dtype=torch.bfloat16, device="cuda") for x in t]
        state["turned"] = [torch.empty(shape(x)[1:], dtype=torch.bfloat16, device="cuda") for x in t]
        state["held"] = [tuple(torch.empty(B, H, sum(t[k] for k in _kept(p, len(t) - 1)), D, dtype=torch.bfloat16, device="cuda")
                               for _ in range(2)) for p in _policies(case)] if case["export"] else []
    return state


def run(state):
    case = state["case"]
    return _run_own(case, state) if own else _run_plain(case, state)


def _run_plain(case, state):
    if case["kind"] == "hold":
        # rows behind the last state stay as they were
        if case["packed"]:
            n = state["starts"][1][-1]
            return tuple(torch.cat((_held(state[i][:n].float()).to(torch.bfloat16), torch.zeros_like(state[i][n:]))) for i in "kv")
        out = tuple(_held(state[i].float()).to(torch.bfloat16) for i in "kv")
        beyond = torch.arange(case["keys"], device="cuda") >= state["lengths"][:, None]
        return tuple(x.masked_fill_(beyond[:, :, None, None], 0) for x in out)
    if case["kind"] == "cross":
        return _plain_cross(case, state, 2 ** 30)
    out = _plain_image(case, state, state["tables"], 2 ** 30)
    return {"o": [o.to(torch.bfloat16) for o in out["o"]], "held": [tuple(x.to(torch.bfloat16) for x in p) for p in out["held"]]}


def _run_own(case, state):
    if case["kind"] == "hold":
        amskv.amskv_cross_hold(state["cross"], state["k"], state["v"], *state["held"], **state["where"])
        amskv.amskv_cross_export(state["cross"], *state["held"], *state["out"], **state["where"])
        return state["out"]
    if case["kind"] == "cross":
        amskv.amskv_cross_attend(state["cross"], state["q"], *state["held"], state["out"], workspace=state["workspace"], **state["where"])
        return state["out"]
    handle, rope, turned, tables = state["cache"].handle, state["rope"], state["turned"], state["tables"]
    width = case["heads"] * case["head_dim"]
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

    def turned(t, where):
        pairing, axes, rot = _rope(case)
        y = t.clone()
        n = rot // 2 // axes
        for i in range(rot // 2):   # pair by pair, as the definition has it
            f = BASE ** (-(i % n) / n)
            if case["stretch"] > 1:
                ramp = min(1.0, max(0.0, (TRAINED * f / (2 * math.pi) - 1.0) / 31.0))
                f = f * ramp + f / case["stretch"] * (1.0 - ramp)
            angle = where[..., i // n] * f
            c, s = _amplitude(case) * torch.cos(angle), _amplitude(case) * torch.sin(angle)
            a, b = (i, i + rot // 2) if pairing == "half" else (2 * i, 2 * i + 1)
            y[..., a] = t[..., a] * c - t[..., b] * s
            y[..., b] = t[..., a] * s + t[..., b] * c
        return y

    def two(e):   # 2^e
        return ((e.long() + 1023) << 52).view(wide)

    def in_4_bits(t):
        numbers = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=wide, device=t.device)
        out = torch.empty(t.shape, dtype=wide, device=t.device)
        flat, to = t.reshape(-1, GROUP), out.view(-1, GROUP)
        for i in range(0, flat.shape[0], 2 ** 22):
            y = flat[i:i + 2 ** 22].to(wide)
            top = y.abs().amax(dim=1, keepdim=True)
            e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -300) / 7.0))
            e = torch.where(top > 7.0 * two(e), e + 1, e)               # log2 next to a power of two
            e = torch.where(top <= 7.0 * two(e - 1), e - 1, e).clamp(min=-100, max=125)
            z = y.abs() / two(e)
            at = torch.bucketize(z, (numbers[1:] + numbers[:-1]) / 2)   # a middle goes down ...
            odd = at % 2 == 1                                           # ... and from there, under an odd code, to the even one above
            middle = (numbers[at.clamp(max=6) + 1] + numbers[at]) / 2
            at = torch.where(odd & (z == middle) & (at < 7), at + 1, at)
            to[i:i + 2 ** 22] = numbers[at] * two(e) * torch.sign(y)
        return out

    def attention(q, k, v):
        out = torch.empty_like(q)
        step = max(1, 2 ** 28 // (q.shape[1] * k.shape[1]))
        for i in range(0, q.shape[0], step):
            s = torch.bmm(q[i:i + step], k[i:i + step].transpose(1, 2).contiguous()) / math.sqrt(q.shape[-1])
            p = torch.exp(s - s.max(dim=2, keepdim=True).values)
            out[i:i + step] = torch.bmm(p / p.sum(dim=2, keepdim=True), v[i:i + step])
        return out

    B, D = case["batch"], case["head_dim"]
    if case["kind"] == "hold":
        out = tuple(in_4_bits(x[i]) for i in "kv")
        for y in out:   # nothing is written behind the last state
            if case["packed"]:
                y[int(x["offsets"][-1]):] = 0
            else:
                for b, n in enumerate(x["lengths"].tolist()):
                    y[b, n:] = 0
        return out
    H = case["heads"]
    if case["kind"] == "cross":
        out = torch.zeros(x["q"].shape, dtype=wide, device="cuda")
        ends, lengths, share = x["offsets"].tolist(), x["lengths"].tolist(), H // case["kv_heads"]
        for b in range(B):
            n = lengths[b]
            if n:
                k, v = (in_4_bits(t[ends[b]:ends[b] + n] if case["packed"] else t[b, :n]).permute(1, 0, 2) for t in (x["k"], x["v"]))
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
                a, b = turned(a, x["where"][s]), turned(b, x["where"][s])
                a = a.to(torch.bfloat16).to(wide)
            if not _in_place(case, policy, s):
                b, c = in_4_bits(b), in_4_bits(c)
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
