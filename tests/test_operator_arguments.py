"""What the rotary, 8-bit and cross-attention calls refuse, and the host side of the 8-bit cache: no GPU needed."""
import math
import os
import subprocess
import sys

import pytest

import paper_2511_16047_amd as amskv
from oracle import amskv_oracle as orc

VAR = (1, 2, 3, 4, 5, 6, 8, 10, 13, 16)
A = 1 << 20          # an address that is never followed: every call here ends in the checks
INVALID, ORDER, NO_MEMORY, SMALL = (amskv.AMSKV_ERR_INVALID_ARG, amskv.AMSKV_ERR_ORDER, amskv.AMSKV_ERR_NO_DEVICE_MEMORY,
                                    amskv.AMSKV_ERR_ARENA_TOO_SMALL)


def _refused(status, call, *a, **k):
    with pytest.raises(amskv.AmskvError) as e:
        call(*a, **k)
    assert e.value.status == status


def _rope(**k):
    return amskv.Rope(**dict(dict(rot_dim=64), **k))


@pytest.mark.parametrize("bad", [dict(rot_dim=0), dict(rot_dim=24), dict(rot_dim=144), dict(rot_dim=-16), dict(pairing=2), dict(axes=0),
                                 dict(axes=3), dict(base=0.0), dict(base=math.nan), dict(base=math.inf), dict(factor=0.5),
                                 dict(factor=math.inf), dict(amplitude=0.0), dict(amplitude=math.nan), dict(low=1.0), dict(low=2.0, high=1.0),
                                 dict(low=1.0, high=32.0), dict(low=1.0, high=math.inf, original=8.0), dict(low=-1.0, high=2.0, original=8.0)],
                         ids=str)
def test_tables(bad):
    _refused(INVALID, amskv.amskv_rope_table, _rope(**bad), A, A, 4)


def test_tables_buffers():
    for p, t, n in ((None, A, 4), (A, None, 4), (A + 4, A, 4), (A, A + 8, 4), (A, A, -1), (A, A, 1 << 40)):
        _refused(INVALID, amskv.amskv_rope_table, _rope(), p, t, n)
    amskv.amskv_rope_table(_rope(), None, None, 0)       # no tokens: nothing to do
    _refused(INVALID, amskv.amskv_rope_table, None, A, A, 4)
    _refused(INVALID, amskv.amskv_rope_table, _rope(), A, A, (1 << 25) + 1)


def test_rows_beyond_a_launch():
    row = amskv.Strides(1 << 33, 1 << 28, 64)
    _refused(INVALID, amskv.amskv_rotate, **dict(ROTATE, rope=_rope(), batch=33, heads=8, tokens=1 << 21, x_strides=row, out_strides=row))


ROTATE = dict(dtype=amskv.AMSKV_DTYPE_BF16, head_dim=64, batch=2, heads=3, tokens=5, table=A, table_batch=0, x=A,
              x_strides=amskv.Strides(960, 320, 64), out=2 * A, out_strides=amskv.Strides(960, 320, 64))


@pytest.mark.parametrize("bad", [dict(dtype=2), dict(dtype=-1), dict(head_dim=96), dict(head_dim=32), dict(batch=-1), dict(heads=-1),
                                 dict(tokens=-1), dict(tokens=1 << 23), dict(batch=1 << 20, heads=1 << 10), dict(table=None),
                                 dict(table=A + 4), dict(x=None), dict(x=A + 2), dict(out=None), dict(out=A + 8), dict(table_batch=-4),
                                 dict(table_batch=2), dict(x_strides=amskv.Strides(960, 324, 64)), dict(x_strides=amskv.Strides(-960, 320, 64)),
                                 dict(out_strides=amskv.Strides(960, 320, 0)), dict(out_strides=amskv.Strides(960, 320, 32)),
                                 dict(x_strides=None), dict(out=A, out_strides=amskv.Strides(1920, 320, 64)), dict(rope=_rope(rot_dim=80))], ids=str)
def test_rotate(bad):
    a = dict(ROTATE, rope=_rope(), **{})
    a.update(bad)
    _refused(INVALID, amskv.amskv_rotate, **a)


@pytest.mark.parametrize("strides", [(960, 64, 64), (64, 320, 64), (320, 320, 64), (959 - 63, 320, 64), (64, 128, 320), (960, 256, 64), (384, 192, 128)],
                         ids=str)
def test_rows_written_twice(strides):
    """[2][3][5] rows: some would share memory, wholly or in part."""
    _refused(INVALID, amskv.amskv_rotate, **dict(ROTATE, rope=_rope(), out_strides=amskv.Strides(*strides)))
    _refused(INVALID, amskv.amskv_cross_attend, _cross(batch=2, heads=3, q_tokens=5, o=amskv.Strides(*strides)), A, A, A, A)


@pytest.mark.parametrize("empty", ["batch", "heads", "tokens"])
def test_rotate_nothing(empty):
    amskv.amskv_rotate(**dict(ROTATE, rope=_rope(), table=None, x=None, out=None, **{empty: 0}))


def test_rotary_append():
    pol = [(2, 2, False)]
    h = amskv.amskv_cache_create(1, 3, 64, VAR, VAR, 2, amskv.AMSKV_DTYPE_BF16, pol)
    call = lambda **k: amskv.amskv_append_scale_rotary(**dict(dict(cache=h, layer=0, s=0, rope=_rope(), table=A, Q=A, q_token_stride=0, Q_out=A, K=A,
                                                                   V=A), **k))
    try:
        for bad in (dict(rope=None), dict(rope=_rope(rot_dim=128)), dict(table=None), dict(table=A + 4), dict(K=None), dict(V=None), dict(Q=None),
                    dict(Q_out=None), dict(Q=A + 8), dict(K=A + 8), dict(V=A + 2), dict(layer=1), dict(s=-1), dict(s=10), dict(cache=None)):
            _refused(INVALID, call, **bad)
        _refused(ORDER, call, s=1)
        _refused(NO_MEMORY, call)
        assert amskv.amskv_cache_layout(h, 0) == []
        amskv.amskv_cache_set_io_layout(h, amskv.AMSKV_IO_TOKEN_MAJOR, 192, 576, 192)
        for bad in (dict(q_token_stride=100), dict(q_token_stride=196), dict(q_token_stride=-576), dict(q_token_stride=576)):
            _refused(INVALID, call, **bad)               # the last one: in place, but read and written at two strides
        _refused(NO_MEMORY, call, q_token_stride=576, Q_out=2 * A)
    finally:
        amskv.amskv_cache_destroy(h)


def _cross(**k):
    s = amskv.Strides(6 * 64 * 7, 64 * 7, 64)
    kv = amskv.Strides(3 * 64 * 11, 64, 3 * 64)
    return amskv.Cross(**dict(dict(batch=2, heads=6, kv_heads=3, head_dim=64, dtype=amskv.AMSKV_DTYPE_BF16, q_tokens=7, kv_tokens=11, q=s, k=kv,
                                   v=kv, o=s), **k))


@pytest.mark.parametrize("bad", [dict(batch=-1), dict(heads=-6), dict(kv_heads=0), dict(kv_heads=4), dict(kv_heads=-3), dict(head_dim=80),
                                 dict(dtype=amskv.AMSKV_DTYPE_F32), dict(dtype=amskv.AMSKV_DTYPE_BF16_KV8), dict(q_tokens=-1), dict(kv_tokens=-1),
                                 dict(q_tokens=1 << 23), dict(kv_tokens=(1 << 26) + 1), dict(batch=1 << 23), dict(softmax_scale=-1.0),
                                 dict(softmax_scale=math.inf), dict(softmax_scale=math.nan), dict(batch=1 << 15, heads=512, kv_heads=1, q_tokens=257)],
                         ids=str)
def test_cross_shapes(bad):
    _refused(INVALID, amskv.amskv_cross_workspace_bytes, _cross(**bad))
    _refused(INVALID, amskv.amskv_cross_attend, _cross(**bad), A, A, A, A)


@pytest.mark.parametrize("bad", [dict(Q=None), dict(K=None), dict(V=None), dict(O=None), dict(Q=A + 2), dict(K=A + 8), dict(V=A + 4), dict(O=A + 8),
                                 dict(lengths=A, offsets=A), dict(lengths=A + 2), dict(offsets=A + 1), dict(workspace=A + 8, workspace_bytes=1 << 20)],
                         ids=str)
def test_cross_buffers(bad):
    _refused(INVALID, amskv.amskv_cross_attend, **dict(dict(cross=_cross(kv_rows=22), Q=A, K=A, V=A, O=A), **bad))


def test_cross_strides_and_rows():
    for bad in (dict(q=amskv.Strides(1, 448, 64)), dict(k=amskv.Strides(2112, 64, 100)), dict(o=amskv.Strides(2688, 448, 0)),
                dict(v=amskv.Strides(2112, -64, 192)), dict(k=amskv.Strides(1 << 30, 64, 1 << 23))):
        _refused(INVALID, amskv.amskv_cross_attend, _cross(**bad), A, A, A, A)
    for rows in (-1, 1 << 31):
        _refused(INVALID, amskv.amskv_cross_attend, _cross(kv_rows=rows), A, A, A, A, offsets=A)
    _refused(INVALID, amskv.amskv_cross_workspace_bytes, None)


def test_cross_nothing():
    for empty in (dict(batch=0), dict(heads=0, kv_heads=0), dict(q_tokens=0)):
        assert amskv.amskv_cross_workspace_bytes(_cross(**empty)) == 0
        amskv.amskv_cross_attend(_cross(**empty), None, None, None, None)


def test_cross_workspace():
    """Few rows over many states ask for one, and a smaller one than they ask for is refused."""
    x = _cross(kv_tokens=16000, k=amskv.Strides(16000 * 192, 64, 192), v=amskv.Strides(16000 * 192, 64, 192))
    need = amskv.amskv_cross_workspace_bytes(x)
    assert need > 0 and amskv.amskv_cross_workspace_bytes(_cross()) == 0
    _refused(SMALL, amskv.amskv_cross_attend, x, A, A, A, A, workspace=A, workspace_bytes=need - 1)


# ---------------------------------------------------------------- the 8-bit cache's host side
def _args(pols, **k):
    a = dict(dict(layers=len(pols), heads=3, head_dim=64, sides_h=VAR, sides_w=VAR, batch=2, dtype=amskv.AMSKV_DTYPE_BF16_KV8, policies=pols), **k)
    return a


def test_eight_bits_are_for_scale_windows():
    _refused(INVALID, amskv.amskv_cache_create, **_args([(2, 2, False)], fuse_append=True))
    _refused(INVALID, amskv.amskv_cache_create, **_args([], layers=1, policies=None, budgets=[(174, 274, 5, 0.5)]))
    _refused(INVALID, amskv.amskv_cache_create, **_args([], layers=1, policies=None, windows=[(170, 5)]))


def _slot(t):
    return (t + 15) // 16 * 16


@pytest.mark.parametrize("layout", [amskv.AMSKV_LAYOUT_COMPACT, amskv.AMSKV_LAYOUT_PLANNED])
@pytest.mark.parametrize("borrow", [False, True])
def test_eight_bits_layout(layout, borrow):
    pols = [(2, 2, False), (0, 0, True), (1, 3, False), (0, 0, False)]
    tokens = [s * s for s in VAR]
    B, H, D = 2, 3, 64
    h = amskv.amskv_cache_create(**_args(pols), layout=layout, borrow_unretained=borrow)
    try:
        for layer, pol in enumerate(pols):
            cap = amskv.amskv_cache_capacity_tokens(h, layer)
            assert cap % 16 == 0
            for s in range(len(VAR)):
                amskv.amskv_append_scale(h, layer, s)
                now = amskv.amskv_cache_layout(h, layer)
                assert [x[0] for x in now] == orc.kept_scales(pol, s)
                at, held = [], 0
                for scale, off, n in now:
                    assert n == tokens[scale]
                    if off < 0:
                        assert borrow and scale == s
                        held += 2 * 2 * B * H * D * n
                        continue
                    assert off % 16 == 0 and off + _slot(n) <= cap
                    at.append((off, off + _slot(n)))
                    held += 2 * B * H * (D * n + _slot(n) // 16 * 4)
                assert all(a[1] <= b[0] for a, b in zip(sorted(at), sorted(at)[1:]))      # no two scales share a block
                assert amskv.amskv_cache_bytes_held(h, layer) == held
    finally:
        amskv.amskv_cache_destroy(h)


def test_eight_bits_arena():
    """Codes and scales of K and V, rounded up to 256 bytes each, and no workspace."""
    cap, bh = sum(_slot(s * s) for s in VAR), 6
    up = lambda x: (x + 255) // 256 * 256
    need = amskv.amskv_cache_required_bytes(**_args([(0, 0, True)]))
    assert need == 2 * up(bh * cap * 64) + 2 * up(bh * cap // 16 * 4)


def test_eight_bits_strides():
    h = amskv.amskv_cache_create(**_args([(2, 2, False)]))
    try:
        _refused(INVALID, amskv.amskv_cache_set_io_layout, h, amskv.AMSKV_IO_TOKEN_MAJOR, 192, 1 << 23, 192)
        amskv.amskv_cache_set_io_layout(h, amskv.AMSKV_IO_TOKEN_MAJOR, 1 << 23, (1 << 23) - 8, 1 << 23)
    finally:
        amskv.amskv_cache_destroy(h)


def test_eight_bits_refuse_the_analysis():
    h = amskv.amskv_cache_create(**_args([(2, 2, False)]))
    try:
        amskv.amskv_append_scale(h, 0, 0)
        amskv.amskv_append_scale(h, 0, 1)
        _refused(INVALID, amskv.amskv_interscale_similarity, h, 0, 1, 3)
        _refused(INVALID, amskv.amskv_interscale_similarity_enqueue, h, 0, 1)
        _refused(INVALID, amskv.amskv_interscale_similarity_enqueue_static, h, 0, 1, True, A)
        _refused(INVALID, amskv.amskv_interscale_similarity_collect, h, 1, 3)
        _refused(INVALID, amskv.amskv_attention_density, h, 0, 1, A, 3)
        _refused(INVALID, amskv.amskv_attention_density_enqueue, h, 0, 1, A, A)
        _refused(INVALID, amskv.amskv_attend_density, h, 0, 1, A, A, A)
        _refused(NO_MEMORY, amskv.amskv_attend, h, 0, 1, A, A)
        _refused(NO_MEMORY, amskv.amskv_cache_export, h, 0, A, A)
        assert [x[0] for x in amskv.amskv_cache_layout(h, 0)] == [0, 1]
    finally:
        amskv.amskv_cache_destroy(h)


# ---------------------------------------------------------------- how the calls are made
CALLS = """
import sys
if sys.argv[1] == "ctypes":
    sys.modules["paper_2511_16047_amd._pycalls"] = None      # as where it is not built: importing it raises ImportError
import ctypes
import paper_2511_16047_amd as amskv
rope, st = amskv.Rope(rot_dim=64), amskv.Strides(64, 64, 64)
cross = amskv.Cross(batch=1, heads=1, kv_heads=1, head_dim=64, dtype=amskv.AMSKV_DTYPE_BF16, q_tokens=1, kv_tokens=1, q=st, k=st, v=st, o=st)
h = amskv.amskv_cache_create(1, 1, 64, (1,), (1,), 1, amskv.AMSKV_DTYPE_BF16, [(0, 0, True)])
A = 4096
calls = [lambda: amskv.amskv_rotate(rope, 1, 64, 1, 1, 1, A, 0, A + 2, st, A, st, stream=0),
         lambda: amskv.amskv_rotate(None, 1, 64, 1, 1, 1, A, 0, A, st, A, st),
         lambda: amskv.amskv_rotate(rope, 1, 64, 1, 0, 1, None, 0, None, st, None, st),
         lambda: amskv.amskv_rotate(rope, 1, 64, 1, 0, 1, None, 0, None, ctypes.pointer(st), None, st),
         lambda: amskv.amskv_append_scale_rotary(h, 0, 0, rope, A, A, 0, A, A, A),
         lambda: amskv.amskv_append_scale_rotary(ctypes.c_void_p(h), 0, 0, rope, A, A, 0, A, A, A, stream=ctypes.c_void_p(0).value),
         lambda: amskv.amskv_append_scale_rotary(None, 0, 0, rope, A, A, 0, A, A, A),
         lambda: amskv.amskv_append_scale_rotary(h, 0, 0, None, A, A, 0, A, A, A),
         lambda: amskv.amskv_cross_attend(cross, A, A, A, A + 8),
         lambda: amskv.amskv_cross_attend(cross, A, A, A, A, lengths=A, offsets=A),
         lambda: amskv.amskv_cross_attend(None, A, A, A, A),
         lambda: amskv.amskv_rotate(st, 1, 64, 1, 1, 1, A, 0, A, st, A, st),
         lambda: amskv.amskv_cross_attend(rope, A, A, A, A)]
for call in calls:
    try:
        call()
        print("0")
    except amskv.AmskvError as e:
        print(e.status)
    except (TypeError, ctypes.ArgumentError):
        print("wrong")
amskv.amskv_cache_destroy(h)
"""


@pytest.mark.parametrize("way", ["extension", "ctypes"])
def test_both_ways_to_make_a_call(way):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    p = subprocess.run([sys.executable, "-c", CALLS, way], cwd=root, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert p.returncode == 0, p.stdout
    want = [INVALID, INVALID, 0, 0, NO_MEMORY, NO_MEMORY, INVALID, INVALID, INVALID, INVALID, INVALID, "wrong", "wrong"]
    assert p.stdout.split() == [str(x) for x in want]
