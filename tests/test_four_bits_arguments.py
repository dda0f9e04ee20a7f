"""What the calls about K and V in 4 bits refuse, and the host side of the 4-bit cache: no GPU needed."""
import math

import pytest

import paper_2511_16047_amd as amskv
from oracle import amskv_oracle as orc

VAR = (1, 2, 3, 4, 5, 6, 8, 10, 13, 16)
KV4 = amskv.AMSKV_DTYPE_BF16_KV4
A = 1 << 20          # addresses that are never followed: every call here ends in the checks
INVALID, NO_MEMORY, SMALL = amskv.AMSKV_ERR_INVALID_ARG, amskv.AMSKV_ERR_NO_DEVICE_MEMORY, amskv.AMSKV_ERR_ARENA_TOO_SMALL


def _refused(status, call, *a, **k):
    with pytest.raises(amskv.AmskvError) as e:
        call(*a, **k)
    assert e.value.status == status


# ---------------------------------------------------------------- the cache
def _args(pols, **k):
    return dict(dict(layers=len(pols), heads=3, head_dim=64, sides_h=VAR, sides_w=VAR, batch=2, dtype=KV4, policies=pols), **k)


def test_four_bits_are_for_scale_windows():
    _refused(INVALID, amskv.amskv_cache_create, **_args([(2, 2, False)], fuse_append=True))
    _refused(INVALID, amskv.amskv_cache_create, **_args([(2, 2, False)], head_dim=96))
    _refused(INVALID, amskv.amskv_cache_create, **_args([(2, 2, False)], dtype=4))
    _refused(INVALID, amskv.amskv_cache_create, **_args([], layers=1, policies=None, budgets=[(174, 274, 5, 0.5)]))
    _refused(INVALID, amskv.amskv_cache_create, **_args([], layers=1, policies=None, windows=[(170, 5)]))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", [amskv.AMSKV_LAYOUT_COMPACT, amskv.AMSKV_LAYOUT_PLANNED])
@pytest.mark.parametrize("borrow", [False, True])
def test_layout(D, layout, borrow):
    """Slots of as many tokens as a scale has, wherever an ordinary cache has them."""
    pols = [(2, 2, False), (0, 0, True), (1, 3, False), (0, 0, False)]
    tokens = [s * s for s in VAR]
    B, H = 2, 3
    h = amskv.amskv_cache_create(**_args(pols, head_dim=D), layout=layout, borrow_unretained=borrow)
    plain = amskv.amskv_cache_create(**_args(pols, head_dim=D, dtype=amskv.AMSKV_DTYPE_BF16), layout=layout, borrow_unretained=borrow)
    try:
        for layer, pol in enumerate(pols):
            assert amskv.amskv_cache_capacity_tokens(h, layer) == amskv.amskv_cache_capacity_tokens(plain, layer)
            for s in range(len(VAR)):
                amskv.amskv_append_scale(h, layer, s)
                amskv.amskv_append_scale(plain, layer, s)
                now = amskv.amskv_cache_layout(h, layer)
                assert now == amskv.amskv_cache_layout(plain, layer)
                assert [x[0] for x in now] == orc.kept_scales(pol, s)
                held = sum(2 * B * H * tokens[scale] * (D // 2 + D // 32 if off >= 0 else 2 * D) for scale, off, _ in now)
                assert amskv.amskv_cache_bytes_held(h, layer) == held
    finally:
        amskv.amskv_cache_destroy(h)
        amskv.amskv_cache_destroy(plain)


def test_arena():
    """Codes and powers of K and V, rounded up to 256 bytes each, and no workspace."""
    cap, bh = sum(s * s for s in VAR), 6
    up = lambda x: (x + 255) // 256 * 256
    for D in (64, 128):
        assert amskv.amskv_cache_required_bytes(**_args([(0, 0, True)], head_dim=D)) == 2 * up(bh * cap * D // 2) + 2 * up(bh * cap * D // 32)


def test_strides():
    h = amskv.amskv_cache_create(**_args([(2, 2, False)]))
    try:
        _refused(INVALID, amskv.amskv_cache_set_io_layout, h, amskv.AMSKV_IO_TOKEN_MAJOR, 192, 1 << 23, 192)
        amskv.amskv_cache_set_io_layout(h, amskv.AMSKV_IO_TOKEN_MAJOR, 1 << 23, (1 << 23) - 8, 1 << 23)
    finally:
        amskv.amskv_cache_destroy(h)


def test_the_analysis_is_refused():
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
        _refused(NO_MEMORY, amskv.amskv_append_scale, h, 0, 2, A, A)
        assert [x[0] for x in amskv.amskv_cache_layout(h, 0)] == [0, 1]
    finally:
        amskv.amskv_cache_destroy(h)


# ---------------------------------------------------------------- held states
def _cross(**k):
    s = amskv.Strides(6 * 64 * 7, 64 * 7, 64)
    kv = amskv.Strides(3 * 64 * 11, 64, 3 * 64)
    return amskv.Cross(**dict(dict(batch=2, heads=6, kv_heads=3, head_dim=64, dtype=KV4, q_tokens=7, kv_tokens=11, kv_rows=22, q=s, k=kv, v=kv, o=s), **k))


def test_held_bytes():
    for D in (64, 128):
        assert amskv.amskv_cross_held_bytes(_cross(head_dim=D)) == 2 * 3 * 11 * (D // 2 + D // 32)
        assert amskv.amskv_cross_held_bytes(_cross(head_dim=D), packed=True) == 3 * 22 * (D // 2 + D // 32)
    assert amskv.amskv_cross_held_bytes(_cross(batch=0)) == 0 and amskv.amskv_cross_held_bytes(_cross(kv_tokens=0)) == 0
    big = _cross(batch=1 << 10, heads=1 << 10, kv_heads=1 << 10, q_tokens=1, head_dim=128, kv_tokens=1 << 26)
    assert amskv.amskv_cross_held_bytes(big) == (1 << 46) * 68
    for rows in (-1, 1 << 31):
        _refused(INVALID, amskv.amskv_cross_held_bytes, _cross(kv_rows=rows), packed=True)
    _refused(INVALID, amskv.amskv_cross_held_bytes, None)


def _hold(**k):
    amskv.amskv_cross_hold(**dict(dict(cross=_cross(), K=A, V=2 * A, K_held=3 * A, V_held=4 * A), **k))


def _export(**k):
    amskv.amskv_cross_export(**dict(dict(cross=_cross(), K_held=3 * A, V_held=4 * A, K_out=A, V_out=2 * A), **k))


@pytest.mark.parametrize("bad", [dict(batch=-1), dict(heads=-6), dict(kv_heads=0), dict(kv_heads=4), dict(kv_heads=-3), dict(head_dim=80),
                                 dict(dtype=amskv.AMSKV_DTYPE_F32), dict(dtype=amskv.AMSKV_DTYPE_BF16_KV8), dict(dtype=amskv.AMSKV_DTYPE_BF16),
                                 dict(kv_tokens=-1), dict(kv_tokens=(1 << 26) + 1), dict(batch=1 << 23), dict(heads=0, kv_heads=1 << 24),
                                 dict(softmax_scale=math.nan)], ids=str)
def test_held_shapes(bad):
    for call in (_hold, _export):
        _refused(INVALID, call, cross=_cross(**bad))
    _refused(INVALID, amskv.amskv_cross_held_bytes, _cross(**bad))


@pytest.mark.parametrize("bad", [dict(lengths=A, offsets=A), dict(lengths=A + 2), dict(offsets=A + 1), dict(K_held=None), dict(V_held=None),
                                 dict(K_held=3 * A + 8), dict(V_held=3 * A), dict(cross=None)], ids=str)
def test_held_buffers(bad):
    _refused(INVALID, _hold, **bad)
    if bad != dict(V_held=3 * A):   # (one held tensor may be read for both)
        _refused(INVALID, _export, **bad)


def test_held_directions():
    for bad in (dict(K=None, V=None), dict(K=A + 2), dict(V=A + 8), dict(K=3 * A), dict(V=3 * A), dict(K=4 * A)):
        _refused(INVALID, _hold, **bad)
    for bad in (dict(K_out=None, V_out=None), dict(K_out=A + 2), dict(V_out=A), dict(K_out=3 * A), dict(V_out=3 * A)):
        _refused(INVALID, _export, **bad)
    for rows in (-1, 1 << 31):
        for call in (_hold, _export):
            _refused(INVALID, call, cross=_cross(kv_rows=rows), offsets=A)
    far = amskv.Strides(1 << 37, 1 << 33, 64)
    for call in (_hold, _export):   # 2^36 rows and 2^26 more
        _refused(INVALID, call, cross=_cross(batch=1025, heads=1, kv_heads=1, q_tokens=1, kv_tokens=1 << 26, k=far, v=far))


@pytest.mark.parametrize("strides", [(2112, 64, 100), (-2112, 64, 192), (2112, 64, 1 << 41)], ids=str)
def test_held_strides(strides):
    for call in (_hold, _export):
        _refused(INVALID, call, cross=_cross(k=amskv.Strides(*strides)))
        _refused(INVALID, call, cross=_cross(v=amskv.Strides(*strides)))


@pytest.mark.parametrize("strides", [(2112, 64, 64), (0, 64, 192), (64, 64, 192), (2112, 64, 184), (2048, 64, 192)], ids=str)
def test_read_back_rows_written_twice(strides):
    _refused(INVALID, _export, cross=_cross(k=amskv.Strides(*strides)))
    _refused(INVALID, _export, cross=_cross(v=amskv.Strides(*strides)))


def test_held_nothing():
    for empty in (dict(batch=0), dict(kv_tokens=0), dict(heads=0, kv_heads=0)):
        amskv.amskv_cross_hold(_cross(**empty), None, None, None, None)
        amskv.amskv_cross_export(_cross(**empty), None, None, None, None)
    amskv.amskv_cross_hold(_cross(kv_rows=0), None, None, None, None, offsets=A)
    amskv.amskv_cross_hold(_cross(batch=0), A, 2 * A, 3 * A, 4 * A, offsets=A)


@pytest.mark.parametrize("bad", [dict(Q=None), dict(K=None), dict(V=None), dict(O=None), dict(Q=A + 2), dict(K=A + 8), dict(V=A + 4), dict(O=A + 8),
                                 dict(lengths=A, offsets=A), dict(lengths=A + 2), dict(offsets=A + 1), dict(workspace=A + 8, workspace_bytes=1 << 20)],
                         ids=str)
def test_attention_buffers(bad):
    _refused(INVALID, amskv.amskv_cross_attend, **dict(dict(cross=_cross(), Q=A, K=A, V=A, O=A), **bad))


def test_attention_strides_and_workspace():
    for bad in (dict(q=amskv.Strides(1, 448, 64)), dict(o=amskv.Strides(2688, 448, 0)), dict(o=amskv.Strides(2688, 448, 32))):
        _refused(INVALID, amskv.amskv_cross_attend, _cross(**bad), A, A, A, A)
    x = _cross(kv_tokens=16000, k=amskv.Strides(7, 7, 7), v=amskv.Strides(7, 7, 7))      # held tensors have no strides
    need = amskv.amskv_cross_workspace_bytes(x)
    assert need > 0
    _refused(SMALL, amskv.amskv_cross_attend, x, A, A, A, A, workspace=A, workspace_bytes=need - 1)
    for empty in (dict(batch=0), dict(heads=0, kv_heads=0), dict(q_tokens=0)):
        assert amskv.amskv_cross_workspace_bytes(_cross(**empty)) == 0
        amskv.amskv_cross_attend(_cross(**empty), None, None, None, None)
