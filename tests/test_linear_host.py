"""What the calls of linear layers and experts refuse, before anything touches a GPU (on the CPU: the pointers are numbers)."""
import ctypes as C

import pytest

from paper_2501_10054_amd import tardis as T

P = C.c_void_p(0x4000)


def _desc(**kw):
    base = dict(n_in=64, n_out=256, dtype=T.BF16, out_dtype=T.BF16, act=0, reserved=0, W=0x1000, b=None)
    base.update(kw)
    return T.tardis_linear_desc(**base)


BAD_DESC = [(dict(W=None), T.ERR_INVALID_ARG), (dict(reserved=1), T.ERR_INVALID_ARG), (dict(dtype=T.FP8_E4M3), T.ERR_DTYPE), (dict(dtype=9), T.ERR_DTYPE),
            (dict(out_dtype=T.FP8_E4M3), T.ERR_DTYPE), (dict(act=4), T.ERR_INVALID_ARG), (dict(act=-1), T.ERR_INVALID_ARG), (dict(n_in=0), T.ERR_SHAPE),
            (dict(n_out=-1), T.ERR_SHAPE), (dict(n_in=(1 << 22) + 1), T.ERR_SHAPE), (dict(n_out=(1 << 22) + 1), T.ERR_SHAPE),
            (dict(W=0x1001), T.ERR_INVALID_ARG), (dict(b=0x1001), T.ERR_INVALID_ARG), (dict(W=0x1002, dtype=T.F32), T.ERR_INVALID_ARG)]


def linear(desc, x=P, n=4, pitch=64, r=None, y=P, work=None, bytes_=0):
    return T.lib().tardis_linear(desc, x, n, pitch, r, y, work, bytes_, None)


def grouped(desc, experts=4, x=P, x_rows=8, pitch=64, offsets=P, order=P, per_token=2, positions=16, y=P, work=None, bytes_=0):
    return T.lib().tardis_grouped_linear(desc, experts, x, x_rows, pitch, offsets, order, per_token, positions, y, work, bytes_, None)


def route(logits=P, n=8, experts=16, k=2, dtype=T.F32, renormalise=1, ids=P, weights=P, offsets=P, order=P, place=P, work=None, bytes_=0):
    return T.lib().tardis_moe_route(logits, n, experts, k, dtype, renormalise, ids, weights, offsets, order, place, work, bytes_, None)


def combine(z=P, rows=16, place=P, weights=P, n=8, k=2, d=64, dtype=T.BF16, r=None, y=P, out=T.BF16):
    return T.lib().tardis_moe_combine(z, rows, place, weights, n, k, d, dtype, r, y, out, None)


@pytest.mark.parametrize("change,status", BAD_DESC)
def test_bad_descriptions(change, status):
    assert linear(_desc(**change)) == status
    assert grouped(_desc(**change)) == status
    assert T.lib().tardis_linear_workspace(_desc(**change), P, 4, 64, C.c_int64()) == status
    assert T.lib().tardis_grouped_linear_workspace(_desc(**change), 4, P, 8, 64, 1, 16, C.c_int64()) == status


def test_linear_refuses():
    assert linear(None) == T.ERR_INVALID_ARG
    odd = C.c_void_p(0x4001)
    for kw in (dict(x=None), dict(y=None), dict(x=odd), dict(y=odd), dict(r=odd), dict(work=C.c_void_p(0x4008), bytes_=64), dict(work=P, bytes_=-1)):
        assert linear(_desc(), **kw) == T.ERR_INVALID_ARG, kw
    assert linear(_desc(out_dtype=T.F32), y=C.c_void_p(0x4002)) == T.ERR_INVALID_ARG
    for kw in (dict(n=-1), dict(n=(1 << 30) + 1), dict(pitch=63), dict(pitch=(1 << 30) + 1)):
        assert linear(_desc(), **kw) == T.ERR_SHAPE, kw
    assert linear(_desc(), n=0, x=None, y=None) == T.OK
    assert T.lib().tardis_linear_workspace(_desc(), P, 4, 64, None) == T.ERR_INVALID_ARG
    assert T.lib().tardis_linear_workspace(_desc(), P, -1, 64, C.c_int64()) == T.ERR_SHAPE
    assert T.lib().tardis_linear_workspace(_desc(), P, 4, 63, C.c_int64()) == T.ERR_SHAPE
    got = C.c_int64(7)
    assert T.lib().tardis_linear_workspace(_desc(), P, 0, 64, got) == T.OK and got.value == 0


def test_more_tiles_than_a_launch_takes():
    """Refused on the host, with and without groups."""
    big = dict(n_in=64, n_out=1 << 22)
    assert linear(_desc(**big), n=1 << 30) == T.ERR_SHAPE
    assert grouped(_desc(**big), x_rows=1 << 30, positions=1 << 30) == T.ERR_SHAPE


def test_grouped_refuses():
    assert grouped(None) == T.ERR_INVALID_ARG
    odd = C.c_void_p(0x4002)
    for kw in (dict(x=None), dict(y=None), dict(offsets=None), dict(offsets=odd), dict(order=odd), dict(x=C.c_void_p(0x4001))):
        assert grouped(_desc(), **kw) == T.ERR_INVALID_ARG, kw
    for kw in (dict(experts=0), dict(experts=65537), dict(x_rows=-1), dict(pitch=63), dict(positions=-1), dict(per_token=0), dict(positions=(1 << 30) + 1),
               dict(order=None, x_rows=15)):
        assert grouped(_desc(), **kw) == T.ERR_SHAPE, kw
    for kw in (dict(work=C.c_void_p(0x4008), bytes_=64), dict(work=P, bytes_=-1)):
        assert grouped(_desc(), **kw) == T.ERR_INVALID_ARG, kw
    assert T.lib().tardis_grouped_linear_workspace(_desc(), 4, P, 8, 64, 1, 16, None) == T.ERR_INVALID_ARG
    for experts, x_rows, pitch, ordered, rows in ((0, 8, 64, 1, 16), (65537, 8, 64, 1, 16), (4, 8, 63, 1, 16), (4, 8, 64, 0, 16), (4, -1, 64, 1, 16)):
        assert T.lib().tardis_grouped_linear_workspace(_desc(), experts, P, x_rows, pitch, ordered, rows, C.c_int64()) == T.ERR_SHAPE
    assert grouped(_desc(), positions=0, offsets=None, x=None, y=None) == T.OK
    assert grouped(_desc(), x_rows=0, x=None) == T.OK


def test_route_refuses():
    odd = C.c_void_p(0x4002)
    for kw in (dict(offsets=None), dict(logits=None), dict(ids=None), dict(weights=None), dict(order=None), dict(place=None), dict(renormalise=2),
               dict(logits=odd), dict(ids=odd), dict(offsets=odd), dict(work=odd)):
        assert route(**kw) == T.ERR_INVALID_ARG, kw
    for kw in (dict(experts=0), dict(experts=1025), dict(k=0), dict(k=17, experts=64), dict(k=3, experts=2), dict(n=-1), dict(n=1 << 30, k=2)):
        assert route(**kw) == T.ERR_SHAPE, kw
    assert route(dtype=T.FP8_E4M3) == T.ERR_DTYPE
    need = C.c_int64()
    assert T.lib().tardis_moe_route_workspace(100000, 64, 2, need) == T.OK and need.value > 0
    assert route(n=100000, experts=64) == T.ERR_INVALID_ARG                                        # none given
    assert route(n=100000, experts=64, work=P, bytes_=need.value - 1) == T.ERR_INVALID_ARG
    assert T.lib().tardis_moe_route_workspace(8, 64, 2, need) == T.OK and need.value == 0
    assert T.lib().tardis_moe_route_workspace(8, 1025, 2, need) == T.ERR_SHAPE
    assert T.lib().tardis_moe_route_workspace(-1, 64, 2, need) == T.ERR_SHAPE
    assert T.lib().tardis_moe_route_workspace(8, 64, 17, need) == T.ERR_SHAPE
    assert T.lib().tardis_moe_route_workspace(8, 2, 3, need) == T.ERR_SHAPE
    assert T.lib().tardis_moe_route_workspace(8, 64, 2, None) == T.ERR_INVALID_ARG


def test_combine_refuses():
    odd = C.c_void_p(0x4001)
    for kw in (dict(z=None), dict(place=None), dict(weights=None), dict(y=None), dict(z=odd), dict(r=odd), dict(place=odd)):
        assert combine(**kw) == T.ERR_INVALID_ARG, kw
    for kw in (dict(rows=-1), dict(n=-1), dict(k=0), dict(k=1025), dict(d=0), dict(d=(1 << 22) + 1)):
        assert combine(**kw) == T.ERR_SHAPE, kw
    assert combine(dtype=T.FP8_E4M3) == T.ERR_DTYPE and combine(out=5) == T.ERR_DTYPE
    assert combine(n=0, z=None, place=None, weights=None, y=None) == T.OK
