"""What the norm, rows in e4m3 and layers in 8 and 4 bits refuse, before anything touches a GPU (on the CPU: the pointers are numbers)."""
import ctypes as C
import math

import pytest
import torch

from paper_2501_10054_amd import tardis as T

P = C.c_void_p(0x4000)
ODD = C.c_void_p(0x4001)


def norm(x=P, n=4, pitch=64, r=None, sum=None, y=P, scales=None, **kw):
    base = dict(d=64, dtype=T.BF16, out_dtype=T.BF16, eps=1e-5, reserved=0, weight=None)
    base.update(kw)
    return T.lib().tardis_rms_norm(T.tardis_norm_desc(**base), x, n, pitch, r, sum, y, scales, None)


def rows(x=P, n=4, d=64, pitch=64, dtype=T.BF16, codes=P, scales=P):
    return T.lib().tardis_fp8_rows(x, n, d, pitch, dtype, codes, scales, None)


def desc8(**kw):
    base = dict(n_in=64, n_out=256, out_dtype=T.BF16, act=0, W=0x1000, W_scales=None, b=None)
    base.update(kw)
    return T.tardis_linear_fp8_desc(**base)


def desc4(**kw):
    base = dict(n_in=64, n_out=256, dtype=T.BF16, out_dtype=T.BF16, act=0, group=32, W=0x1000, scales=0x2000, zeros=None, b=None)
    base.update(kw)
    return T.tardis_linear_4bit_desc(**base)


def eight(desc, x=P, sx=None, n=4, pitch=64, r=None, y=P, work=None, bytes_=0):
    return T.lib().tardis_linear_fp8(desc, x, sx, n, pitch, r, y, work, bytes_, None)


def four(desc, x=P, n=4, pitch=64, r=None, y=P, work=None, bytes_=0):
    return T.lib().tardis_linear_4bit(desc, x, n, pitch, r, y, work, bytes_, None)


def test_norm_refuses():
    assert T.lib().tardis_rms_norm(None, P, 4, 64, None, None, P, None, None) == T.ERR_INVALID_ARG
    for kw in (dict(x=None), dict(y=None), dict(x=ODD), dict(y=ODD), dict(r=ODD), dict(sum=ODD), dict(weight=0x4001), dict(reserved=1), dict(eps=-1e-9), dict(eps=math.nan),
               dict(eps=math.inf), dict(scales=P), dict(out_dtype=T.FP8_E4M3), dict(out_dtype=T.FP8_E4M3, scales=C.c_void_p(0x4002)), dict(dtype=T.F32, x=C.c_void_p(0x4002)),
               dict(sum=P, pitch=72), dict(out_dtype=T.F32, y=C.c_void_p(0x4002))):
        assert norm(**kw) == T.ERR_INVALID_ARG, kw
    for kw in (dict(dtype=T.FP8_E4M3), dict(dtype=7), dict(out_dtype=5)):
        assert norm(**kw) == T.ERR_DTYPE, kw
    for kw in (dict(d=0), dict(d=(1 << 22) + 1, pitch=1 << 23), dict(n=-1), dict(n=(1 << 30) + 1), dict(pitch=63), dict(pitch=(1 << 30) + 1)):
        assert norm(**kw) == T.ERR_SHAPE, kw
    assert norm(n=0, x=None, y=None) == T.OK


def test_rows_refuse():
    for kw in (dict(x=None), dict(codes=None), dict(scales=None), dict(x=ODD), dict(scales=C.c_void_p(0x4002))):
        assert rows(**kw) == T.ERR_INVALID_ARG, kw
    assert rows(dtype=T.FP8_E4M3) == T.ERR_DTYPE
    for kw in (dict(d=0), dict(n=-1), dict(pitch=63), dict(n=(1 << 30) + 1)):
        assert rows(**kw) == T.ERR_SHAPE, kw
    assert rows(n=0, x=None, codes=None, scales=None) == T.OK


@pytest.mark.parametrize("change,status", [(dict(W=None), T.ERR_INVALID_ARG), (dict(out_dtype=T.FP8_E4M3), T.ERR_DTYPE), (dict(act=4), T.ERR_INVALID_ARG),
                                           (dict(act=-1), T.ERR_INVALID_ARG), (dict(n_in=0), T.ERR_SHAPE), (dict(n_out=0), T.ERR_SHAPE), (dict(n_in=(1 << 22) + 1), T.ERR_SHAPE),
                                           (dict(n_out=(1 << 22) + 1), T.ERR_SHAPE), (dict(b=0x1001), T.ERR_INVALID_ARG)])
def test_descriptions_that_both_layers_refuse(change, status):
    for call, desc in ((eight, desc8), (four, desc4)):
        assert call(desc(**change)) == status
    assert T.lib().tardis_linear_fp8_workspace(desc8(**change), P, 4, 64, C.c_int64()) == status
    assert T.lib().tardis_linear_4bit_workspace(desc4(**change), 4, 64, C.c_int64()) == status


def test_layers_refuse():
    assert eight(None) == four(None) == T.ERR_INVALID_ARG
    for call, desc in ((eight, desc8), (four, desc4)):
        for kw in (dict(x=None), dict(y=None), dict(y=ODD), dict(r=ODD), dict(work=C.c_void_p(0x4008), bytes_=64), dict(work=P, bytes_=-1)):
            assert call(desc(), **kw) == T.ERR_INVALID_ARG, kw
        assert call(desc(out_dtype=T.F32), y=C.c_void_p(0x4002)) == T.ERR_INVALID_ARG
        for kw in (dict(n=-1), dict(n=(1 << 30) + 1), dict(pitch=63), dict(pitch=(1 << 30) + 1)):
            assert call(desc(), **kw) == T.ERR_SHAPE, kw
        assert call(desc(), n=0, x=None, y=None) == T.OK
    assert eight(desc8(), sx=C.c_void_p(0x4002)) == eight(desc8(W_scales=0x4002)) == T.ERR_INVALID_ARG
    assert four(desc4(), x=ODD) == four(desc4(W=0x1004)) == four(desc4(scales=None)) == four(desc4(scales=0x2001)) == T.ERR_INVALID_ARG
    for group in (0, 16, 48, 256, -32):
        assert four(desc4(group=group)) == T.ERR_INVALID_ARG
    assert four(desc4(dtype=T.FP8_E4M3)) == four(desc4(dtype=9)) == T.ERR_DTYPE
    assert T.lib().tardis_linear_fp8_workspace(desc8(), P, 4, 64, None) == T.lib().tardis_linear_4bit_workspace(desc4(), 4, 64, None) == T.ERR_INVALID_ARG
    got = C.c_int64(7)
    assert T.lib().tardis_linear_fp8_workspace(desc8(), P, 0, 64, got) == T.OK and got.value == 0


def test_more_tiles_than_a_launch_takes():
    assert eight(desc8(n_out=1 << 22), n=1 << 30) == T.ERR_SHAPE


@pytest.mark.parametrize("group,n_in", [(32, 32), (32, 70), (64, 100), (128, 300), (128, 1)])
def test_packed_codes(group, n_in):
    gen = torch.Generator().manual_seed(n_in)
    q = torch.randint(0, 16, (5, n_in), generator=gen, dtype=torch.uint8)
    words = T.tardis_pack_4bit(q, group)
    assert words.dtype == torch.int32 and words.shape == (5, -(-n_in // group) * group // 8)
    for c in range(words.shape[1] * 8):
        code = words[:, c // 8].long() >> (4 * (c % 8 // 2) + 16 * (c % 2)) & 15
        assert torch.equal(code, q[:, c].long() if c < n_in else torch.zeros(5, dtype=torch.int64))
