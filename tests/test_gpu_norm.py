"""The root-mean-square norm and rows in e4m3 against their definition in 64 bits.

Tolerance.  s is rounded once (2^-24 of itself; of the mean's root as much at most), the factor 1 / rms once, the product with it and the one with the weight
once each: 5 times 2^-24 of y, and 2^-24 for what the factor's steps in 64 bits add to its rounding.  Then one rounding to the output's type: eps / 2.  A
scale is the largest |y| divided by 448: 7 times 2^-24.  A code is the nearest of y / scale: half a step is 2^-4 of a normal value at most, 2^-10 below 2^-6, and
the reciprocal, the product and the scale's own error move y / scale by 10 times 2^-24."""
import math

import pytest
import torch

from low_bits_calls import NORM
from paper_2501_10054_amd import tardis as T
from test_gpu_linear import inside

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = 2.0 ** -24
OUTS = [torch.float32, torch.bfloat16, T.FP8]
SIZES = [(1, 1), (3, 7), (9, 8), (1, 64), (5, 65), (257, 128), (33, 1000), (64, 520), (2, 4096), (7, 4097), (19, 11008), (3, 16384), (2, 16385), (3, 32768), (2, 32769), (2, 70001)]


def reference(x, weight, residual, eps):
    s = x.double() if residual is None else x.double() + residual.double()
    y = s / (s.pow(2).mean(1, keepdim=True) + eps).sqrt()
    return s, y if weight is None else y * weight.double()


def check(got, want, off):
    assert got.shape == want.shape
    err = (got.double() - want).abs()
    assert not torch.isnan(err).any()
    assert (err <= off).all(), (err / off).max().item()


def check_codes(codes, scales, y):
    top = (y.abs().amax(1) / 448.0).clamp_min(2.0 ** -126)
    check(scales, top, 7 * U * top)
    v = y / scales.double()[:, None]
    check(codes.float(), v, torch.maximum(2.0 ** -4 * v.abs(), torch.full_like(v, 2.0 ** -10)) + 10 * U * v.abs())


def check_norm(got, x, weight, residual, eps, out):
    s, y = reference(x, weight, residual, eps)
    got = got if isinstance(got, tuple) else (got,)
    assert len(got) == (2 if out == T.FP8 else 1) + (residual is not None)
    if residual is not None:
        check(got[-1], s, torch.finfo(x.dtype).eps / 2 * s.abs() + U * s.abs() + 1e-45)
    if out == T.FP8:
        check_codes(got[0], got[1], y)
    else:
        check(got[0], y, (torch.finfo(out).eps / 2 + 6 * U) * y.abs() + 2.0 ** -149)


@pytest.mark.parametrize("case", range(len(SIZES)))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("gap", [0, 8, 3])
def test_norm(case, dtype, gap):
    n, d = SIZES[case]
    gen = torch.Generator(device=DEV).manual_seed(100 * case + gap)
    x = inside((n, d), dtype, gen, gap=gap, lead=case % 3)
    weight = inside((1, d), dtype, gen, lead=1)[0] if (case + gap) % 4 else None
    residual = inside((n, d), dtype, gen, lead=1) if (case + gap) % 2 else None
    for out in OUTS:
        check_norm(T.tardis_rms_norm(x, weight, residual=residual, eps=1e-5, out_dtype=out), x, weight, residual, 1e-5, out)


@pytest.mark.parametrize("case", range(len(SIZES)))
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("gap", [0, 3])
def test_fp8_rows(case, dtype, gap):
    n, d = SIZES[case]
    gen = torch.Generator(device=DEV).manual_seed(100 * case + gap)
    x = inside((n, d), dtype, gen, gap=gap, lead=case % 3)
    x[n // 2] = 0
    codes, scales = T.tardis_fp8_rows(x)
    check_codes(codes, scales, x.double())
    assert (codes[n // 2].float() == 0).all()


def test_sums_of_squares_over_the_whole_range_of_fp32():
    """Rows of any magnitude: squares of 1e38 and of 1e-38 are no fp32 values."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn(8, 1000, device=DEV, generator=gen)
    x *= torch.tensor([1e38 / 6, 1e30, 1e19, 1.0, 1e-19, 1e-25, 1e-30, 1e-36], device=DEV)[:, None]
    for eps in (0.0, 1e-30, 1e-6):
        for dtype in (torch.float32, torch.bfloat16):
            xs = x.to(dtype)
            for out in OUTS:
                # (below 2^-126 fp32 has fewer bits: an absolute error of 2^-149)
                s, y = reference(xs, None, None, eps)
                got = T.tardis_rms_norm(xs, eps=eps, out_dtype=out)
                if out == T.FP8:
                    check_codes(*got, y)
                else:
                    check(got, y, (torch.finfo(out).eps / 2 + 6 * U) * y.abs() + 2.0 ** -133)


def test_rows_of_zeros_and_rows_that_are_not_finite():
    x = torch.randn(6, 520, device=DEV)
    x[1] = 0
    x[2, 7] = math.inf
    x[3, 9] = math.nan
    for eps in (0.0, 1e-5):
        y = T.tardis_rms_norm(x, eps=eps)
        alone = T.tardis_rms_norm(x[:1], eps=eps)
        assert torch.equal(y[:1], alone) and (y[1] == 0).all()
        assert torch.isnan(y[2, 7]) and (y[2, :7] == 0).all() and torch.isnan(y[3]).all() and torch.isfinite(y[4:]).all()
        codes, scales = T.tardis_rms_norm(x, eps=eps, out_dtype=T.FP8)
        assert (codes[1].float() == 0).all() and scales[1] == 2.0 ** -126
        assert torch.isnan(codes[3].float()).all() and torch.isfinite(codes[4:].float()).all()
    codes, scales = T.tardis_fp8_rows(x)
    assert torch.isinf(scales[2]) and torch.isnan(codes[2, 7].float()) and (codes[2, 8:].float() == 0).all()
    assert torch.isnan(codes[3, 9].float()) and torch.isfinite(scales[3]) and torch.isfinite(codes[3, 10:].float()).all()


@pytest.mark.parametrize("d", [520, 4096, 40000])
def test_the_sum_may_be_what_it_is_made_from(d):
    gen = torch.Generator(device=DEV).manual_seed(d)
    x, r = (torch.randn(5, d, device=DEV, generator=gen).bfloat16() for _ in range(2))
    for out in OUTS:
        *want, total = T.tardis_rms_norm(x, residual=r, out_dtype=out)
        for own in (r.clone(), x.clone()):
            a, b = (x, own) if torch.equal(own, r) else (own, r)
            *got, got_total = T.tardis_rms_norm(a, residual=b, out_dtype=out, sum=own)
            assert got_total is own and torch.equal(own, total)
            assert all(torch.equal(p.float(), q.float()) for p, q in zip(got, want))


@pytest.mark.parametrize("out", OUTS)
@pytest.mark.parametrize("n,d", [(3, 7), (5, 513), (2, 4099), (2, 40001)])
def test_nothing_else_is_written(out, n, d):
    gen = torch.Generator(device=DEV).manual_seed(d)
    x = torch.randn(n, d, device=DEV, generator=gen)
    store = torch.full((n * d + 64,), 7.0, device=DEV).to(out)
    kept = torch.full((n * d + 64,), 7.0, device=DEV)
    scales = torch.full((n + 8,), 7.0, device=DEV)
    T.tardis_rms_norm(x, residual=x, out_dtype=out, y=store[5:5 + n * d].view(n, d), sum=kept[5:5 + n * d].view(n, d), scales=scales[3:3 + n] if out == T.FP8 else None)
    for t, size in ((store, n * d), (kept, n * d)):
        assert (t[:5].float() == 7).all() and (t[5 + size:].float() == 7).all()
    assert (scales[:3] == 7).all() and (scales[3 + n:] == 7).all()


def test_more_than_2_to_the_31_elements():
    n, d = 140000, 16384
    x = torch.zeros(n, d, dtype=torch.bfloat16, device=DEV)
    gen = torch.Generator(device=DEV).manual_seed(1)
    last = torch.randn(3, d, device=DEV, generator=gen).bfloat16()
    x[-3:] = last
    codes, scales = T.tardis_rms_norm(x, eps=1e-5, out_dtype=T.FP8)
    check_codes(codes[-3:], scales[-3:], reference(last, None, None, 1e-5)[1])
    assert (codes[:1000].float() == 0).all() and (scales[:-3] == 2.0 ** -126).all()


def test_a_graph_and_another_stream():
    gen = torch.Generator(device=DEV).manual_seed(8)
    x, r = (torch.randn(40, 4096, device=DEV, generator=gen).bfloat16() for _ in range(2))
    w = torch.randn(4096, device=DEV, generator=gen).bfloat16()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = T.tardis_rms_norm(x, w, residual=r, out_dtype=T.FP8, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = T.tardis_rms_norm(x, w, residual=r, out_dtype=T.FP8)
    for i in range(3):
        x.copy_(torch.randn(40, 4096, device=DEV, generator=gen))
        graph.replay()
        torch.cuda.synchronize()
        want = T.tardis_rms_norm(x, w, residual=r, out_dtype=T.FP8)
        assert all(torch.equal(a.float(), b.float()) for a, b in zip(got, want))
    assert torch.isfinite(other[0].float()).all()


def test_no_rows():
    x = torch.zeros(0, 64, device=DEV)
    y, total = T.tardis_rms_norm(x, residual=x)
    codes, scales = T.tardis_fp8_rows(x)
    assert y.shape == total.shape == codes.shape == (0, 64) and scales.shape == (0,)


@pytest.mark.parametrize("call", range(len(NORM)))
def test_every_kernel(call):
    """The calls of low_bits_calls.py, by which every kernel is reached."""
    _, n, d, dtype, out = NORM[call]
    gen = torch.Generator(device=DEV).manual_seed(call)
    dtype, out = T._TORCH_DTYPE[dtype], T.FP8 if out == T.FP8_E4M3 else T._TORCH_DTYPE[out]
    x, r = inside((n, d), dtype, gen), inside((n, d), dtype, gen)
    weight = torch.randn(d, device=DEV, generator=gen).to(dtype)
    check_norm(T.tardis_rms_norm(x, weight, residual=r, out_dtype=out), x, weight, r, 1e-6, out)
