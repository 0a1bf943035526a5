"""Codes of rows in e4m3 are the nearest of y / scale, ties to even: compared code by code with a division in fp32 and one rounding on the CPU.

Rows in bf16 have many exact ties (values and the row's largest are of 8 bits), so a quotient that is off by a rounding shows.  No tolerance: a quotient in fp32 is
rounded correctly, and so is its code."""
import math

import numpy as np
import pytest
import torch

from paper_2501_10054_amd import tardis as T

pytestmark = pytest.mark.gpu
DEV = "cuda"


def expected(y):
    """y in fp32, on the CPU -> codes, scales"""
    top = np.nan_to_num(np.abs(y.numpy()), nan=0.0, posinf=math.inf).max(1)
    with np.errstate(over="ignore"):
        scales = torch.from_numpy(np.maximum(top / np.float32(448.0), np.float32(2.0 ** -126)))
    return (y / scales[:, None]).to(T.FP8), scales


def check(got, y):
    codes, scales = (t.cpu() for t in got)
    want, want_scales = expected(y)
    assert torch.equal(scales, want_scales)
    nan = torch.isnan(want.float())
    assert torch.equal(torch.isnan(codes.float()), nan)
    off = (codes.view(torch.uint8) != want.view(torch.uint8)) & ~nan
    assert not off.any(), (off.sum().item(), off.any(1).sum().item())


def rows(n, d, dtype, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(n, d, device=DEV, generator=gen)
    x[:, torch.randperm(d, device=DEV, generator=gen)[:max(1, d // 100)]] *= 8.0
    return x.to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,d", [(1, 16384), (960, 4096), (257, 5137), (300, 40000), (3, 70001), (5, 7)])
def test_codes_of_rows(n, d, dtype):
    x = rows(n, d, dtype, n + d)
    check(T.tardis_fp8_rows(x), x.float().cpu())


def test_every_pair_of_magnitudes():
    """Every bf16 value of two powers of two in rows whose largest is each of the 128 mantissas: every tie that bf16 has."""
    m = 1.0 + torch.arange(128, device=DEV) / 128.0
    x = (m[None, :] * 2.0 ** -torch.arange(0, 12, device=DEV)[:, None]).reshape(1, -1).repeat(128, 1)
    x = torch.cat([torch.where(x <= m[:, None], x, torch.zeros_like(x)), m[:, None]], 1).bfloat16()
    check(T.tardis_fp8_rows(torch.cat([x, -x])), torch.cat([x, -x]).float().cpu())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_codes_of_rows_of_any_magnitude(dtype):
    x = rows(24, 1000, torch.float32, 3)
    x /= x.abs().amax(1, keepdim=True)
    x *= 2.0 ** torch.tensor([127.5, 127, 126, 120, 110, 100, 72, 71, 64, 40, 1, 0, -1, -30, -64, -90, -100, -110, -117, -118, -120, -126, -130, -140],
                             device=DEV, dtype=torch.float64)[:, None].float()
    x = x.to(dtype)
    x[3, 5], x[4, 6], x[9] = math.nan, math.inf, 0.0
    check(T.tardis_fp8_rows(x), x.float().cpu())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,d", [(40, 4096), (2048, 4096), (9, 513), (2, 40000)])
def test_codes_of_a_norm(n, d, dtype):
    """Of small whole numbers, whose squares have the same sum in any order: y in fp32 and y that becomes codes are the same."""
    gen = torch.Generator(device=DEV).manual_seed(n)
    x, r = (torch.randint(-100, 101, (n, d), device=DEV, generator=gen).to(dtype) for _ in range(2))
    weight = torch.randn(d, device=DEV, generator=gen).to(dtype)
    for w in (None, weight):
        y, _ = T.tardis_rms_norm(x, w, residual=r, eps=1e-5, out_dtype=torch.float32)
        codes, scales, _ = T.tardis_rms_norm(x, w, residual=r, eps=1e-5, out_dtype=T.FP8)
        check((codes, scales), y.cpu())
