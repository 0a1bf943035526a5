"""Every activation of the linear layer takes a NaN for a NaN, and an infinity for what the function has there."""
import math

import pytest
import torch

from paper_2501_10054_amd import tardis as T
from test_gpu_linear import ACTS

pytestmark = pytest.mark.gpu
DEV = "cuda"
# (staged, direct, ranges of K that are joined, large tiles)
SIZES = [(5, 1, 3), (40, 129, 96), (64, 64, 64), (8, 16384, 256), (333, 11008, 1024), (2048, 512, 4096)]


@pytest.mark.parametrize("n,n_in,n_out", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("act", ACTS)
def test_a_nan_stays_a_nan(n, n_in, n_out, dtype, act):
    gen = torch.Generator(device=DEV).manual_seed(n + n_in)
    x = torch.randn(n, n_in, device=DEV, generator=gen).to(dtype)
    W = torch.randn(n_out, n_in, device=DEV, generator=gen).mul_(0.05).to(dtype)
    x[n // 2, n_in - 1], x[0] = math.nan, 0.0
    x[0, 0], W[:, 0] = math.inf, 1.0
    W[0, 0] = -1.0
    for out in (torch.bfloat16, torch.float32):
        for residual in (None, torch.ones(n, n_out, dtype=out, device=DEV)):
            y = T.tardis_linear(x, W, act=act, residual=residual, out_dtype=out)
            assert torch.isnan(y[n // 2]).all()
            assert torch.isfinite(y[1:n // 2]).all() and torch.isfinite(y[n // 2 + 1:]).all()
            assert (y[0, 1:] == math.inf).all()
            if act == "relu":
                assert y[0, 0] == (0.0 if residual is None else 1.0)
            else:                                    # -inf; GELU is -inf times 0 there
                assert y[0, 0] == -math.inf if act == "identity" else torch.isnan(y[0, 0])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("act", ACTS)
def test_a_nan_in_a_group_stays_a_nan(dtype, act):
    gen = torch.Generator(device=DEV).manual_seed(4)
    for rows, n_in, n_out in ((24, 512, 64), (24, 511, 64), (1024, 512, 2048)):
        x = torch.randn(rows, n_in, device=DEV, generator=gen).to(dtype)
        W = torch.randn(2, n_out, n_in, device=DEV, generator=gen).mul_(0.05).to(dtype)
        x[rows // 3, 7] = math.nan
        offsets = torch.tensor([0, rows // 2, rows], dtype=torch.int32, device=DEV)
        y = T.tardis_grouped_linear(x, W, offsets, act=act)
        assert torch.isnan(y[rows // 3]).all() and torch.isnan(y).sum() == n_out
