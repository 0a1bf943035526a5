"""GELU in the linear layer at its own accuracy: rows whose pre-activation is exact (one weight of 1, the others 0), against 64 bits.

Tolerances.  Alone and for outputs in bf16 GELU is z Phi(z) with Phi(-|z|) off by less than 2^-14 of itself (a fit, 3.4e-5, and five fp32 steps and two
approximations of 2^-22); with a residual, or for outputs in fp32, its error is below 2^-20 of z.  The residual's addition rounds by 2^-24 of the sum of
its terms' sizes, and the result is rounded once more to the type of y.  Below -13 GELU leaves the normal values: 1e-37 more."""
import math

import pytest
import torch

from paper_2501_10054_amd import tardis as T
from test_gpu_linear_tiles import _instances, _lib, ptr, tile

pytestmark = pytest.mark.gpu
DEV = "cuda"
GELU16 = 4                                                   # kActGelu16 of linear.h


def gelu64(z):
    """GELU, and Phi(-|z|)"""
    z = z.double()
    q = 0.5 * torch.special.erfc(z.abs() / math.sqrt(2.0))
    return z * torch.where(z > 0, 1.0 - q, q), q


def one_hot(n, n_in, n_out, dtype, gen, std):
    """x, W and the pre-activations z of the rows: x W^T has z[m] in all columns of row m"""
    x, W = torch.zeros(n, n_in, dtype=dtype, device=DEV), torch.zeros(n_out, n_in, dtype=dtype, device=DEV)
    z = (torch.randn(n, device=DEV, generator=gen) * std).bfloat16()
    x[:, n_in // 2], W[:, n_in // 2] = z.to(dtype), 1.0
    return x, W, z


def within(y, want, off):
    bound = off + (torch.finfo(y.dtype).eps / 2) * (want.abs() + off) + 1e-37
    worst = ((y.double() - want).abs() / bound).max().item()
    assert worst <= 1.0, worst


# (rows of one element and of an odd number, of whole pieces; ranges of K that are joined; large tiles)
@pytest.mark.parametrize("n,n_in,n_out", [(3000, 1, 4), (333, 129, 70), (3000, 64, 64), (1, 4096, 512), (8, 16384, 256), (333, 11008, 1024), (2048, 512, 4096)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
def test_a_residual_that_cancels(n, n_in, n_out, dtype, out):
    """The sum is rounded once: where the residual takes GELU's result away, GELU's own error is what is left."""
    gen = torch.Generator(device=DEV).manual_seed(n + n_in)
    x, W, z = one_hot(n, n_in, n_out, dtype, gen, 1.6)
    g, _ = gelu64(z)
    r = (-g)[:, None].repeat(1, n_out).to(out)
    r[:, 1::2] = torch.randn(r[:, 1::2].shape, device=DEV, generator=gen).to(out)
    y = T.tardis_linear(x, W, act="gelu_erf", residual=r, out_dtype=out)
    size = g.abs()[:, None] + r.double().abs()
    within(y, g[:, None] + r.double(), 2.0 ** -20 * z.double().abs()[:, None] + 2.0 ** -24 * size)


@pytest.mark.parametrize("f32,direct,shape", _instances())
def test_every_kernel(f32, direct, shape):
    """By its number, alone and with a residual."""
    lib = _lib()
    m, n, sl = tile(lib, direct, shape)
    es, dtype = (4, torch.float32) if f32 else (2, torch.bfloat16)
    gen = torch.Generator(device=DEV).manual_seed(100 * shape + 10 * f32 + direct)
    rows, n_out, n_in = 2 * m + 5, n + 8, 2 * sl // es
    x, W, z = one_hot(rows, n_in, n_out, dtype, gen, 2.5)
    g, q = gelu64(z)
    r = (-g)[:, None].repeat(1, n_out).bfloat16()
    for act, residual in ((GELU16, None), (T.ACT["gelu_erf"], r)):
        y = torch.empty(rows, n_out, dtype=torch.bfloat16, device=DEV)
        st = lib.linear_probe(f32, direct, shape, ptr(x), rows, n_in * es, ptr(W), None, ptr(residual), ptr(y), rows, n_out, n_in * es, act, 0, 1, None, None, 0, 1,
                              torch.cuda.current_stream().cuda_stream)
        assert st == T.OK
        zz = z.double().abs()[:, None]
        if residual is None:
            within(y, g[:, None].expand(-1, n_out), 2.0 ** -14 * q[:, None] * zz)
        else:
            within(y, g[:, None] + r.double(), 2.0 ** -20 * zz + 2.0 ** -24 * (g.abs()[:, None] + r.double().abs()))
