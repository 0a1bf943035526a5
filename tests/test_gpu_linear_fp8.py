"""The linear layer on e4m3 codes with scales against its definition in 64 bits.

Tolerance of an element: as the layer's in bf16 (test_gpu_linear.py: K / 32 instructions and 40 more additions, each off by 2^-23 of a partial sum, which
stays below 4 q + |z|), and one rounding each for the token's and the column's scale: 2^-23 of z.  With outputs in bf16 the matrix instruction may drop of
each of K products what is below 2^-13 of the largest of 32: K errors of either sign, of at most 2^-13 max |x| max |W| each, whose sum stays below 4 sqrt(K)
of that."""
import math

import pytest
import torch

from low_bits_calls import EIGHT
from paper_2501_10054_amd import tardis as T
from test_gpu_linear import ACTS, SIZES, check, inside, sigma

pytestmark = pytest.mark.gpu
DEV = "cuda"


def codes(shape, gen, gap=0, lead=0):
    """Codes of normal values whose memory is surrounded by NaN codes"""
    n, k = shape
    store = torch.full((lead + n * (k + gap) + 4096,), 0x7F, dtype=torch.uint8, device=DEV).view(T.FP8)
    t = store[lead:lead + n * (k + gap)].view(n, k + gap)[:, :k]
    t.copy_((torch.randn(n, k, device=DEV, generator=gen) * 20.0).to(T.FP8))
    return t


def layer64(x, sx, W, sw, b, act, out=torch.bfloat16):
    x64, w64 = x.double(), W.double()
    if sx is not None:
        x64 = x64 * sx.double()[:, None]
    if sw is not None:
        w64 = w64 * sw.double()[:, None]
    z = torch.mm(w64, x64.t().contiguous()).t()
    q = torch.mm(w64 ** 2, (x64 ** 2).t().contiguous()).t().sqrt()
    off = (W.shape[1] / 32 + 40) * 2.0 ** -23 * (4.0 * q + z.abs()) + 2.0 ** -23 * z.abs()
    if out == torch.bfloat16:
        off = off + 4.0 * math.sqrt(W.shape[1]) * 2.0 ** -13 * x64.abs().amax(1)[:, None] * w64.abs().amax(1)
    if b is not None:
        z = z + b.double()
    return sigma(z, act), 1.13 * off + 2.0 ** -20 * z.abs()


def scales(n, gen, k):
    return torch.exp(torch.randn(n, device=DEV, generator=gen)) * (1.0 / (20.0 * k ** 0.25))


@pytest.mark.parametrize("case", range(len(SIZES)))
@pytest.mark.parametrize("gap", [0, 16, 3])
def test_linear(case, gap):
    n, n_in, n_out = SIZES[case]
    gen = torch.Generator(device=DEV).manual_seed(2000 + 7 * case + gap)
    act = ACTS[(case + gap) % 4]
    x, W = codes((n, n_in), gen, gap=gap), codes((n_out, n_in), gen)
    sx = scales(n, gen, n_in) if case % 5 else None
    sw = scales(n_out, gen, n_in) if case % 7 else None
    if sx is None or sw is None:
        act = "identity"
    for out in (torch.float32, torch.bfloat16):
        b = torch.randn(n_out, device=DEV, generator=gen).to(out) if case % 2 == 0 else None
        r = torch.randn(n, n_out, device=DEV, generator=gen).to(out) if (case + gap) % 3 != 1 else None
        y = T.tardis_linear_fp8(x, sx, W, sw, b, act=act, residual=r, out_dtype=out)
        want, off = layer64(x, sx, W, sw, b, act, out)
        check(y, want if r is None else want + r.double(), off)


def test_at_any_address_and_nothing_else_is_written():
    gen = torch.Generator(device=DEV).manual_seed(5)
    for n, n_in, n_out in [(1, 300, 77), (4, 256, 64), (70, 512, 200), (150, 1024, 136), (300, 4096, 512)]:
        x, W = codes((n, n_in), gen, lead=1), codes((n_out, n_in), gen, lead=3)
        sx, sw = scales(n, gen, n_in), scales(n_out, gen, n_in)
        for out in (torch.float32, torch.bfloat16):
            r = inside((n, n_out), out, gen, lead=1)
            y = torch.zeros(n * n_out + 8, dtype=out, device=DEV)
            got = T.tardis_linear_fp8(x, sx, W, sw, act="gelu_erf", residual=r, out_dtype=out, y=y[1:1 + n * n_out].view(n, n_out))
            want, off = layer64(x, sx, W, sw, None, "gelu_erf", out)
            check(got, want + r.double(), off)
            assert y[0] == 0 and (y[1 + n * n_out:] == 0).all()


def test_every_code():
    """All 256 codes on either side: products of every pair, summed with zeros."""
    every = torch.arange(256, dtype=torch.uint8, device=DEV).view(T.FP8)
    for n_in in (64, 256, 1000):
        x, W = torch.zeros(256, n_in, device=DEV).to(T.FP8), torch.zeros(256, n_in, device=DEV).to(T.FP8)
        x[:, n_in // 3], W[:, n_in // 3] = every, every
        y = T.tardis_linear_fp8(x, None, W, None, out_dtype=torch.float32)
        want = every.float()[:, None] * every.float()
        assert torch.equal(torch.isnan(y), torch.isnan(want))
        assert torch.equal(torch.nan_to_num(y), torch.nan_to_num(want))


def test_a_row_that_is_not_finite_stays_alone():
    gen = torch.Generator(device=DEV).manual_seed(7)
    for n, n_in, n_out in [(5, 1000, 40), (40, 1408, 96), (200, 1001, 130), (300, 520, 260)]:
        x, W = codes((n, n_in), gen), codes((n_out, n_in), gen)
        sx, sw = scales(n, gen, n_in), scales(n_out, gen, n_in)
        x[2, 3] = math.nan
        sx[3] = math.inf
        y = T.tardis_linear_fp8(x, sx, W, sw)
        want, off = layer64(x, sx, W, sw, None, "identity")
        assert torch.isnan(y[2]).all() and not torch.isfinite(y[3]).any()
        fine = [0, 1] + list(range(4, n))
        check(y[fine], want[fine], off[fine])


def test_without_working_memory():
    """The call does with less, or with none."""
    gen = torch.Generator(device=DEV).manual_seed(9)
    for n, n_in, n_out in [(1, 16384, 96), (300, 4001, 1000), (8, 8192, 256)]:
        x, W, sx, sw = codes((n, n_in), gen), codes((n_out, n_in), gen), scales(n, gen, n_in), scales(n_out, gen, n_in)
        y = torch.empty(n, n_out, dtype=torch.bfloat16, device=DEV)
        desc = T.tardis_linear_fp8_desc(n_in, n_out, T.BF16, T.ACT["identity"], W.data_ptr(), sw.data_ptr(), None)
        want, off = layer64(x, sx, W, sw, None, "identity")
        for room in (0, 1000):
            work = torch.empty(room, dtype=torch.uint8, device=DEV) if room else None
            st = T.lib().tardis_linear_fp8(desc, x.data_ptr(), sx.data_ptr(), n, n_in, None, y.data_ptr(), None if work is None else work.data_ptr(), room,
                                           torch.cuda.current_stream().cuda_stream)
            assert st == T.OK
            check(y, want, off)


def test_no_rows():
    W = torch.zeros(16, 64, device=DEV).to(T.FP8)
    assert T.tardis_linear_fp8(torch.zeros(0, 64, device=DEV).to(T.FP8), None, W, None).shape == (0, 16)


@pytest.mark.parametrize("call", range(len(EIGHT)))
def test_every_kernel(call):
    """The calls of low_bits_calls.py, by which every kernel is reached."""
    _, n, n_in, n_out, gap, out = EIGHT[call]
    gen = torch.Generator(device=DEV).manual_seed(call)
    out = T._TORCH_DTYPE[out]
    x, W, sx, sw = codes((n, n_in), gen, gap=gap), codes((n_out, n_in), gen), scales(n, gen, n_in), scales(n_out, gen, n_in)
    b, r = torch.randn(n_out, device=DEV, generator=gen).to(out), torch.randn(n, n_out, device=DEV, generator=gen).to(out)
    y = T.tardis_linear_fp8(x, sx, W, sw, b, act="relu", residual=r, out_dtype=out)
    want, off = layer64(x, sx, W, sw, b, "relu", out)
    check(y, want + r.double(), off)
