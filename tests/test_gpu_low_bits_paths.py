"""Layers in 8 and 4 bits on small whole numbers, whose products and sums every kernel has exactly: no tolerance but the rounding of the output.

e4m3: codes -3 .. 3, so products are whole, at most 9, and no instruction cuts anything from them (multiples of 2^(2 - 13) are kept); sums stay below 2^17.
4 bits: tokens -4 .. 4 and scales 1, 2 or 4: a group's sums of raised codes stay below 128 x 31 x 4 < 2^14, a row's terms add up to less than
16384 x 15 x 4 x 4 < 2^22.  Bias and residual are whole numbers below 2^10."""
import pytest
import torch

from low_bits_paths import FEW_TOKENS, LARGE_TILES
from paper_2501_10054_amd import tardis as T
from test_gpu_linear import check, inside, sigma

pytestmark = pytest.mark.gpu
DEV = "cuda"


def whole(gen, lo, hi, *shape):
    return torch.randint(lo, hi + 1, shape, device=DEV, generator=gen)


def padded(t, dtype, gen, gap=0):
    """t in memory that is surrounded by NaNs"""
    if dtype == T.FP8:
        store = torch.full((t.shape[0] * (t.shape[1] + gap) + 4096,), 0x7F, dtype=torch.uint8, device=DEV).view(T.FP8)
        to = store[:t.shape[0] * (t.shape[1] + gap)].view(t.shape[0], -1)[:, :t.shape[1]]
    else:
        to = inside(t.shape, dtype, gen, gap=gap)
    to.copy_(t.to(dtype))
    return to


@pytest.mark.parametrize("gap", [0, 16])
@pytest.mark.parametrize("n,n_in,n_out,launches", LARGE_TILES)
def test_large_tiles(n, n_in, n_out, launches, gap):
    gen = torch.Generator(device=DEV).manual_seed(n + n_in)
    x, W = (padded(whole(gen, -3, 3, rows, n_in), T.FP8, gen, g) for rows, g in ((n, gap), (n_out, 0)))
    z = torch.mm(x.float(), W.float().t().contiguous())
    b, r = whole(gen, -500, 500, n_out).bfloat16(), whole(gen, -500, 500, n, n_out).bfloat16()
    halves, twos = 2.0 ** -(whole(gen, 0, 3, n).float()), 2.0 ** whole(gen, 0, 3, n_out).float()
    run = lambda **kw: T.tardis_linear_fp8(x, None, W, None, **kw)
    assert torch.equal(run(), z.bfloat16())
    assert torch.equal(run(b=b, act="relu", residual=r), ((z + b.float()).clamp_min(0) + r.float()).bfloat16())
    assert torch.equal(T.tardis_linear_fp8(x, halves, W, twos, b, residual=r), (z * halves[:, None] * twos + b.float() + r.float()).bfloat16())
    # GELU of numbers whose sums are exact: only its own error and the rounding
    small = 2.0 ** -9 * torch.ones(n, device=DEV)
    want = sigma(z.double() / 512 + b.double() / 512, "gelu_erf")
    off = 2.0 ** -20 * (z.double() / 512 + b.double() / 512).abs()
    for residual in (None, r):
        y = T.tardis_linear_fp8(x, small, W, None, (b.float() / 512).bfloat16(), act="gelu_erf", residual=residual)
        if residual is None:
            # (for outputs in bf16 without a residual sigma itself is good to bf16's rounding: test_gpu_linear_gelu.py)
            check(y, want, off + 2.0 ** -8 * want.abs())
        else:
            check(y, want + r.double(), off)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n,n_in,n_out,dtype,rows,chunks", FEW_TOKENS)
def test_few_tokens(n, n_in, n_out, dtype, rows, chunks, group):
    gen = torch.Generator(device=DEV).manual_seed(n + n_in + group)
    dtype = T._TORCH_DTYPE[dtype]
    four_bits(gen, n, n_in, n_out, group, dtype)


def four_bits(gen, n, n_in, n_out, group, dtype, gap=3):
    groups = -(-n_in // group)
    x = padded(whole(gen, -4, 4, n, n_in), dtype, gen, gap)
    q, zeros = whole(gen, 0, 15, n_out, n_in).to(torch.uint8), whole(gen, 0, 15, n_out, groups).to(torch.uint8)
    scales = (2.0 ** whole(gen, 0, 2, n_out, groups).float()).to(dtype)
    W = T.tardis_pack_4bit(q, group)
    b, r = whole(gen, -500, 500, n_out).float(), whole(gen, -500, 500, n, n_out).float()
    for z0 in (zeros, None):
        spread = lambda t: torch.repeat_interleave(t.double(), group, 1)[:, :n_in]
        weights = (q.double() - (8.0 if z0 is None else spread(z0))) * spread(scales)
        z = torch.mm(x.double(), weights.t().contiguous())
        assert z.abs().max() < 2 ** 22
        assert torch.equal(T.tardis_linear_4bit(x, W, scales, z0, group=group, out_dtype=torch.float32), z.float())
        y = T.tardis_linear_4bit(x, W, scales, z0, b, group=group, act="relu", residual=r, out_dtype=torch.float32)
        assert torch.equal(y, ((z + b.double()).clamp_min(0) + r.double()).float())
        b16, r16 = b.bfloat16(), r.bfloat16()
        y = T.tardis_linear_4bit(x, W, scales, z0, b16, group=group, residual=r16, out_dtype=torch.bfloat16)
        assert torch.equal(y, (z + b16.double() + r16.double()).float().bfloat16())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,n_in,n_out,group", [(2 * 16384 + 5, 200, 40, 32), (16384 + 64, 70, 130, 64), (16384 + 1, 129, 17, 128)])
def test_more_tokens_than_are_done_together(n, n_in, n_out, group, dtype):
    """16384 at a time: the rest of the tokens is a call of its own, also of a few."""
    gen = torch.Generator(device=DEV).manual_seed(n)
    four_bits(gen, n, n_in, n_out, group, dtype)
