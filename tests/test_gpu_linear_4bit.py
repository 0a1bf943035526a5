"""The linear layer with 4-bit weights against its definition in 64 bits.

Tolerance of an element.  Every product is exact.  The sum of a group takes two instructions for each 32 columns and part of a token (bf16: one, fp32: three), each
off by 2^-23 of a partial sum, which holds codes and zero points raised by 16: below 4 sqrt(sum ((16 + max(15, zero)) scale x)^2).  Parts of an fp32 token are
exact.  Groups are added in fp32: one rounding each of a wavefront's share, 40 more for the wavefronts and ranges, below 4 q + |z|."""
import math

import pytest
import torch

from low_bits_calls import FOUR
from paper_2501_10054_amd import tardis as T
from test_gpu_linear import ACTS, check, inside, sigma

pytestmark = pytest.mark.gpu
DEV = "cuda"
# n, n_in, n_out
SIZES = [(1, 1, 1), (3, 7, 5), (1, 16384, 96), (2, 512, 16), (5, 2048, 300), (16, 4096, 64), (17, 40, 65), (31, 1000, 129), (33, 4096, 64),
         (64, 1408, 1000), (65, 129, 1030), (130, 1000, 257), (200, 2048, 512), (333, 1416, 1000), (700, 264, 776), (1, 128, 20000), (1025, 100, 40)]


def weights(n_out, n_in, group, dtype, gen, zeros, most=16):
    groups = -(-n_in // group)
    q = torch.randint(0, 16, (n_out, n_in), device=DEV, generator=gen, dtype=torch.uint8)
    scales = (torch.exp(torch.randn(n_out, groups, device=DEV, generator=gen)) * (0.2 / math.sqrt(n_in))).to(dtype)
    z = torch.randint(0, most, (n_out, groups), device=DEV, generator=gen, dtype=torch.uint8) if zeros else None
    return q, scales, z


def layer64(x, q, scales, zeros, b, act, group):
    n_in, parts = x.shape[1], 3 if x.dtype == torch.float32 else 1
    spread = lambda t: torch.repeat_interleave(t.double(), group, 1)[:, :n_in]
    s = spread(scales)
    z0 = torch.full_like(s, 8.0) if zeros is None else spread(zeros.clamp_max(128))
    x64 = x.double()
    w = s * (q.double() - z0)
    z = torch.mm(w, x64.t().contiguous()).t()
    size = torch.mm(w ** 2, (x64 ** 2).t().contiguous()).t().sqrt()
    raised = (s * (16.0 + z0.clamp_min(15.0))) ** 2
    inner = torch.zeros_like(z)
    for k in range(0, n_in, group):
        inner += torch.mm(raised[:, k:k + group], (x64[:, k:k + group] ** 2).t().contiguous()).t().sqrt()
    off = 2.0 ** -23 * (2 * parts * group // 32) * 4.0 * inner + (scales.shape[1] + 40) * 2.0 ** -24 * (4.0 * size + z.abs())
    if b is not None:
        z = z + b.double()
    return sigma(z, act), 1.13 * off + 2.0 ** -20 * z.abs()


@pytest.mark.parametrize("case", range(len(SIZES)))
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("gap", [0, 3])
def test_linear(case, group, dtype, gap):
    n, n_in, n_out = SIZES[case]
    gen = torch.Generator(device=DEV).manual_seed(3000 + 7 * case + gap + group)
    act = ACTS[(case + gap + group // 32) % 4]
    x = inside((n, n_in), dtype, gen, gap=gap, lead=case % 2)
    q, scales, zeros = weights(n_out, n_in, group, dtype, gen, (case + gap) % 2 == 0)
    W = T.tardis_pack_4bit(q, group)
    for out in (torch.float32, torch.bfloat16):
        b = torch.randn(n_out, device=DEV, generator=gen).to(out) if case % 2 == 0 else None
        r = torch.randn(n, n_out, device=DEV, generator=gen).to(out) if (case + gap) % 3 != 1 else None
        y = T.tardis_linear_4bit(x, W, scales, zeros, b, group=group, act=act, residual=r, out_dtype=out)
        want, off = layer64(x, q, scales, zeros, b, act, group)
        check(y, want if r is None else want + r.double(), off)


@pytest.mark.parametrize("group", [32, 64, 128])
def test_every_code_and_zero_point(group):
    """One column at a time: 16 codes by 256 zero points (above 128: 128), exactly."""
    n_in = 2 * group
    q = torch.arange(16, device=DEV, dtype=torch.uint8).repeat_interleave(256)[:, None].expand(-1, n_in).contiguous()
    zeros = torch.arange(256, device=DEV).repeat(16).to(torch.uint8)[:, None].expand(-1, 2).contiguous()
    scales = torch.ones(4096, 2, device=DEV, dtype=torch.bfloat16)
    for n in (1, 20, 100):
        x = torch.zeros(n, n_in, device=DEV, dtype=torch.bfloat16)
        at = torch.arange(n, device=DEV) * 37 % n_in
        x[torch.arange(n), at] = 3.0
        y = T.tardis_linear_4bit(x, T.tardis_pack_4bit(q, group), scales, zeros, group=group, out_dtype=torch.float32)
        want = 3.0 * (q[:, 0].float() - zeros[:, 0].clamp_max(128).float())
        assert torch.equal(y, want.expand(n, -1))


def test_the_order_of_columns():
    """A token that has one column finds that column's code."""
    gen = torch.Generator(device=DEV).manual_seed(4)
    for group, n_in in ((32, 70), (64, 100), (128, 300), (128, 256)):
        q = torch.randint(0, 16, (48, n_in), device=DEV, generator=gen, dtype=torch.uint8)
        scales = torch.ones(48, -(-n_in // group), device=DEV)
        for n in (n_in, 16):
            x = torch.eye(n_in, device=DEV)[:n]
            y = T.tardis_linear_4bit(x, T.tardis_pack_4bit(q, group), scales, group=group)
            assert torch.equal(y, q.float().t()[:n] - 8.0)


def test_codes_behind_the_last_column_count_for_nothing():
    gen = torch.Generator(device=DEV).manual_seed(5)
    for group, n_in in ((32, 33), (64, 100), (128, 129), (128, 5)):
        q, scales, zeros = weights(40, n_in, group, torch.bfloat16, gen, True)
        W = T.tardis_pack_4bit(q, group)
        full = torch.full((40, W.shape[1] * 8), 15, device=DEV, dtype=torch.uint8)
        full[:, :n_in] = q
        for n in (1, 20, 200):
            x = inside((n, n_in), torch.bfloat16, gen)           # (NaNs behind the last row)
            assert torch.equal(T.tardis_linear_4bit(x, T.tardis_pack_4bit(full, group), scales, zeros, group=group),
                               T.tardis_linear_4bit(x, W, scales, zeros, group=group))


def test_a_row_that_is_not_finite_stays_alone():
    gen = torch.Generator(device=DEV).manual_seed(7)
    for dtype in (torch.bfloat16, torch.float32):
        for n, n_in, n_out in [(5, 1000, 40), (40, 1408, 96), (200, 1001, 130)]:
            x = torch.randn(n, n_in, device=DEV, generator=gen).to(dtype)
            q, scales, zeros = weights(n_out, n_in, 128, dtype, gen, True)
            x[2, 3], x[3, 5] = math.nan, math.inf
            y = T.tardis_linear_4bit(x, T.tardis_pack_4bit(q, 128), scales, zeros)
            want, off = layer64(x, q, scales, zeros, None, "identity", 128)
            assert torch.isnan(y[2]).all() and torch.isnan(y[3]).all()
            fine = [0, 1] + list(range(4, n))
            check(y[fine], want[fine], off[fine])


def test_nothing_else_is_written_and_the_residual_may_be_the_output():
    gen = torch.Generator(device=DEV).manual_seed(6)
    for n, n_in, n_out in [(1, 4096, 517), (3, 300, 5), (64, 1000, 65), (333, 1408, 1000)]:
        x = torch.randn(n, n_in, device=DEV, generator=gen).bfloat16()
        q, scales, zeros = weights(n_out, n_in, 64, torch.bfloat16, gen, True)
        W = T.tardis_pack_4bit(q, 64)
        for out in (torch.float32, torch.bfloat16):
            store = torch.full((n * n_out + 16,), 7.0, device=DEV).to(out)
            r = store[5:5 + n * n_out].view(n, n_out)
            r.copy_(torch.randn(n, n_out, device=DEV, generator=gen))
            want = T.tardis_linear_4bit(x, W, scales, zeros, group=64, residual=r, out_dtype=out)
            T.tardis_linear_4bit(x, W, scales, zeros, group=64, residual=r, y=r, out_dtype=out)
            assert torch.equal(r, want) and (store[:5] == 7).all() and (store[5 + n * n_out:] == 7).all()


def test_without_working_memory():
    gen = torch.Generator(device=DEV).manual_seed(9)
    for n, n_in, n_out in [(1, 16384, 96), (8, 8192, 256), (100, 4001, 1000)]:
        x = torch.randn(n, n_in, device=DEV, generator=gen).bfloat16()
        q, scales, zeros = weights(n_out, n_in, 128, torch.bfloat16, gen, True)
        W = T.tardis_pack_4bit(q, 128)
        y = torch.empty(n, n_out, dtype=torch.float32, device=DEV)
        desc = T.tardis_linear_4bit_desc(n_in, n_out, T.BF16, T.F32, T.ACT["identity"], 128, W.data_ptr(), scales.data_ptr(), zeros.data_ptr(), None)
        want, off = layer64(x, q, scales, zeros, None, "identity", 128)
        for room in (0, 1000):
            work = torch.empty(room, dtype=torch.uint8, device=DEV) if room else None
            st = T.lib().tardis_linear_4bit(desc, x.data_ptr(), n, n_in, None, y.data_ptr(), None if work is None else work.data_ptr(), room,
                                            torch.cuda.current_stream().cuda_stream)
            assert st == T.OK
            check(y, want, off)


def test_no_rows():
    W, scales = torch.zeros(16, 16, dtype=torch.int32, device=DEV), torch.ones(16, 1, device=DEV)
    assert T.tardis_linear_4bit(torch.zeros(0, 128, device=DEV), W, scales).shape == (0, 16)


@pytest.mark.parametrize("call", range(len(FOUR)))
def test_every_kernel(call):
    """The calls of low_bits_calls.py, by which every kernel is reached."""
    _, n, n_in, n_out, group, dtype = FOUR[call]
    gen = torch.Generator(device=DEV).manual_seed(call)
    x = inside((n, n_in), T._TORCH_DTYPE[dtype], gen)
    q, scales, zeros = weights(n_out, n_in, group, x.dtype, gen, True)
    r = torch.randn(n, n_out, device=DEV, generator=gen)
    y = T.tardis_linear_4bit(x, T.tardis_pack_4bit(q, group), scales, zeros, group=group, act="relu", residual=r, out_dtype=torch.float32)
    want, off = layer64(x, q, scales, zeros, None, "relu", group)
    check(y, want + r.double(), off)
