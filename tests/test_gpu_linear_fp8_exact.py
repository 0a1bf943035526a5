"""What sums of the layer on e4m3 codes may lose: nothing where exact sums are asked for, and by default, for outputs in bf16, what the header says.

Bounds.  fp32 sums: K / 32 instructions and 40 more additions, each off by 2^-23 of a partial sum, which stays below S = sum |x W| (terms of one sign are
among the inputs).  By default each of the products of eight neighbouring columns is cut to a multiple of 2^(e - 13), e the largest sum of two codes'
exponents, which keeps the product that has it whole: at most 7 2^-13 sum 2^e < 2^-10 S', S' the sum with codes below 2^-6 taken as 2^-6.  Normal values: seven errors of an
eight are independent, of either sign and below g = 2^-13 of its largest product, so of a mean square below g^2 / 3 each.
Residuals that take the sum away leave only its errors: the result's rounding is then 2^-8 of a small number."""
import math

import pytest
import torch

import test_gpu_linear_fp8 as eight
from paper_2501_10054_amd import tardis as T
from test_gpu_linear import ACTS, SIZES, check

pytestmark = pytest.mark.gpu
DEV = "cuda"
# tiles of the faster instruction, the large ones, K in ranges, and few tokens, whose sums are always exact
CALLS = [(40, 8192, 4096), (64, 4096, 11008), (333, 11008, 4096), (700, 2048, 8192), (150, 11008, 1024), (512, 1000, 4096), (4, 4096, 512)]


def _inputs(kind, n, n_in, n_out, gen):
    def pick(rows, values):
        v = torch.tensor(values, device=DEV)
        return v[torch.randint(0, len(values), (rows, n_in), device=DEV, generator=gen)]

    first = torch.arange(n_in, device=DEV) % 8 == 3
    if kind == "one large of eight":                    # the large ones of either sign, the small ones of one
        sign = torch.where(torch.arange(n_in, device=DEV) // 8 % 2 == 0, 1.0, -1.0)
        x, W = pick(n, [2.25, 2.5, 2.75]), pick(n_out, [2.25, 2.5, 2.75])
        x, W = torch.where(first, 256.0 * sign, x), torch.where(first, pick(n_out, [208.0, 256.0]), W)
    elif kind == "subnormal codes":                     # a large code meets a subnormal one
        x, W = pick(n, [1.75 / 64, 1.875 / 64]), pick(n_out, [1 / 64, 1.125 / 64])
        x, W = torch.where(first, 448.0, x), torch.where(first, pick(n_out, [1 / 512, -1 / 512]), W)
    elif kind == "every code":
        def some(rows):
            c = torch.randint(0, 127, (rows, n_in), device=DEV, generator=gen) + 128 * torch.randint(0, 2, (rows, n_in), device=DEV, generator=gen)
            return c.to(torch.uint8).view(T.FP8)
        return some(n), some(n_out)
    elif kind == "of one sign":
        x, W = (torch.randn(rows, n_in, device=DEV, generator=gen).abs() * 20 for rows in (n, n_out))
    else:
        return eight.codes((n, n_in), gen), eight.codes((n_out, n_in), gen)
    return x.to(T.FP8), W.to(T.FP8)


KINDS = ["normal", "of one sign", "every code", "one large of eight", "subnormal codes"]


def _sums(x, W):
    """z, S, S' in 64 bits"""
    def raised(t):
        t = t.double().abs()
        return torch.where(t > 0, t.clamp_min(2.0 ** -6), t)

    mm = lambda a, b: torch.mm(a, b.t().contiguous())
    return mm(x.double(), W.double()), mm(x.double().abs(), W.double().abs()), mm(raised(x), raised(W))


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("call", range(len(CALLS)))
def test_what_a_sum_loses(call, kind):
    n, n_in, n_out = CALLS[call]
    gen = torch.Generator(device=DEV).manual_seed(100 * call + KINDS.index(kind))
    x, W = _inputs(kind, n, n_in, n_out, gen)
    z, S, raised = _sums(x, W)
    sums = (n_in / 32 + 40) * 2.0 ** -23 * S
    r = (-z).bfloat16()
    for residual in (None, r):
        want = z if residual is None else z + r.double()
        for exact in (True, False):
            y = T.tardis_linear_fp8(x, None, W, None, residual=residual, exact=exact)
            check(y, want, sums if exact else sums + 2.0 ** -10 * raised)


@pytest.mark.parametrize("call", [(333, 11008, 4096), (700, 2048, 8192)])
def test_what_normal_values_lose(call):
    n, n_in, n_out = call
    gen = torch.Generator(device=DEV).manual_seed(n)
    x, W = _inputs("normal", n, n_in, n_out, gen)
    z, _, _ = _sums(x, W)
    r = (-z).bfloat16()
    rows, cols = torch.arange(0, n, n // 32, device=DEV)[:32], torch.arange(0, n_out, n_out // 64, device=DEV)[:64]
    y = T.tardis_linear_fp8(x, None, W, None, residual=r)
    want = z + r.double()
    err = (y.double() - want)[rows][:, cols]
    p = x[rows].double()[:, None, :] * W[cols].double()
    lost = (7.0 / 3.0 * (2.0 ** -13 * p.abs().view(len(rows), len(cols), -1, 8).amax(3)) ** 2).sum(2)
    rounded = (2.0 ** -8 * want[rows][:, cols]) ** 2
    rms = err.pow(2).mean().sqrt()
    assert rms <= (lost + rounded).mean().sqrt(), (rms.item(), lost.mean().sqrt().item())
    relative = (err.pow(2).mean() / p.pow(2).sum(2).mean()).sqrt().item()
    print(f"{call}: {relative:.2e} of the root of the squares' sum")


@pytest.mark.parametrize("case", range(len(SIZES)))
@pytest.mark.parametrize("gap", [0, 3])
def test_exact_sums(case, gap):
    """The layer's own test, with exact sums: bound as for outputs in fp32."""
    n, n_in, n_out = SIZES[case]
    gen = torch.Generator(device=DEV).manual_seed(5000 + 7 * case + gap)
    act = ACTS[(case + gap) % 4]
    x, W = eight.codes((n, n_in), gen, gap=gap), eight.codes((n_out, n_in), gen)
    sx, sw = eight.scales(n, gen, n_in), eight.scales(n_out, gen, n_in)
    b = torch.randn(n_out, device=DEV, generator=gen).bfloat16() if case % 2 == 0 else None
    r = torch.randn(n, n_out, device=DEV, generator=gen).bfloat16() if (case + gap) % 3 != 1 else None
    y = T.tardis_linear_fp8(x, sx, W, sw, b, act=act, residual=r, exact=True)
    want, off = eight.layer64(x, sx, W, sw, b, act, torch.float32)
    check(y, want if r is None else want + r.double(), off)
    # in fp32 the same sums
    full = T.tardis_linear_fp8(x, sx, W, sw, None if b is None else b.float(), act=act, residual=None if r is None else r.float(), out_dtype=torch.float32, exact=True)
    check(full, want if r is None else want + r.double(), off)


def test_exact_sums_in_a_graph_and_on_another_stream():
    gen = torch.Generator(device=DEV).manual_seed(11)
    x, W = eight.codes((150, 4096), gen), eight.codes((1000, 4096), gen)
    sx, sw = eight.scales(150, gen, 4096), eight.scales(1000, gen, 4096)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = T.tardis_linear_fp8(x, sx, W, sw, act="gelu_erf", stream=side, exact=True)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(other, T.tardis_linear_fp8(x, sx, W, sw, act="gelu_erf", exact=True))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = T.tardis_linear_fp8(x, sx, W, sw, act="gelu_erf", exact=True)
    for _ in range(3):
        x.copy_((torch.randn(150, 4096, device=DEV, generator=gen) * 20.0).to(T.FP8))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, T.tardis_linear_fp8(x, sx, W, sw, act="gelu_erf", exact=True))
        want, off = eight.layer64(x, sx, W, sw, None, "gelu_erf", torch.float32)
        check(y, want, off)
        torch.cuda.synchronize()
