"""Sums of the layer on e4m3 codes with outputs in bf16 where they are asked to be exact: the bounds of outputs in fp32."""
import pytest
import torch

import test_gpu_linear_fp8 as eight
from paper_2501_10054_amd import tardis as T
from test_gpu_linear import ACTS, SIZES, check

pytestmark = pytest.mark.gpu
DEV = "cuda"


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
