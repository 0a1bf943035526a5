"""Tokens in fp32 on 4-bit weights: sums are as good as those of fp32, although codes and zero points are multiplied with 16 added to them.

Bound, for the mean square of the errors of a call.  Of a token's three parts in bf16 the head's products are 2^8 and 2^16 times the others', whose sums are apart, so
that the head's instructions alone count: two for each 32 columns (codes, zero points), each off by 2^-24 of the raised products that it adds, R = sqrt(sum ((16 +
max(15, zero)) x)^2) of its columns.  Behind them a sum of fp32 for each group, and 40 more, each off by 2^-24 of the row's sum at most."""
import math

import pytest
import torch

from paper_2501_10054_amd import tardis as T
from test_gpu_linear_4bit import weights

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n,n_in,n_out", [(1, 1408, 2048), (1, 640, 272), (1, 4096, 512), (4, 784, 1000), (16, 2048, 300), (40, 1408, 512), (100, 512, 2000)])
def test_sums_of_fp32(n, n_in, n_out, group, zeros):
    off, err = [], []
    for seed in range(16):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        x = torch.randn(n, n_in, device=DEV, generator=gen)
        x[:, torch.randperm(n_in, device=DEV, generator=gen)[:max(1, n_in // 100)]] *= 8.0
        q, scales, z0 = weights(n_out, n_in, group, torch.float32, gen, zeros)
        y = T.tardis_linear_4bit(x, T.tardis_pack_4bit(q, group), scales, z0, group=group)
        spread = lambda t: torch.repeat_interleave(t.double(), group, 1)[:, :n_in]
        zero = spread(z0) if zeros else torch.full((n_out, n_in), 8.0, device=DEV, dtype=torch.float64)
        want = torch.mm(x.double(), ((q.double() - zero) * spread(scales)).t().contiguous())
        raised = ((16.0 + zero.clamp_min(15.0)) * spread(scales)) ** 2
        inner = 2.0 * torch.mm(x.double() ** 2, raised.t().contiguous())       # (two instructions for each 32 columns: R^2 of all of them)
        off.append((2.0 ** -48 * (inner + (scales.shape[1] + 40) * want ** 2)).mean().item())
        err.append((y.double() - want).pow(2).mean().item())
    rms, bound = math.sqrt(sum(err)), math.sqrt(sum(off))
    assert rms <= bound, rms / bound
