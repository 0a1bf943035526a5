"""Calls of linear layers and experts at the limits of what a launch takes, against 64 bits (tolerances as in test_gpu_linear)."""
import math

import pytest
import torch

from paper_2501_10054_amd import tardis as T
from test_gpu_linear import check

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("dtype,tokens,n_out,experts", [(torch.bfloat16, 4096, 32768, 4096), (torch.float32, 65536, 2048, 65536)])
def test_many_experts_with_few_tokens(dtype, tokens, n_out, experts):
    """Tiles of few rows would be more than a launch takes.  n_in = 8: a sum of at most 8 products."""
    gen = torch.Generator(device=DEV).manual_seed(21)
    x = torch.randn(tokens, 8, device=DEV, generator=gen).to(dtype)
    W = torch.empty(experts, n_out, 8, dtype=dtype, device=DEV)
    for e in range(0, experts, 1024):
        W[e:e + 1024] = torch.randn(W[e:e + 1024].shape, device=DEV, generator=gen)
    chosen, slots = torch.sort(torch.randint(0, experts, (tokens,), device=DEV, generator=gen), stable=True)
    offsets = torch.searchsorted(chosen, torch.arange(experts + 1, device=DEV)).int()
    y = T.tardis_grouped_linear(x, W, offsets, act="relu", order=slots.int(), out_dtype=torch.bfloat16)
    step = (1 << 23) // n_out
    for p in range(0, tokens, step):
        terms = W[chosen[p:p + step]].double() * x[slots[p:p + step]].double()[:, None, :]
        z, q = terms.sum(-1), (terms ** 2).sum(-1).sqrt()
        off = (8 + 40) * 2.0 ** -23 * (4.0 * q + z.abs())
        check(y[p:p + step], z.clamp_min(0.0), off)
    assert math.isfinite(y.float().abs().max().item())
