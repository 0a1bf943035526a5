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


@pytest.mark.parametrize("per_token", [1, 2, 64, (1 << 30) - 1, 1 << 30])
@pytest.mark.parametrize("n_in,n_out,positions", [(64, 24, 20), (63, 24, 20), (256, 512, 1500)])
def test_negative_slots_are_of_no_token(per_token, n_in, n_out, positions):
    """Whatever the experts of a token: their rows are left as they are."""
    gen = torch.Generator(device=DEV).manual_seed(per_token % 1000)
    x = torch.randn(8, n_in, device=DEV, generator=gen).bfloat16()
    W = torch.randn(2, n_out, n_in, device=DEV, generator=gen).mul_(0.1).bfloat16()
    order = torch.randint(0, min(8 * per_token, (1 << 31) - 1), (positions,), device=DEV, generator=gen).int()
    bad = torch.rand(positions, device=DEV, generator=gen) < 0.3
    order[bad] = torch.tensor([-1, -2, -64, -(1 << 30), -(1 << 31)], device=DEV).int()[torch.arange(int(bad.sum()), device=DEV) % 5]
    offsets = torch.tensor([0, positions // 3, positions], device=DEV).int()
    y = torch.full((positions, n_out), 5.0, device=DEV)
    T.tardis_grouped_linear(x, W, offsets, order=order, per_token=per_token, out_dtype=torch.float32, y=y)
    assert (y[bad] == 5.0).all()
    expert = (torch.arange(positions, device=DEV) >= positions // 3).long()
    token = torch.div(order.long().clamp_min(0), per_token, rounding_mode="floor")
    for e in range(2):
        p = torch.nonzero(~bad & (expert == e)).flatten()
        terms = torch.mm(W[e].double(), x[token[p]].double().t().contiguous()).t()
        check(y[p], terms, (n_in / 32 + 40) * 2.0 ** -23 * (4.0 * torch.mm(W[e].double() ** 2, (x[token[p]].double() ** 2).t().contiguous()).t().sqrt() + terms.abs()))


def test_a_sum_of_experts_of_more_than_2_to_the_32_threads():
    """One slot with weight 1 for a token: its row of z as it is."""
    torch.cuda.empty_cache()
    n, d = (1 << 21) + 3, 16384
    gen = torch.Generator(device=DEV).manual_seed(8)
    z = torch.randn(7, d, device=DEV, generator=gen).bfloat16()
    place = torch.randint(-1, 7, (n, 1), device=DEV, generator=gen).int()
    y = T.tardis_moe_combine(z, place, torch.ones(n, 1, device=DEV))
    z8 = torch.cat([z, torch.zeros(1, d, device=DEV).bfloat16()])       # (a place of -1: the last)
    for t in range(0, n, 1 << 16):
        assert torch.equal(y[t:t + (1 << 16)], z8[place[t:t + (1 << 16), 0].long()])
    del y
    torch.cuda.empty_cache()


def test_copies_of_more_than_2_to_the_32_pieces():
    """Rows of an odd length, 64 GB of them: their aligned copy has every row in its place."""
    torch.cuda.empty_cache()
    n, n_in, n_out = 4194309, 8191, 2048
    gen = torch.Generator(device=DEV).manual_seed(9)
    some = torch.randn(999, n_in, device=DEV, generator=gen).bfloat16()
    W = (torch.randn(n_out, n_in, device=DEV, generator=gen) * 0.02).bfloat16()
    x = torch.empty(n, n_in, dtype=torch.bfloat16, device=DEV)
    for m in range(0, n, 999):
        x[m:m + 999] = some[:min(999, n - m)]
    y = T.tardis_linear(x, W)
    terms = torch.mm(some.double(), W.double().t().contiguous())
    q = torch.mm(some.double() ** 2, (W.double() ** 2).t().contiguous()).sqrt()
    off = (n_in / 32 + 40) * 2.0 ** -23 * (4.0 * q + terms.abs())
    for m in (0, 999 * 1024, 999 * 2099, 999 * 2100, 999 * 4197, n // 999 * 999):
        rows = min(999, n - m)
        check(y[m:m + rows], terms[:rows], off[:rows])
    first = y[:999 * 1024].view(1024, 999, n_out)
    for m in range(0, n - 999 * 1024, 999 * 1024):   # (the order of a sum goes by the tile: results below 16 may be rounded to neighbours, 2^-4 apart)
        assert (y[m:m + 999 * 1024].view_as(first).float() - first.float()).abs().max().item() < 0.1
    del x, y, first
    torch.cuda.empty_cache()


def test_the_last_token_of_a_prompt():
    """One row of a tensor whose rows are a prompt apart, and as it is by itself: the same call."""
    gen = torch.Generator(device=DEV).manual_seed(10)
    W = (torch.randn(512, 4096, device=DEV, generator=gen) * 0.02).bfloat16()
    prompt = torch.randn(1, 1500, 4096, device=DEV, generator=gen).bfloat16()
    last = prompt[:, -1]
    assert last.stride(0) * 2 > 1 << 23
    assert torch.equal(T.tardis_linear(last, W), T.tardis_linear(last.reshape(-1).clone()[None], W))
    far = torch.as_strided(prompt, (1, 4096), ((1 << 30) + 1, 1))
    assert torch.equal(T.tardis_linear(far, W), T.tardis_linear(prompt[:, 0].clone(), W))
