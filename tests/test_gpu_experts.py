"""The router's choice (whole numbers equal, weights within the roundings of an exponential, a sum and a quotient) and the sum of the
experts' outputs, against their definition in 64 bits; the four steps of a mixture of experts together, on another stream and in a graph."""
import math

import numpy as np
import pytest
import torch

from paper_2501_10054_amd import tardis as T
from test_gpu_linear import check, inside, sigma

pytestmark = pytest.mark.gpu
DEV = "cuda"


def route64(logits, k, renormalise):
    l = logits.double().cpu().numpy()
    n, experts = l.shape
    l = np.where(np.isnan(l), -np.inf, l)
    rank = np.argsort(-l, axis=1, kind="stable")[:, :k]
    top = np.take_along_axis(l, rank, 1)
    ids = np.where(top > -np.inf, rank, -1)
    most = l.max(1, keepdims=True)
    with np.errstate(invalid="ignore"):
        p = np.where(l == -np.inf, 0.0, np.where(l == most, 1.0, np.exp(l - most)))
    chosen = np.where(ids >= 0, np.take_along_axis(p, rank, 1), 0.0)
    total = (chosen if renormalise else p).sum(1, keepdims=True)
    weights = chosen / np.where(total > 0, total, 1.0)
    flat = ids.reshape(-1)
    slots = np.flatnonzero(flat >= 0)
    slots = slots[np.argsort(flat[slots], kind="stable")]
    order, place = np.full(n * k, -1), np.full(n * k, -1)
    order[:slots.size] = slots
    place[slots] = np.arange(slots.size)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[flat >= 0], minlength=experts))])
    return ids, weights, offsets, order, place.reshape(n, k)


@pytest.mark.parametrize("experts,k", [(1, 1), (2, 2), (7, 3), (16, 16), (17, 1), (32, 4), (60, 4), (64, 6), (100, 8), (128, 8), (129, 2), (256, 8), (500, 16),
                                       (512, 10), (1000, 5), (1024, 16)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_route(experts, k, dtype):
    """weights: the exponential is off by at most 2 units in the last place and its argument is rounded once (2^-24 of up to 20), the sum of up to
    1024 terms by 2^-24 of each partial sum in a chain of at most 16 + 10 additions, the quotient once."""
    gen = torch.Generator(device=DEV).manual_seed(experts * 31 + k)
    for n in (0, 1, 5, 63, 64, 65, 256, 257, 300, 1500, 5000):
        logits = (torch.randn(n, experts, device=DEV, generator=gen) * 2.0).to(dtype)
        if n > 4:
            logits[:, torch.rand(experts, device=DEV, generator=gen) < 0.2] = -math.inf
            logits[torch.rand(n, device=DEV, generator=gen) < 0.1] = -math.inf
            logits[1] = 0.5                                          # ties all over
            logits[2, experts // 2] = math.inf
            logits[3, experts - 1] = math.nan
            logits[4] = torch.finfo(dtype).min                       # the type's lowest value is a logit like others
        for renormalise in (True, False):
            got = T.tardis_moe_route(logits, k, renormalise=renormalise)
            want = route64(logits, k, renormalise)
            for name, g, w in zip(("ids", "weights", "offsets", "order", "place"), got, want):
                g = g.cpu().numpy()
                if name == "weights":
                    assert g.dtype == np.float32
                    assert (np.abs(g - w) <= (20 + 2 * 2 + 26 + 2) * 2.0 ** -24 * w + 1e-37).all(), (n, renormalise)
                else:
                    assert np.array_equal(g, w), (n, renormalise, name)


@pytest.mark.parametrize("d", [1, 7, 64, 100, 1001, 2048, 4096])
@pytest.mark.parametrize("k", [1, 2, 8, 9, 17])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_combine(d, k, dtype):
    """A chain of k fused multiply-adds and the residual's addition, each off by 2^-24 of a partial sum, then one rounding."""
    gen = torch.Generator(device=DEV).manual_seed(d + k)
    for n in (1, 6, 130):
        rows = n * k + 3
        z = inside((rows, d), dtype, gen)
        z[rows - 1] = math.nan                                       # a row that no slot has
        place = torch.randperm(rows - 1, device=DEV, generator=gen)[:n * k].view(n, k).int()
        place[torch.rand(n, k, device=DEV, generator=gen) < 0.1] = -1
        place[0, 0] = rows if n > 1 else place[0, 0]                 # past the last row: dropped as well
        if n > 2:
            place[2] = -1
        w = torch.rand(n, k, device=DEV, generator=gen)
        w[place < 0] = math.nan                                      # (never used)
        for out in (torch.float32, torch.bfloat16):
            r = torch.randn(n, d, device=DEV, generator=gen).to(out) if k != 2 else None
            y = T.tardis_moe_combine(z, place, w, residual=r, out_dtype=out)
            there = (place >= 0) & (place < rows)
            terms = torch.where(there, w.double(), 0.0)[..., None] * torch.where(there[..., None], z.double()[place.clamp(0, rows - 1).long()], 0.0)
            want, size = terms.sum(1), terms.abs().sum(1)
            if r is not None:
                want, size = want + r.double(), size + r.double().abs()
            check(y, want, (k + 1) * 2.0 ** -24 * size)
            if n > 2:
                assert torch.equal(y[2], r[2] if r is not None else torch.zeros_like(y[2]))


def test_combine_of_nothing():
    r = torch.randn(3, 40, device=DEV)
    none = torch.full((3, 2), -1, dtype=torch.int32, device=DEV)
    assert torch.equal(T.tardis_moe_combine(torch.empty(0, 40, device=DEV), none, torch.ones(3, 2, device=DEV), residual=r), r)
    assert T.tardis_moe_combine(torch.randn(4, 40, device=DEV), none[:0], torch.ones(0, 2, device=DEV)).shape == (0, 40)


def experts_layer(x, Wr, W1, b1, W2, k):
    ids, w, offsets, order, place = T.tardis_moe_route(T.tardis_linear(x, Wr, out_dtype=torch.float32), k)
    h = T.tardis_grouped_linear(x, W1, offsets, b1, act="gelu_erf", order=order, per_token=k)
    z = T.tardis_grouped_linear(h, W2, offsets)
    return T.tardis_moe_combine(z, place, w, residual=x), ids, w


def make_layer(gen, n, d, h, experts):
    x = torch.randn(n, d, device=DEV, generator=gen).bfloat16()
    Wr = torch.randn(experts, d, device=DEV, generator=gen).mul_(2.0 / math.sqrt(d)).bfloat16()
    W1 = torch.randn(experts, h, d, device=DEV, generator=gen).mul_(1.0 / math.sqrt(d)).bfloat16()
    W2 = torch.randn(experts, d, h, device=DEV, generator=gen).mul_(1.0 / math.sqrt(h)).bfloat16()
    b1 = torch.randn(experts, h, device=DEV, generator=gen).mul_(0.1).bfloat16()
    return x, Wr, W1, b1, W2


@pytest.mark.parametrize("n", [1, 9, 200])
def test_a_layer_of_experts(n):
    """Against 64 bits with the choice that the router made.  Rounded to bf16 on the way: the hidden activations and the experts' outputs, each by
    2^-8 of itself at most - off by at most 2^-8 (W2 |h| + |z|) for an expert's output."""
    gen = torch.Generator(device=DEV).manual_seed(n)
    d, h, experts, k = 256, 520, 8, 2
    x, Wr, W1, b1, W2 = make_layer(gen, n, d, h, experts)
    y, ids, w = experts_layer(x, Wr, W1, b1, W2, k)
    want, off = x.double(), torch.zeros(n, d, dtype=torch.float64, device=DEV)
    for t in range(n):
        for j in range(k):
            e = int(ids[t, j])
            hid = sigma(torch.mv(W1[e].double(), x[t].double()) + b1[e].double(), "gelu_erf")
            z = torch.mv(W2[e].double(), hid)
            want[t] += w[t, j].double() * z
            off[t] += w[t, j].double() * 2.0 ** -8 * (torch.mv(W2[e].double().abs(), hid.abs()) + z.abs()) * 1.01
    check(y, want, off)


def test_another_stream_and_a_graph():
    """The whole layer captured once; replayed with other tokens in the same place, with eager work in between."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    n, d, h, experts, k = 300, 256, 512, 8, 2
    x, *weights = make_layer(gen, n, d, h, experts)
    tokens = [torch.randn(n, d, device=DEV, generator=gen).bfloat16() for _ in range(4)]
    eager = []
    for t in tokens:
        eager.append(experts_layer(t, *weights, k)[0].clone())
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        on_side = experts_layer(tokens[0], *weights, k)[0]
    side.synchronize()
    assert torch.equal(on_side, eager[0])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = experts_layer(x, *weights, k)[0]
    for t, want in list(zip(tokens, eager)) * 2:
        x.copy_(t)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want)
        assert torch.equal(experts_layer(t, *weights, k)[0], want)


def test_a_stream_that_is_given():
    """Outputs and working memory belong to the stream of the call: while it waits there, other work of the current stream gets none of it."""
    gen = torch.Generator(device=DEV).manual_seed(17)
    x, W = torch.randn(8, 16384, device=DEV, generator=gen).bfloat16(), (torch.randn(256, 16384, device=DEV, generator=gen) * 0.01).bfloat16()
    logits = torch.randn(4096, 64, device=DEV, generator=gen)
    want, routed = T.tardis_linear(x, W), T.tardis_moe_route(logits, 4)
    z = torch.randn(4096 * 4, 64, device=DEV, generator=gen)
    summed = T.tardis_moe_combine(z, routed[4], routed[1])
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        y, r = T.tardis_linear(x, W, stream=stream), T.tardis_moe_route(logits, 4, stream=stream)
        s = T.tardis_moe_combine(z, r[4], r[1], stream=stream)
        others = [torch.full((size,), 255, dtype=torch.uint8, device=DEV) for size in [1 << b for b in range(9, 21)] * 4]
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(s, summed) and all(torch.equal(a, b) for a, b in zip(r, routed))
        assert all((o == 255).all() for o in others)
    assert torch.equal(T.tardis_linear(x, W, stream=0), want)


def test_the_example_runs():
    """examples/expert_layer.py: two bf16 roundings on the way and one at the end, 2^-8 each at most in the norm."""
    import importlib.util
    import os
    at = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "expert_layer.py")
    spec = importlib.util.spec_from_file_location("expert_layer", at)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    assert example.main(tokens=40, width=256, hidden=136, experts=12, chosen=3) < 3 * 2.0 ** -8
