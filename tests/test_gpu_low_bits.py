"""A feed-forward block in 8 and in 4 bits as a model runs it: norm with the residual, up projection, down projection onto the residual - step by step against
the steps' definitions in 64 bits (each step's tolerance: its own test), on one stream, on several, and in a graph that is replayed."""
import pytest
import torch

import test_gpu_linear_4bit as four
import test_gpu_linear_fp8 as eight
import test_gpu_norm as norm
from paper_2501_10054_amd import tardis as T
from test_gpu_linear import check

pytestmark = pytest.mark.gpu
DEV = "cuda"


class Block:
    def __init__(self, d, h, seed, group=64):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.gen, self.group = gen, group
        self.weight = (1.0 + 0.1 * torch.randn(d, device=DEV, generator=gen)).bfloat16()
        W1, W2 = torch.randn(h, d, device=DEV, generator=gen) * 0.05, torch.randn(d, h, device=DEV, generator=gen) * 0.05
        self.b1 = torch.randn(h, device=DEV, generator=gen).bfloat16()
        self.up8, self.down8 = T.tardis_fp8_rows(W1), T.tardis_fp8_rows(W2)
        self.up4, self.down4 = (four.weights(*W.shape, group, torch.bfloat16, gen, True) for W in (W1, W2))
        self.packed4 = [T.tardis_pack_4bit(w[0], group) for w in (self.up4, self.down4)]

    def eight(self, x, residual):
        """-> all that the steps give"""
        a, sa, total = T.tardis_rms_norm(x, self.weight, residual=residual, out_dtype=T.FP8)
        h = T.tardis_linear_fp8(a, sa, *self.up8, self.b1, act="gelu_erf")
        c, sc = T.tardis_fp8_rows(h)
        return a, sa, total, h, c, sc, T.tardis_linear_fp8(c, sc, *self.down8, residual=total)

    def four(self, x, residual):
        a, total = T.tardis_rms_norm(x, self.weight, residual=residual)
        h = T.tardis_linear_4bit(a, self.packed4[0], *self.up4[1:], self.b1, group=self.group, act="gelu_tanh")
        return a, total, h, T.tardis_linear_4bit(h, self.packed4[1], *self.down4[1:], group=self.group, residual=total)

    def check_eight(self, outs, x, residual):
        a, sa, total, h, c, sc, y = outs
        norm.check_norm((a, sa, total), x, self.weight, residual, 1e-6, T.FP8)
        check(h, *eight.layer64(a, sa, *self.up8, self.b1, "gelu_erf"))
        norm.check_codes(c, sc, h.double())
        want, off = eight.layer64(c, sc, *self.down8, None, "identity")
        check(y, want + total.double(), off)

    def check_four(self, outs, x, residual):
        a, total, h, y = outs
        norm.check_norm((a, total), x, self.weight, residual, 1e-6, torch.bfloat16)
        check(h, *four.layer64(a, *self.up4, self.b1, "gelu_tanh", self.group))
        want, off = four.layer64(h, *self.down4, None, "identity", self.group)
        check(y, want + total.double(), off)

    def tokens(self, n):
        return [torch.randn(n, self.weight.numel(), device=DEV, generator=self.gen).bfloat16() for _ in range(2)]


@pytest.mark.parametrize("n,d,h", [(1, 1024, 4096), (7, 520, 1416), (64, 1024, 2048), (300, 512, 2048)])
def test_block(n, d, h):
    block = Block(d, h, n)
    x, r = block.tokens(n)
    block.check_eight(block.eight(x, r), x, r)
    block.check_four(block.four(x, r), x, r)


def test_two_graphs_and_eager_calls():
    """Two graphs captured one after the other, replayed with eager calls between them, new tokens each time."""
    block = Block(2048, 8192, 3)
    kept = []
    for n in (1, 40):
        x, r = block.tokens(n)
        block.eight(x, r), block.four(x, r)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = block.eight(x, r), block.four(x, r)
        kept.append((graph, x, r, outs))
    for turn in range(3):
        for graph, x, r, (outs8, outs4) in kept:
            for t, fresh in zip((x, r), block.tokens(x.shape[0])):
                t.copy_(fresh)
            graph.replay()
            want8, want4 = block.eight(x, r), block.four(x, r)
            torch.cuda.synchronize()
            assert all(torch.equal(a.float(), b.float()) for a, b in zip(outs8 + outs4, want8 + want4)), turn


def test_streams_side_by_side():
    """Two streams at once, each with its own tokens."""
    block = Block(1024, 8192, 4)
    tokens = [block.tokens(n) for n in (5, 130)]
    want = [(block.eight(x, r), block.four(x, r)) for x, r in tokens]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in tokens]
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append((block.eight(*tokens[i]), block.four(*tokens[i])))
    torch.cuda.synchronize()
    for i in range(2):
        for outs8, outs4 in got[i]:
            assert all(torch.equal(a.float(), b.float()) for a, b in zip(outs8 + outs4, want[i][0] + want[i][1]))
