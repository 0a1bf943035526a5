"""A layer of a mixture of experts on the library's calls: router logits (linear, 32-bit outputs) -> choice -> the experts' up projection with
its activation -> down projection -> weighted sum onto the residual stream.  The result is compared with the definition, in 64 bits, for some tokens,
then the layer is timed as a decode step (captured in a graph) and as a prompt.

    python examples/expert_layer.py [tokens] [width] [hidden] [experts] [chosen]
"""
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

from paper_2501_10054_amd import tardis as T  # noqa: E402


class ExpertLayer:
    def __init__(self, width, hidden, experts, chosen, seed=0, device="cuda"):
        gen = torch.Generator(device=device).manual_seed(seed)
        draw = lambda *shape, std: torch.randn(*shape, device=device, generator=gen).mul_(std).bfloat16()
        self.chosen = chosen
        self.router = draw(experts, width, std=1.0 / math.sqrt(width))
        self.up, self.up_bias = draw(experts, hidden, width, std=1.0 / math.sqrt(width)), draw(experts, hidden, std=0.1)
        self.down = draw(experts, width, hidden, std=1.0 / math.sqrt(hidden))

    def __call__(self, x):
        """x: tokens x width, bf16 -> (the layer's output, the experts that every token took, their weights)"""
        logits = T.tardis_linear(x, self.router, out_dtype=torch.float32)
        ids, weights, offsets, order, place = T.tardis_moe_route(logits, self.chosen)
        h = T.tardis_grouped_linear(x, self.up, offsets, self.up_bias, act="gelu_erf", order=order, per_token=self.chosen)
        z = T.tardis_grouped_linear(h, self.down, offsets)
        return T.tardis_moe_combine(z, place, weights, residual=x), ids, weights

    def defined(self, x, ids, weights):
        """The same in 64 bits for one token and the experts that it took."""
        y = x.double()
        for e, w in zip(ids.tolist(), weights.double()):
            z = torch.mv(self.up[e].double(), x.double()) + self.up_bias[e].double()
            y = y + w * torch.mv(self.down[e].double(), 0.5 * z * torch.erfc(-z / math.sqrt(2.0)))
        return y


def time_us(call, repeats=20):
    begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    call()
    begin.record()
    for _ in range(repeats):
        call()
    end.record()
    end.synchronize()
    return begin.elapsed_time(end) * 1e3 / repeats


def main(tokens=1024, width=2048, hidden=1408, experts=64, chosen=6):
    layer = ExpertLayer(width, hidden, experts, chosen)
    x = torch.randn(tokens, width, device="cuda").bfloat16()
    y, ids, weights = layer(x)
    worst = 0.0
    for t in sorted({0, tokens // 2, tokens - 1}):
        want = layer.defined(x[t], ids[t], weights[t])
        worst = max(worst, ((y[t].double() - want).norm() / want.norm()).item())
    print(f"{tokens} tokens, {chosen} of {experts} experts, {width} x {hidden}: relative error {worst:.1e}")
    print(f"prompt of {tokens} tokens: {time_us(lambda: layer(x)):.1f} us")
    step = x[:16].contiguous()
    layer(step)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer(step)
    print(f"step of {step.shape[0]} tokens, replayed: {time_us(graph.replay):.1f} us")
    return worst


if __name__ == "__main__":
    assert main(*(int(a) for a in sys.argv[1:])) < 1e-2
