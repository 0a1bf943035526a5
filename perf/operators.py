"""The products of feed-forward networks as a model runs them, as cases that can be timed and compared: a linear layer
with bias, activation and residual, and the four steps of a mixture of expert networks - the router's choice, the
experts' products over ragged groups of tokens (up and down), and the sum that goes back to the tokens.

Weights follow the recipe of ``paper_2501_10054_amd.synth`` (N(0, 0.02^2), 1 % of the input columns scaled by 8 in bf16),
tokens are N(0, 1); all of it is drawn on the GPU from the seed.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_MOST_FLOPS = 2.75e11          # of a bf16 case, the size of the largest listed ones
_MOST_FLOPS_F32 = 3.0e10


def _linear(name, n, n_in, n_out, **more):
    c = {"name": name, "kind": "linear", "n": n, "n_in": n_in, "n_out": n_out, "dtype": "bf16", "out": "bf16",
         "act": "identity", "bias": False, "residual": False, "pitch": 0}
    c.update(more)
    return c


def _grouped(name, n, n_in, n_out, experts, k, **more):
    c = {"name": name, "kind": "grouped", "n": n, "n_in": n_in, "n_out": n_out, "experts": experts, "k": k,
         "dtype": "bf16", "out": "bf16", "act": "identity", "bias": False, "gather": True, "skew": 0.0}
    c.update(more)
    return c


def _route(name, n, experts, k, **more):
    c = {"name": name, "kind": "route", "n": n, "experts": experts, "k": k, "dtype": "f32", "renormalise": True,
         "masked": False}
    c.update(more)
    return c


def _combine(name, n, d, k, **more):
    c = {"name": name, "kind": "combine", "n": n, "d": d, "k": k, "dtype": "bf16", "out": "bf16", "residual": True,
         "dropped": False}
    c.update(more)
    return c


def listed():
    return [
        # decode step of one sequence: the down projection of a 7B-class FFN onto the residual stream
        _linear("linear_token", 1, 16384, 4096, bias=True, residual=True),
        # a router's logits for a decode step of 64 sequences: 32-bit outputs of a narrow layer, where latency counts
        _linear("linear_router", 64, 4096, 64, out="f32"),
        # a short prompt of odd length through the down projection of a layer that is not a power of two
        _linear("linear_rows_333", 333, 11008, 4096, residual=True),
        # the up projection of a prompt
        _linear("linear_prompt", 2048, 4096, 16384, bias=True, act="gelu_erf"),
        # a small 32-bit model whose sizes are not round, rows taken out of a wider buffer
        _linear("linear_f32", 509, 1000, 1500, dtype="f32", out="f32", bias=True, act="gelu_tanh", pitch=24),
        # decode step of 32 sequences over 64 experts
        _route("route_step", 32, 64, 6, dtype="bf16"),
        # a prompt batch over 128 experts, some of them switched off, with padding tokens that choose none
        _route("route_prompt", 16384, 128, 8, masked=True),
        # decode step of 16 sequences: every expert has one or two tokens, or none
        _grouped("grouped_step", 16, 4096, 2048, 16, 2, act="gelu_erf", bias=True),
        # the experts' up projection for a prompt
        _grouped("grouped_prompt_up", 2048, 4096, 8192, 8, 2, act="gelu_erf", bias=True),
        # the experts' down projection where a few experts have most of the tokens
        _grouped("grouped_prompt_down", 1003, 1408, 2048, 64, 4, gather=False, skew=1.0),
        # decode step of 32 sequences: the sum of the experts' outputs onto the residual stream
        _combine("combine_step", 32, 2048, 6),
        # the same for a prompt batch, with tokens that some experts or all of them dropped
        _combine("combine_prompt", 8192, 4096, 8, dropped=True),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(hi, lo))))))

    def width(lo, hi):           # most widths of real layers are round, some are not
        w = log_int(lo, hi)
        step = rng.choice([128, 128, 64, 8, 8, 1])
        return max(lo, w // step * step)

    kind = rng.choice(["linear", "linear", "grouped", "grouped", "route", "combine"])
    act = rng.choice(["identity", "gelu_erf", "gelu_tanh", "relu"])
    bias = rng.random() < 0.5
    if kind in ("linear", "grouped"):
        dtype = rng.choice(["bf16", "bf16", "bf16", "bf16", "f32"])
        out = "f32" if dtype == "f32" or rng.random() < 0.2 else "bf16"
        most = _MOST_FLOPS if dtype == "bf16" else _MOST_FLOPS_F32
    if kind == "linear":
        n_in, n_out = width(64, 16384), width(64, 16384)
        n = log_int(1, min(3000, most / (2.0 * n_in * n_out)))
        c = _linear("", n, n_in, n_out, dtype=dtype, out=out, act=act, bias=bias, residual=rng.random() < 0.5,
                    pitch=rng.choice([0, 0, 8, 64, 3]))
    elif kind == "grouped":
        experts = log_int(2, 64)
        n_in = width(128, 8192)
        n_out = width(128, min(8192, 2.6e8 / (experts * n_in)))
        k = rng.randint(1, min(8, experts))
        n = log_int(1, min(3000, most / (2.0 * n_in * n_out * k)))
        c = _grouped("", n, n_in, n_out, experts, k, dtype=dtype, out=out, act=act, bias=bias,
                     gather=rng.random() < 0.5, skew=rng.choice([0.0, 1.0]))
    elif kind == "route":
        experts = log_int(2, 512)
        c = _route("", log_int(1, 16384 * 128 / max(experts, 128)), experts, rng.randint(1, min(8, experts)),
                   dtype=rng.choice(["f32", "bf16"]), renormalise=rng.random() < 0.5, masked=rng.random() < 0.5)
    else:
        k, d = rng.randint(1, 8), width(64, 4096)
        c = _combine("", log_int(1, 8192), d, k, dtype=rng.choice(["bf16", "bf16", "f32"]),
                     out=rng.choice(["bf16", "f32"]), residual=rng.random() < 0.5, dropped=rng.random() < 0.5)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _normal(gen, *shape, std=1.0):
    return torch.randn(*shape, device=DEV, generator=gen).mul_(std)


def _matrix(gen, n_out, n_in, dtype):
    W = _normal(gen, n_out, n_in, std=0.02)
    if dtype == "bf16":
        W[:, torch.randperm(n_in, device=DEV, generator=gen)[:max(1, n_in // 100)]] *= 8.0
    return W.to(_TORCH[dtype])


def _choice(gen, case):
    """The k experts of every token, n x k: distinct ones, some experts more popular than others with skew."""
    score = _normal(gen, case["n"], case["experts"]) + case["skew"] * _normal(gen, case["experts"])
    return score.topk(case["k"], dim=1).indices


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    state = {"case": case}
    if case["kind"] == "linear":
        n, n_in, n_out, dt = case["n"], case["n_in"], case["n_out"], _TORCH[case["dtype"]]
        state["W"] = _matrix(gen, n_out, n_in, case["dtype"])
        state["x"] = _normal(gen, n, n_in + case["pitch"]).to(dt)[:, :n_in]
        state["b"] = _normal(gen, n_out, std=0.1).to(dt) if case["bias"] else None
        state["r"] = _normal(gen, n, n_out).to(_TORCH[case["out"]]) if case["residual"] else None
    elif case["kind"] == "grouped":
        n, k, E, dt = case["n"], case["k"], case["experts"], _TORCH[case["dtype"]]
        state["W"] = torch.stack([_matrix(gen, case["n_out"], case["n_in"], case["dtype"]) for _ in range(E)])
        state["b"] = _normal(gen, E, case["n_out"], std=0.1).to(dt) if case["bias"] else None
        chosen, slots = torch.sort(_choice(gen, case).reshape(-1), stable=True)
        state["offsets"] = torch.searchsorted(chosen, torch.arange(E + 1, device=DEV)).int()
        # the up projection takes its rows from the tokens, the down projection has them in the experts' order already
        state["order"] = slots.int() if case["gather"] else None
        state["x"] = _normal(gen, n if case["gather"] else n * k, case["n_in"]).to(dt)
        # (the plain form's slices: a program that has only torch knows its groups on the host)
        state["ends"] = state["offsets"].tolist()
    elif case["kind"] == "route":
        n, E = case["n"], case["experts"]
        logits = _normal(gen, n, E, std=2.0).to(_TORCH[case["dtype"]])
        if case["masked"]:
            off = torch.rand(E, device=DEV, generator=gen) < 0.1
            off[0] = False
            logits[:, off] = -math.inf                                   # experts that are switched off
            logits[torch.rand(n, device=DEV, generator=gen) < 0.02] = -math.inf   # padding
        state["logits"] = logits
    else:
        n, k, d = case["n"], case["k"], case["d"]
        place = torch.randperm(n * k, device=DEV, generator=gen).view(n, k).int()
        if case["dropped"]:
            place[torch.rand(n, k, device=DEV, generator=gen) < 0.02] = -1
            place[torch.rand(n, device=DEV, generator=gen) < 0.01] = -1
        w = torch.rand(n, k, device=DEV, generator=gen) + 0.05
        state["weights"] = w / w.sum(1, keepdim=True)
        state["place"] = place
        state["z"] = _normal(gen, n * k, d).to(_TORCH[case["dtype"]])
        state["r"] = _normal(gen, n, d).to(_TORCH[case["out"]]) if case["residual"] else None
    return state


# ------------------------------------------------------------------ one pass
def run(state):
    case = state["case"]
    if own:
        from paper_2501_10054_amd import tardis as T
        if case["kind"] == "linear":
            return T.tardis_linear(state["x"], state["W"], state["b"], act=case["act"], residual=state["r"],
                                   out_dtype=_TORCH[case["out"]])
        if case["kind"] == "grouped":
            return T.tardis_grouped_linear(state["x"], state["W"], state["offsets"], state["b"], act=case["act"],
                                           order=state["order"], per_token=case["k"], out_dtype=_TORCH[case["out"]])
        if case["kind"] == "route":
            return T.tardis_moe_route(state["logits"], case["k"], renormalise=case["renormalise"])
        return T.tardis_moe_combine(state["z"], state["place"], state["weights"], residual=state["r"],
                                    out_dtype=_TORCH[case["out"]])
    return _PLAIN[case["kind"]](case, state)


def _act(z, act):
    if act == "gelu_erf":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    return z.clamp_min(0.0) if act == "relu" else z


def _layer(x, W, b, act):
    z = x.float() @ W.float().t()
    if b is not None:
        z = z + b.float()
    return _act(z, act)


def _plain_linear(case, state):
    y = _layer(state["x"], state["W"], state["b"], case["act"])
    if state["r"] is not None:
        y = y + state["r"].float()
    return y.to(_TORCH[case["out"]])


def _plain_grouped(case, state):
    x, ends = state["x"], state["ends"]
    if state["order"] is not None:
        x = x[(state["order"] // case["k"]).long()]
    y = torch.empty(x.shape[0], case["n_out"], dtype=_TORCH[case["out"]], device=x.device)
    # (a product for each expert: every other form multiplies rows by matrices that are not theirs)
    for e in range(case["experts"]):
        if ends[e + 1] > ends[e]:
            rows = slice(ends[e], ends[e + 1])
            b = None if state["b"] is None else state["b"][e]
            y[rows] = _layer(x[rows], state["W"][e], b, case["act"]).to(y.dtype)
    return y


def _plain_route(case, state):
    l, k, E = state["logits"].float(), case["k"], case["experts"]
    l = torch.where(torch.isnan(l), -math.inf, l)
    top, ids = torch.sort(l, dim=1, descending=True, stable=True)
    most, top, ids = top[:, :1], top[:, :k], ids[:, :k]
    there = top > -math.inf
    p = torch.where(there, torch.where(top == most, 1.0, torch.exp(top - most)), 0.0)
    if case["renormalise"]:
        total = p.sum(1, keepdim=True)
    else:
        total = torch.where(l > -math.inf, torch.where(l == most, 1.0, torch.exp(l - most)), 0.0).sum(1, keepdim=True)
    weights = torch.where(there, p / total, 0.0)
    ids = torch.where(there, ids, -1)
    # slots in the order of their experts; those without one behind the last
    key, order = torch.sort(torch.where(ids < 0, E, ids).reshape(-1), stable=True)
    offsets = torch.searchsorted(key, torch.arange(E + 1, device=key.device))
    at = torch.arange(key.numel(), device=key.device)
    place = torch.empty_like(order)
    place[order] = torch.where(key < E, at, -1)
    order = torch.where(key < E, order, -1)
    return ids.int(), weights, offsets.int(), order.int(), place.view(-1, k).int()


def _plain_combine(case, state):
    place = state["place"]
    z = state["z"].float()[place.clamp_min(0).long()]
    y = (torch.where(place >= 0, state["weights"], 0.0)[..., None] * z).sum(1)
    if state["r"] is not None:
        y = y + state["r"].float()
    return y.to(_TORCH[case["out"]])


_PLAIN = {"linear": _plain_linear, "grouped": _plain_grouped, "route": _plain_route, "combine": _plain_combine}


def work(case):
    es = 4 if case.get("dtype") == "f32" else 2
    eo = 4 if case.get("out") == "f32" else 2
    n = case["n"]
    if case["kind"] == "linear":
        K, N = case["n_in"], case["n_out"]
        nbytes = es * (n * K + N * K + (N if case["bias"] else 0)) + eo * n * N * (2 if case["residual"] else 1)
        flops = 2.0 * n * N * K
    elif case["kind"] == "grouped":
        K, N, E, k = case["n_in"], case["n_out"], case["experts"], case["k"]
        hit = E * (1.0 - (1.0 - k / E) ** n)                             # experts that some token chose (without skew)
        nbytes = es * ((n if case["gather"] else n * k) * K + hit * N * (K + (1 if case["bias"] else 0)))
        nbytes += eo * n * k * N + 4 * (E + 1) + (4 * n * k if case["gather"] else 0)
        flops = 2.0 * n * k * N * K
    elif case["kind"] == "route":
        E, k = case["experts"], case["k"]
        nbytes, flops = es * n * E + 16 * n * k + 4 * (E + 1), 4.0 * n * E
    else:
        d, k = case["d"], case["k"]
        nbytes = es * n * k * d + 8 * n * k + eo * n * d * (2 if case["residual"] else 1)
        flops = 2.0 * n * k * d
    return {"bytes": float(nbytes), "flops": float(flops)}


# ------------------------------------------------------------------ the same in 64 bits
def _phi(z):
    return 0.5 * torch.erfc(-z / math.sqrt(2.0))


def _sigma64(z, act):
    if act == "gelu_erf":
        return z * _phi(z)
    if act == "gelu_tanh":
        return z / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    return torch.relu(z) if act == "relu" else z


def _exact_linear(case, s):
    z = torch.mm(s["W"].double(), s["x"].double().t().contiguous()).t()
    if s["b"] is not None:
        z = z + s["b"].double()
    y = _sigma64(z, case["act"])
    return y if s["r"] is None else y + s["r"].double()


def _exact_grouped(case, s):
    E, k = case["experts"], case["k"]
    positions = s["x"].shape[0] if s["order"] is None else s["order"].numel()
    p = torch.arange(positions, device=DEV)
    expert = (p[:, None] >= s["offsets"][None, 1:]).sum(1)                # the group that holds a position
    y = torch.zeros(positions, case["n_out"], dtype=torch.float64, device=DEV)
    for e in range(E):
        mine = p[expert == e]
        if mine.numel() == 0:
            continue
        x = s["x"][mine] if s["order"] is None else s["x"][torch.div(s["order"][mine].long(), k, rounding_mode="floor")]
        z = torch.mm(s["W"][e].double(), x.double().t().contiguous()).t()
        if s["b"] is not None:
            z = z + s["b"][e].double()
        y[mine] = _sigma64(z, case["act"])
    return y


def _exact_route(case, s):
    l, k, E = s["logits"].double().cpu().numpy(), case["k"], case["experts"]
    n = l.shape[0]
    usable = l > -np.inf
    rank = np.argsort(np.where(usable, -l, np.inf), axis=1, kind="stable")[:, :k]
    taken = np.take_along_axis(usable, rank, 1)
    ids = np.where(taken, rank, -1)
    with np.errstate(invalid="ignore"):
        shifted = np.where(usable, l - np.where(usable, l, -np.inf).max(1, keepdims=True), -np.inf)
    p = np.exp(shifted)
    chosen = np.where(taken, np.take_along_axis(p, rank, 1), 0.0)
    total = (chosen if case["renormalise"] else p).sum(1, keepdims=True)
    weights = chosen / np.where(total > 0.0, total, 1.0)
    flat = ids.reshape(-1)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[flat >= 0], minlength=E))])
    order, place = np.full(n * k, -1), np.full(n * k, -1)
    slots = np.flatnonzero(flat >= 0)
    slots = slots[np.argsort(flat[slots], kind="stable")]
    order[:slots.size] = slots
    place[slots] = np.arange(slots.size)
    whole = [a.astype(np.int32) for a in (ids, offsets, order, place.reshape(n, k))]
    return whole[0], weights, whole[1], whole[2], whole[3]


def _exact_combine(case, s):
    y = torch.zeros(case["n"], case["d"], dtype=torch.float64, device=DEV) if s["r"] is None else s["r"].double()
    for j in range(case["k"]):
        has = torch.nonzero(s["place"][:, j] >= 0).flatten()
        y.index_add_(0, has, s["weights"][has, j, None].double() * s["z"][s["place"][has, j].long()].double())
    return y


_EXACT = {"linear": _exact_linear, "grouped": _exact_grouped, "route": _exact_route, "combine": _exact_combine}


def exact(case, seed):
    return _EXACT[case["kind"]](case, prepare(case, seed))
