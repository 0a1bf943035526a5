"""Feed-forward layers in 8 and 4 bits as a model runs them, as cases that can be timed and compared: the root-mean-square
norm in front of a layer with the residual's addition (output in bf16, fp32 or e4m3 with a scale for each row), rows put into e4m3 without a
norm, a linear layer whose tokens and weights are in e4m3, and a linear layer with 4-bit weights in groups.

Weights follow the recipe of ``paper_2501_10054_amd.synth`` (N(0, 0.02^2), 1 % of the input columns scaled by 8), tokens are N(0, 1)
with 1 % of the columns scaled by 8, as residual streams have them; all of it is drawn on the GPU from the seed.
"""
import math

import torch

own = False

DEV = "cuda"
_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
_MOST_FLOPS = 2.75e11          # of a drawn case, the size of the largest listed one
_MOST_ELEMENTS = 3.4e7         # of a drawn norm
_LEAST_SCALE = 2.0 ** -126
_E4M3_MOST = 448.0


def _norm(name, n, d, **more):
    c = {"name": name, "kind": "norm", "n": n, "d": d, "dtype": "bf16", "out": "bf16", "weight": True, "residual": True,
         "eps": 1e-5, "pitch": 0}
    c.update(more)
    return c


def _rows(name, n, d, **more):
    c = {"name": name, "kind": "rows", "n": n, "d": d, "dtype": "bf16", "pitch": 0, "padding": False}
    c.update(more)
    return c


def _linear8(name, n, n_in, n_out, **more):
    c = {"name": name, "kind": "linear8", "n": n, "n_in": n_in, "n_out": n_out, "out": "bf16", "act": "identity",
         "bias": False, "residual": False, "pitch": 0}
    c.update(more)
    return c


def _linear4(name, n, n_in, n_out, group, **more):
    c = {"name": name, "kind": "linear4", "n": n, "n_in": n_in, "n_out": n_out, "group": group, "dtype": "bf16",
         "out": "bf16", "act": "identity", "zeros": False, "bias": False, "residual": False, "pitch": 0}
    c.update(more)
    return c


def listed():
    return [
        # decode step of one sequence, in front of a layer in bf16: latency counts
        _norm("norm_token", 1, 4096),
        # decode step of 32 sequences, in front of a layer in e4m3
        _norm("norm_step_e4m3", 32, 4096, out="e4m3"),
        # a prompt batch on its way into a layer in e4m3
        _norm("norm_prompt_e4m3", 8192, 4096, out="e4m3"),
        # a 32-bit model whose width is not round, rows taken out of a wider buffer, nothing added
        _norm("norm_odd_f32", 1021, 5137, dtype="f32", out="f32", residual=False, pitch=3),
        # the activations of one token on their way into a down projection in e4m3
        _rows("rows_token", 1, 16384),
        # the same for a prompt, some rows of it padding
        _rows("rows_prompt", 2048, 16384, padding=True),
        # decode step of one sequence: the down projection of a 7B-class FFN onto the residual stream
        _linear8("linear8_token", 1, 16384, 4096, bias=True, residual=True),
        # a short prompt of odd length through the down projection of a layer that is not a power of two
        _linear8("linear8_rows_333", 333, 11008, 4096, residual=True),
        # the up projection of a prompt
        _linear8("linear8_prompt", 2048, 4096, 16384, bias=True, act="gelu_erf"),
        # decode step of one sequence: the down projection with 4-bit weights
        _linear4("linear4_token", 1, 16384, 4096, 128, bias=True, residual=True),
        # decode step of 13 sequences: the up projection of a layer that is not a power of two, with zero points
        _linear4("linear4_step_13", 13, 4096, 11008, 64, zeros=True, act="gelu_erf"),
        # the up projection of a short prompt
        _linear4("linear4_prompt", 512, 4096, 16384, 128, zeros=True, bias=True, act="gelu_tanh"),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(hi, lo))))))

    def width(lo, hi):           # most widths of real layers are round, some are not
        w = log_int(lo, hi)
        step = rng.choice([128, 128, 64, 8, 8, 1])
        return max(lo, w // step * step)

    kind = rng.choice(["norm", "norm", "rows", "linear8", "linear8", "linear4", "linear4", "linear4"])
    act = rng.choice(["identity", "gelu_erf", "gelu_tanh", "relu"])
    more = {"act": act, "bias": rng.random() < 0.5, "residual": rng.random() < 0.5}
    if kind in ("norm", "rows"):
        d = width(64, 16384)
        n = log_int(1, min(16384, _MOST_ELEMENTS / d))
        dtype, pitch = rng.choice(["bf16", "bf16", "f32"]), rng.choice([0, 0, 8, 3])
        if kind == "rows":
            c = _rows("", n, d, dtype=dtype, pitch=pitch, padding=rng.random() < 0.5)
        else:
            c = _norm("", n, d, dtype=dtype, out=rng.choice(["bf16", "e4m3", "f32"]), weight=rng.random() < 0.8,
                      residual=rng.random() < 0.6, eps=rng.choice([1e-5, 1e-6]), pitch=pitch)
    elif kind == "linear8":
        n_in, n_out = width(64, 16384), width(64, 16384)
        n = log_int(1, min(3000, _MOST_FLOPS / (2.0 * n_in * n_out)))
        c = _linear8("", n, n_in, n_out, out=rng.choice(["bf16", "bf16", "bf16", "f32"]), pitch=rng.choice([0, 0, 16, 64, 3]),
                     **more)
    else:
        n_in, n_out = width(64, 16384), width(64, 16384)
        most = 0.25 * _MOST_FLOPS / (2.0 * n_in * n_out)
        n = rng.choice([1, log_int(1, min(32, most)), log_int(1, min(1000, most))])
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        c = _linear4("", n, n_in, n_out, rng.choice([32, 64, 128, 128]), dtype=dtype,
                     out="f32" if dtype == "f32" else rng.choice(["bf16", "bf16", "f32"]), zeros=rng.random() < 0.5,
                     pitch=rng.choice([0, 0, 8, 3]), **more)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _normal(gen, *shape, std=1.0):
    return torch.randn(*shape, device=DEV, generator=gen).mul_(std)


def _outliers(gen, X):
    """1 % of the columns scaled by 8."""
    n = X.shape[1]
    X[:, torch.randperm(n, device=DEV, generator=gen)[:max(1, n // 100)]] *= 8.0
    return X


def _tokens(gen, case, d):
    return _outliers(gen, _normal(gen, case["n"], d + case["pitch"])).to(_TORCH[case["dtype"]])[:, :d]


def _codes8(X):
    scales = (X.abs().amax(1) / _E4M3_MOST).clamp_min(_LEAST_SCALE)
    return (X / scales[:, None]).to(torch.float8_e4m3fn), scales


def _packed(q):
    """Codes n_out x n_in, 0 to 15 -> eight columns in 32 bits: column c of the eight at bit 4 (c // 2) + 16 (c % 2)."""
    at = torch.tensor([4 * (c // 2) + 16 * (c % 2) for c in range(8)], dtype=torch.int64, device=q.device)
    words = (q.view(q.shape[0], -1, 8).long() << at).sum(2)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).int()


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    state = {"case": case, "r": None, "b": None, "weight": None}
    n = case["n"]
    if case["kind"] in ("norm", "rows"):
        d = case["d"]
        state["x"] = _tokens(gen, case, d)
        if case["kind"] == "rows":
            if case["padding"]:
                state["x"][torch.rand(n, device=DEV, generator=gen) < 0.02] = 0.0
            return state
        if case["weight"]:
            state["weight"] = (1.0 + _normal(gen, d, std=0.1)).to(_TORCH[case["dtype"]])
        if case["residual"]:
            state["r"] = _normal(gen, n, d).to(_TORCH[case["dtype"]])
        return state
    n_in, n_out = case["n_in"], case["n_out"]
    W = _outliers(gen, _normal(gen, n_out, n_in, std=0.02))
    if case["bias"]:
        state["b"] = _normal(gen, n_out, std=0.1).to(_TORCH[case["out"]])
    if case["residual"]:
        state["r"] = _normal(gen, n, n_out).to(_TORCH[case["out"]])
    if case["kind"] == "linear8":
        state["W"], state["sw"] = _codes8(W)
        x, state["sx"] = _codes8(_outliers(gen, _normal(gen, n, n_in + case["pitch"])))
        state["x"] = x[:, :n_in]
        return state
    state["x"] = _tokens(gen, case, n_in)
    group = case["group"]
    groups = (n_in + group - 1) // group
    W = torch.nn.functional.pad(W, (0, groups * group - n_in)).view(n_out, groups, group)
    if case["zeros"]:
        lo, hi = W.amin(2).clamp_max(0.0), W.amax(2).clamp_min(0.0)
        scales = ((hi - lo) / 15.0).clamp_min(1e-8).to(_TORCH[case["dtype"]])
        zeros = (-lo / scales.float()).round().clamp(0, 15)
        state["zeros"] = zeros.to(torch.uint8)
    else:
        scales = (W.abs().amax(2) / 7.5).clamp_min(1e-8).to(_TORCH[case["dtype"]])
        zeros = torch.full_like(scales, 8.0, dtype=torch.float32)
        state["zeros"] = None
    q = ((W / scales.float()[..., None]).round() + zeros[..., None]).clamp(0, 15)
    state["W"], state["scales"] = _packed(q.view(n_out, groups * group)), scales
    return state


# ------------------------------------------------------------------ one pass
def run(state):
    case = state["case"]
    if own:
        from paper_2501_10054_amd import tardis as T
        if case["kind"] == "norm":
            return T.tardis_rms_norm(state["x"], state["weight"], residual=state["r"], eps=case["eps"],
                                     out_dtype=_TORCH[case["out"]])
        if case["kind"] == "rows":
            return T.tardis_fp8_rows(state["x"])
        if case["kind"] == "linear8":
            return T.tardis_linear_fp8(state["x"], state["sx"], state["W"], state["sw"], state["b"], act=case["act"],
                                       residual=state["r"], out_dtype=_TORCH[case["out"]])
        return T.tardis_linear_4bit(state["x"], state["W"], state["scales"], state["zeros"], state["b"],
                                    group=case["group"], act=case["act"], residual=state["r"], out_dtype=_TORCH[case["out"]])
    return _PLAIN[case["kind"]](case, state)


def _act(z, act):
    if act == "gelu_erf":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (z + 0.044715 * z ** 3)))
    return z.clamp_min(0.0) if act == "relu" else z


def _epilogue(case, state, z):
    if state["b"] is not None:
        z = z + state["b"].float()
    y = _act(z, case["act"])
    if state["r"] is not None:
        y = y + state["r"].float()
    return y.to(_TORCH[case["out"]])


def _plain_norm(case, state):
    """y; with an output in e4m3 (y in units of its row's scale, the scales); with a residual the sum behind them."""
    s = state["x"].float()
    if state["r"] is not None:
        s = s + state["r"].float()
    y = s * torch.rsqrt((s * s).mean(1, keepdim=True) + case["eps"])
    if state["weight"] is not None:
        y = y * state["weight"].float()
    outs = _codes8(y) if case["out"] == "e4m3" else (y.to(_TORCH[case["out"]]),)
    if state["r"] is not None:
        outs += (s.to(state["x"].dtype),)
    return outs if len(outs) > 1 else outs[0]


def _plain_rows(case, state):
    return _codes8(state["x"].float())


def _plain_linear8(case, state):
    z = state["x"].float() @ state["W"].float().t() * state["sx"][:, None] * state["sw"]
    return _epilogue(case, state, z)


def _plain_linear4(case, state):
    words, group = state["W"], case["group"]
    at = torch.tensor([4 * (c // 2) + 16 * (c % 2) for c in range(8)], dtype=torch.int32, device=words.device)
    q = ((words[..., None] >> at) & 15).view(words.shape[0], -1, group).float()
    zeros = 8.0 if state["zeros"] is None else state["zeros"].float()[..., None]
    W = ((q - zeros) * state["scales"].float()[..., None]).view(words.shape[0], -1)[:, :case["n_in"]]
    return _epilogue(case, state, state["x"].float() @ W.t())


_PLAIN = {"norm": _plain_norm, "rows": _plain_rows, "linear8": _plain_linear8, "linear4": _plain_linear4}


def work(case):
    size = {"f32": 4, "bf16": 2, "e4m3": 1}
    n = case["n"]
    if case["kind"] in ("norm", "rows"):
        d, es = case["d"], size[case["dtype"]]
        if case["kind"] == "rows":
            return {"bytes": float(n * d * (es + 1) + 4 * n), "flops": 3.0 * n * d}
        nbytes = n * d * (es * (3 if case["residual"] else 1) + size[case["out"]]) + (es * d if case["weight"] else 0)
        return {"bytes": float(nbytes + (4 * n if case["out"] == "e4m3" else 0)), "flops": 5.0 * n * d}
    K, N, eo = case["n_in"], case["n_out"], size[case["out"]]
    nbytes = eo * (n * N * (2 if case["residual"] else 1) + (N if case["bias"] else 0))
    if case["kind"] == "linear8":
        nbytes += n * K + N * K + 4 * (n + N)
    else:
        es, groups = size[case["dtype"]], (K + case["group"] - 1) // case["group"]
        nbytes += es * n * K + N * groups * (case["group"] // 2 + es + (1 if case["zeros"] else 0))
    return {"bytes": float(nbytes), "flops": 2.0 * n * N * K}


# ------------------------------------------------------------------ the same in 64 bits
def _exact_codes8(y):
    """(y in units of its row's scale, not rounded to e4m3; the scales)"""
    scale = torch.clamp(torch.max(torch.abs(y), dim=1).values / 448, min=2.0 ** -126)
    return y / scale[:, None], scale


def _exact_norm(case, s):
    total = s["x"].double() if s["r"] is None else s["x"].double() + s["r"].double()
    length = torch.linalg.vector_norm(total, dim=1, keepdim=True)
    y = total / torch.sqrt(length * length / case["d"] + case["eps"])
    if s["weight"] is not None:
        y = torch.mul(y, s["weight"].double()[None, :])
    first = _exact_codes8(y) if case["out"] == "e4m3" else (y,)
    if s["r"] is not None:
        return (*first, total)
    return first[0] if len(first) == 1 else first


def _exact_rows(case, s):
    return _exact_codes8(s["x"].double())


def _exact_end(case, s, z):
    if s["b"] is not None:
        z = z + s["b"].double()
    if case["act"] == "gelu_erf":
        z = z * (0.5 * torch.erfc(-z / math.sqrt(2.0)))
    elif case["act"] == "gelu_tanh":
        z = z / (1.0 + torch.exp(-2.0 * math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)))
    elif case["act"] == "relu":
        z = torch.relu(z)
    return z if s["r"] is None else z + s["r"].double()


def _exact_linear8(case, s):
    W = s["W"].double().mul_(s["sw"].double()[:, None])
    x = s["sx"].double()[:, None] * s["x"].double()
    return _exact_end(case, s, torch.mm(W, x.t().contiguous()).t())


def _exact_linear4(case, s):
    N, K, group = case["n_out"], case["n_in"], case["group"]
    words = s["W"].long() & 0xffffffff
    q = torch.empty(N, words.shape[1] * 8, dtype=torch.float64, device=DEV)
    for c in range(8):
        shift = c // 2 * 4 + (16 if c % 2 else 0)
        q[:, c::8] = torch.remainder(torch.div(words, 1 << shift, rounding_mode="floor"), 16).double()
    zeros = torch.full(s["scales"].shape, 8, device=DEV) if s["zeros"] is None else s["zeros"]
    W = (q - torch.repeat_interleave(zeros.double(), group, 1)) * torch.repeat_interleave(s["scales"].double(), group, 1)
    return _exact_end(case, s, torch.mm(W[:, :K], s["x"].double().t().contiguous()).t())


_EXACT = {"norm": _exact_norm, "rows": _exact_rows, "linear8": _exact_linear8, "linear4": _exact_linear4}


def exact(case, seed):
    return _EXACT[case["kind"]](case, prepare(case, seed))
