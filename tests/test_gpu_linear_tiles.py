"""Every kernel of the linear layer, called by its number at sizes on the edges of its tile, against 64 bits (tolerances as in test_gpu_linear)."""
import ctypes as C
import os

import pytest
import torch

from paper_2501_10054_amd import build as B
from paper_2501_10054_amd import tardis as T
from test_gpu_linear import ACTS, check, grouped64, inside, layer64

DEV = "cuda"


def _lib():
    if not os.path.exists(B.LINEAR_PROBE):
        B.build_linear_probe()
    lib = C.CDLL(B.LINEAR_PROBE)
    vp, i64, i = C.c_void_p, C.c_int64, C.c_int
    lib.linear_probe.argtypes = [i, i, i, vp, i64, i64, vp, vp, vp, vp, i64, i64, i64, i, i, i, vp, vp, i, i, vp]
    return lib


def _instances(grouped=0):
    if not os.path.exists(B.LINEAR_PROBE):
        return []
    lib = _lib()
    return [(f32, direct, s) for f32 in (0, 1) for direct in (1, 0) for s in range(lib.linear_probe_shapes(f32, direct)) if lib.linear_probe_has(f32, direct, grouped, s)]


def tile(lib, direct, shape):
    t = (C.c_int * 3)()
    lib.linear_probe_tile(direct, shape, t)
    return list(t)


def ptr(t):
    return None if t is None else t.data_ptr()


def operands(f32, direct, gen, rows, n_in, lead_shape=None):
    """x and its pitch: aligned rows for the kernels that need them, else rows at odd distances"""
    dtype = torch.float32 if f32 else torch.bfloat16
    return inside((rows, n_in), dtype, gen, gap=8 if direct else 3, lead=0 if direct else 1)


@pytest.mark.gpu
@pytest.mark.parametrize("f32,direct,shape", _instances())
def test_edges_of_a_tile(f32, direct, shape):
    lib = _lib()
    m, n, sl = tile(lib, direct, shape)
    es, dtype = (4, torch.float32) if f32 else (2, torch.bfloat16)
    gen = torch.Generator(device=DEV).manual_seed(100 * shape + 10 * f32 + direct)
    step = 16 // es if direct else 1
    per = sl // es
    cases = [(m, n, per), (1, n + 5, 3 * per + step), (m // 2, 2 * n, 2 * per), (m - 1, n - 1, per - step if per > step else step), (m + 1, n + 8, 9 * per),
             (2 * m + m // 4 + 1, n // 2 + 1, 17 * per + 5 * step), (3 * m - 7, 7, step)]
    for number, (rows, n_out, n_in) in enumerate(cases):
        x = operands(f32, direct, gen, rows, n_in)
        W = inside((n_out, n_in), dtype, gen, std=2.0 / n_in ** 0.5, lead=0 if direct else 1)
        b = torch.randn(n_out, device=DEV, generator=gen).to(dtype) if number % 2 else None
        out = torch.float32 if f32 or number % 3 == 0 else torch.bfloat16
        r = torch.randn(rows, n_out, device=DEV, generator=gen).to(out) if number % 2 == 0 else None
        act = ACTS[number % 4]
        y = torch.full((rows + 2, n_out), 3.0, dtype=out, device=DEV)
        st = lib.linear_probe(f32, direct, shape, ptr(x), rows, x.stride(0) * es, ptr(W), ptr(b), ptr(r), y[1:].data_ptr(), rows, n_out, n_in * es, T.ACT[act],
                              int(out == torch.float32), 1, None, None, 0, 1, torch.cuda.current_stream().cuda_stream)
        assert st == T.OK
        want, off = layer64(x, W, b, act)
        check(y[1:-1], want if r is None else want + r.double(), off)
        assert (y[0] == 3.0).all() and (y[-1] == 3.0).all(), (rows, n_out, n_in)     # nothing before, nothing behind


@pytest.mark.gpu
@pytest.mark.parametrize("f32,direct,shape", _instances())
def test_ranges_of_a_row(f32, direct, shape):
    """2, 4 and 8 ranges of K, some of them empty, and with a rest that is no slice: their sums are the product."""
    lib = _lib()
    m, n, sl = tile(lib, direct, shape)
    es, dtype = (4, torch.float32) if f32 else (2, torch.bfloat16)
    gen = torch.Generator(device=DEV).manual_seed(200 * shape + 10 * f32 + direct)
    for ranges, slices in ((2, 5), (4, 9), (8, 3)):
        rows, n_out, n_in = m + 3, n + 9, slices * sl // es + (16 // es)
        x = operands(f32, direct, gen, rows, n_in)
        W = inside((n_out, n_in), dtype, gen, std=2.0 / n_in ** 0.5)
        part = torch.full((ranges, rows, n_out), float("nan"), device=DEV)
        st = lib.linear_probe(f32, direct, shape, ptr(x), rows, x.stride(0) * es, ptr(W), None, None, ptr(part), rows, n_out, n_in * es, T.ACT["identity"], 1, ranges,
                              None, None, 0, 1, torch.cuda.current_stream().cuda_stream)
        assert st == T.OK
        want, off = layer64(x, W, None, "identity")
        check(part.double().sum(0).float(), want, off)


@pytest.mark.gpu
@pytest.mark.parametrize("f32,direct,shape", _instances(grouped=1))
def test_groups(f32, direct, shape):
    """Groups of none, one, some, a tile's and more rows; rows of the tokens by their slots, and as they come."""
    lib = _lib()
    m, n, sl = tile(lib, direct, shape)
    es, dtype = (4, torch.float32) if f32 else (2, torch.bfloat16)
    gen = torch.Generator(device=DEV).manual_seed(300 * shape + 10 * f32 + direct)
    sizes = [0, 1, m, 0, m + 1, m // 4 + 1, m // 2, 2 * m + m // 2 + 3, 0]
    per_token = 3
    rows = (sum(sizes) + per_token - 1) // per_token * per_token
    offsets = torch.tensor([0] + sizes, device=DEV).cumsum(0).int()
    offsets[-1] = rows
    for n_out, n_in, act in ((n + 3, 2 * sl // es + 16 // es, "gelu_erf"), (n // 2, 11 * sl // es, "identity")):
        W = inside((len(sizes), n_out, n_in), dtype, gen, std=2.0 / n_in ** 0.5)
        b = torch.randn(len(sizes), n_out, device=DEV, generator=gen).to(dtype)
        order = torch.randperm(rows, device=DEV, generator=gen).int()
        for x, o in ((operands(f32, direct, gen, rows // per_token, n_in), order), (operands(f32, direct, gen, rows, n_in), None)):
            y = torch.full((rows, n_out), 3.0, device=DEV)
            st = lib.linear_probe(f32, direct, shape, ptr(x), x.shape[0], x.stride(0) * es, ptr(W), ptr(b), None, ptr(y), rows, n_out, n_in * es, T.ACT[act], 1, 1,
                                  ptr(offsets), ptr(o), len(sizes), per_token if o is not None else 1, torch.cuda.current_stream().cuda_stream)
            assert st == T.OK
            check(y, *grouped64(x, W, b, offsets, o, per_token, rows, act))


def test_the_probe_knows_every_kernel():
    """(on the CPU) in bf16 and fp32, for one matrix and for groups: as many as the listing has."""
    if not os.path.exists(B.LINEAR_PROBE):
        pytest.skip("not built")
    count = lambda f32, grouped: sum(i[0] == f32 for i in _instances(grouped))
    assert [count(0, 0), count(0, 1), count(1, 0), count(1, 1)] == [21 + 3, 19 + 3, 13, 10]
