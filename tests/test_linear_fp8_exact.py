"""Layers on e4m3 codes with outputs in bf16 whose sums are asked to be exact: which kernels they take, on the CPU (the library's host code on a runtime without a
GPU), and what is refused."""
import ctypes as C
import random

import pytest

from host_runtime import hip, host  # noqa: F401  (fixtures)
from paper_2501_10054_amd import tardis as T
from test_low_bits_choice import S, W, WORK, X, Y, _launched

SIZES = [(1, 16384, 4096), (16, 4096, 11008), (40, 8192, 4096), (64, 4096, 11008), (333, 11008, 4096), (700, 2048, 8192), (2048, 4096, 16384), (2048, 4001, 8192), (9866, 16, 271)]


def launched(host, n, n_in, n_out, gap, out, act, room=1 << 40):  # noqa: F811
    desc = T.tardis_linear_fp8_desc(n_in, n_out, out, act, W, S, None)
    return [name for name in _launched(host, "tardis_linear_fp8", desc, X, S, n, n_in + gap, None, Y, WORK if room else None, room, None) if name]


@pytest.mark.parametrize("act", range(4))
def test_no_kernel_of_the_faster_instruction(host, act):  # noqa: F811
    rng = random.Random(act)
    drawn = [(rng.randint(1, 3000), rng.randint(1, 12000), rng.randint(1, 12000)) for _ in range(40)]
    near = 0
    for n, n_in, n_out in SIZES + drawn:
        for gap in (0, 16, 3):
            for room in (1 << 40, 0):
                got = launched(host, n, n_in, n_out, gap, T.BF16, act | T.FP8_EXACT, room)
                assert got and all(name.startswith("linear_fp8_kernel exact") for name in got), (n, n_in, n_out, gap, got)
                # by the sizes alone, as outputs in fp32 in which nothing else is possible
                assert launched(host, n, n_in, n_out, gap, T.F32, act | T.FP8_EXACT, room) == launched(host, n, n_in, n_out, gap, T.F32, act, room)
                near += any("near" in name or "quad" in name for name in launched(host, n, n_in, n_out, gap, T.BF16, act, room))
    assert near > 20


def test_plans_of_both_are_kept_apart(host):  # noqa: F811
    """One call after the other, in turn: the plan of the first is not the second's."""
    for _ in range(3):
        assert launched(host, 2048, 4096, 16384, 0, T.BF16, 0)[0].startswith("linear_fp8_quad_kernel")
        assert launched(host, 2048, 4096, 16384, 0, T.BF16, T.FP8_EXACT)[0].startswith("linear_fp8_kernel exact")


def test_working_memory_is_that_of_the_call(host):  # noqa: F811
    """The question knows what the call is asked for: with what it says nothing is left out."""
    lib = host.lib
    lib.tardis_linear_fp8_workspace.argtypes = T.lib().tardis_linear_fp8_workspace.argtypes
    for n, n_in, n_out in SIZES:
        for gap in (0, 3):
            for act in (3, 3 | T.FP8_EXACT):
                need = C.c_int64()
                desc = T.tardis_linear_fp8_desc(n_in, n_out, T.BF16, act, W, S, None)
                assert lib.tardis_linear_fp8_workspace(desc, X, n, n_in + gap, need) == T.OK
                assert launched(host, n, n_in, n_out, gap, T.BF16, act, need.value) == launched(host, n, n_in, n_out, gap, T.BF16, act)


def test_what_is_refused():
    P = C.c_void_p(0x4000)

    def eight(act):
        return T.lib().tardis_linear_fp8(T.tardis_linear_fp8_desc(64, 256, T.BF16, act, 0x1000, None, None), P, None, 0, 64, None, P, None, 0, None)

    assert all(eight(act) == eight(act | T.FP8_EXACT) == T.OK for act in range(4))
    for act in (4, 4 | T.FP8_EXACT, -1, 0x200, 0x300, 1 << 30):
        assert eight(act) == T.ERR_INVALID_ARG, act
    # (it belongs to codes)
    assert T.lib().tardis_linear_4bit(T.tardis_linear_4bit_desc(64, 256, T.BF16, T.BF16, T.FP8_EXACT, 32, 0x1000, 0x2000, None, None), P, 0, 64, None, P, None, 0,
                                      None) == T.ERR_INVALID_ARG
    assert T.lib().tardis_linear(T.tardis_linear_desc(64, 256, T.BF16, T.BF16, T.FP8_EXACT, 0, 0x1000, None), P, 0, 64, None, P, None, 0, None) == T.ERR_INVALID_ARG
