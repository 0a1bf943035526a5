"""Which kernels the norm and the layers in 8 and 4 bits take, on the CPU: the library's host code on a runtime without a GPU.  Every kernel has a call, which
the GPU's tests make."""
import ctypes as C
import re
import subprocess

import pytest

from host_runtime import hip, host  # noqa: F401  (fixtures)
from low_bits_calls import EIGHT, FOUR, NORM
from paper_2501_10054_amd import tardis as T

# (addresses that nothing reads: nothing runs)
X, W, Y, WORK, S = (C.c_void_p(1 << s) for s in (39, 38, 40, 41, 37))
KERNEL = re.compile(r"(linear_fp8_quad_kernel|linear_fp8_kernel|linear4_\w+?_kernel|linear4_kernel|rms_norm_kernel)I(.*?)EEv")
TYPES = {"f": "f32 ", "t": "bf16 ", "6e4m3_t": "exact ", "11e4m3_near_t": "near "}


def _short(symbol):
    m = KERNEL.search(symbol)
    if not m:
        return None
    kind = re.match(r"11e4m3_near_t|6e4m3_t|[ft](?=L)", m[2])
    return m[1] + " " + (TYPES[kind[0]] if kind else "") + " ".join(re.findall(r"L[bi](\d+)", m[2]))


def _launched(host, name, *args):  # noqa: F811
    call = getattr(host.lib, name)
    call.argtypes = getattr(T.lib(), name).argtypes
    host.launches()                                   # (forgets those before)
    assert call(*args) == T.OK
    return [_short(s) for s in host.launches()]


def eight(host, n, n_in, n_out, gap, out, room=1 << 40):  # noqa: F811
    desc = T.tardis_linear_fp8_desc(n_in, n_out, out, T.ACT["relu"], W, S, None)
    return _launched(host, "tardis_linear_fp8", desc, X, S, n, n_in + gap, None, Y, WORK if room else None, room, None)


def four(host, n, n_in, n_out, group, dtype, room=1 << 40):  # noqa: F811
    desc = T.tardis_linear_4bit_desc(n_in, n_out, dtype, T.BF16, T.ACT["relu"], group, W, S, None, None)
    return _launched(host, "tardis_linear_4bit", desc, X, n, n_in, None, Y, WORK if room else None, room, None)


def norm(host, n, d, dtype, out):  # noqa: F811
    return _launched(host, "tardis_rms_norm", T.tardis_norm_desc(d, dtype, out, 1e-5, 0, None), X, n, d, None, None, Y, S if out == T.FP8_E4M3 else None, None)


@pytest.mark.parametrize("name,calls", [("eight", EIGHT), ("four", FOUR), ("norm", NORM)])
def test_the_kernel_of_a_call(host, name, calls):  # noqa: F811
    for kernel, *sizes in calls:
        got = globals()[name](host, *sizes)
        assert kernel in got, (kernel, sizes, got)


def test_every_kernel_has_a_call(host):  # noqa: F811
    names = subprocess.run(["nm", host.lib._name], check=True, capture_output=True, text=True).stdout
    there = {_short(s) for s in re.findall(r"\S*__device_stub__\S+", names)} - {None}
    assert there == {c[0] for c in EIGHT + FOUR + NORM}


def test_working_memory_is_what_the_caller_gives(host):  # noqa: F811
    """Without it, many tokens with 4-bit weights go 16 at a time, and codes of odd rows are not copied."""
    assert four(host, 100, 4096, 4096, 128, T.BF16, room=0) == ["linear4_kernel bf16 4 1"] * 7
    assert len(eight(host, 2048, 4001, 8192, 0, T.BF16, room=0)) == 1
    lib = host.lib
    lib.tardis_linear_4bit_workspace.argtypes = T.lib().tardis_linear_4bit_workspace.argtypes
    need = C.c_int64()
    desc = T.tardis_linear_4bit_desc(4096, 4096, T.BF16, T.BF16, 0, 128, W, S, None, None)
    assert lib.tardis_linear_4bit_workspace(desc, 1, 4096, need) == T.OK and need.value == 0
    assert lib.tardis_linear_4bit_workspace(desc, 100, 4096, need) == T.OK and need.value > 0
    assert four(host, 100, 4096, 4096, 128, T.BF16, room=need.value)[0] == "linear4_prepare_kernel bf16 4"


@pytest.mark.parametrize("n,n_in,n_out", [(1, 1 << 22, 1 << 15), (1 << 28, 64, 1), (1 << 22, 4096, 1 << 10), (16, 1 << 22, 16), (1 << 12, 1, 1 << 22), (5, 128, 1 << 22)])
def test_large_calls_with_4_bit_weights(host, n, n_in, n_out):  # noqa: F811
    """Nothing that the limits allow is refused, and no launch has 2^32 threads (the runtime's double counts them)."""
    for dtype in (T.BF16, T.F32):
        got = four(host, min(n, (1 << 36) // n_out), n_in, n_out, 128, dtype)
        assert 1 <= len(got) <= 1 << 17


@pytest.mark.parametrize("n,d", [(1 << 30, 1), (1 << 26, 2048), (3, 1 << 22)])
def test_large_norms(host, n, d):  # noqa: F811
    for out in (T.BF16, T.FP8_E4M3):
        assert norm(host, n, d, T.BF16, out)
