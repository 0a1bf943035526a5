"""Which kernel a call of the linear layer takes, on the CPU: the library's host code on a runtime without a GPU.  Every kernel has a call."""
import ctypes as C
import re
import subprocess

import pytest

from host_runtime import hip, host  # noqa: F401  (fixtures)
from linear_calls import CALLS
from paper_2501_10054_amd import tardis as T

# (addresses that nothing reads: nothing runs)
X, W, Y, ORDER, OFFSETS, WORK = (C.c_void_p(1 << s) for s in (39, 38, 40, 43, 42, 41))


def _short(symbol):
    m = re.search(r"(linear_\w+?_kernel|linear_kernel)I(.*?)EEv", symbol)
    return None if m is None else (m[1] + " " + " ".join(re.findall(r"L[bi](\d+)", m[2]))).strip(), "F32" if m and m[2].startswith("f") else "BF16"


def launched(host, dtype, n, n_in, n_out, gap, experts, k, room=1 << 40):
    desc = T.tardis_linear_desc(n_in, n_out, dtype, T.BF16, T.ACT["relu"], 0, W, None)
    lib = host.lib
    lib.tardis_linear.argtypes, lib.tardis_grouped_linear.argtypes = T.lib().tardis_linear.argtypes, T.lib().tardis_grouped_linear.argtypes
    host.launches()                                   # (forgets those before)
    work = WORK if room else None
    if experts:
        st = lib.tardis_grouped_linear(desc, experts, X, n, n_in + gap, OFFSETS, ORDER, k, n * k, Y, work, room, None)
    else:
        st = lib.tardis_linear(desc, X, n, n_in + gap, None, Y, work, room, None)
    assert st == T.OK
    return [_short(s)[0] for s in host.launches()]


@pytest.mark.parametrize("call", range(len(CALLS)))
def test_the_kernel_of_a_call(host, call):  # noqa: F811
    kernel, *sizes = CALLS[call]
    assert kernel in launched(host, *sizes)


def test_every_kernel_has_a_call(host):  # noqa: F811
    names = subprocess.run(["nm", host.lib._name], check=True, capture_output=True, text=True).stdout
    there = {_short(s) for s in re.findall(r"\S*__device_stub__\S+", names)}
    there = {s for s in there if s[0] and re.match("linear(_quad)?_kernel ", s[0])}
    have = {(c[0], "F32" if c[1] == T.F32 and "quad" not in c[0] else "BF16") for c in CALLS}
    assert have == there


def test_ranges_and_copies_take_what_the_caller_gives(host):  # noqa: F811
    """A token's long rows are divided in ranges, rows of an odd length copied where many rows read them; without working memory neither."""
    assert launched(host, T.BF16, 8, 16384, 256, 0, 0, 1)[1:] == ["linear_join_kernel"]
    assert len(launched(host, T.BF16, 8, 16384, 256, 0, 0, 1, room=0)) == 1
    copies = launched(host, T.BF16, 2048, 4001, 8192, 0, 0, 1)
    assert copies[:2] == ["linear_pack_kernel"] * 2 and len(copies) == 3
    assert len(launched(host, T.BF16, 2048, 4001, 8192, 0, 0, 1, room=0)) == 1
