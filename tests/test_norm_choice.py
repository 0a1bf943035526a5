"""How many pieces of a row a thread of the norm has, for outputs in e4m3: what was measured to be the fastest (the library's host code on a runtime without a GPU)."""
import pytest

from host_runtime import hip, host  # noqa: F401  (fixtures)
from paper_2501_10054_amd import tardis as T
from test_low_bits_choice import _launched, norm, X, Y, S


@pytest.mark.parametrize("n,d,pieces", [(8192, 4096, 2), (4096, 8192, 2), (16384, 4096, 2), (16384, 2048, 2), (2048, 4096, 4), (2048, 16384, 4), (1000, 11008, 4), (3, 4096, 1)])
def test_pieces(host, n, d, pieces):  # noqa: F811
    for dtype, name in ((T.BF16, "bf16"), (T.F32, "f32")):
        assert norm(host, n, d, dtype, T.FP8_E4M3) == [f"rms_norm_kernel {name} 2 {pieces}"]
        assert _launched(host, "tardis_fp8_rows", X, n, d, d, dtype, Y, S, None) == [f"rms_norm_kernel {name} 2 {pieces}"]


@pytest.mark.parametrize("n,d", [(8192, 4096), (16384, 1024), (100, 16384)])
def test_outputs_that_are_not_codes(host, n, d):  # noqa: F811
    for out in (T.F32, T.BF16):
        assert norm(host, n, d, T.BF16, out)[0].startswith(f"rms_norm_kernel bf16 {out} ")
        assert norm(host, n, d, T.BF16, out)[0].endswith(" 2" if d > 8192 else " 1")
