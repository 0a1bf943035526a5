"""The calls of low_bits_paths.py take the ways that they are there for: the library's host code on a runtime without a GPU."""
import pytest

from host_runtime import hip, host  # noqa: F401  (fixtures)
from low_bits_paths import FEW_TOKENS, LARGE_TILES
from paper_2501_10054_amd import tardis as T
from test_low_bits_choice import eight, four

LDS, WAVES, RING = 160 * 1024, 8, 8 * 8 * 1024        # of a CU; wavefronts of a block; their rings


@pytest.mark.parametrize("n,n_in,n_out,dtype,rows,chunks", FEW_TOKENS)
def test_few_tokens(host, n, n_in, n_out, dtype, rows, chunks):  # noqa: F811
    parts, entry = (1, 4) if dtype == T.BF16 else (3, 8)
    steps, sharing = -(-n_in // 128), WAVES // rows
    for group, want in zip((32, 64, 128), chunks):
        name = f"linear4_kernel {'bf16' if dtype == T.BF16 else 'f32'} {group // 32} {rows}"
        assert four(host, n, n_in, n_out, group, dtype) == [name]
        # steps whose tokens and table are in LDS together, in whole turns of the wavefronts that share a row tile
        fit = (LDS - RING - 16 * n * parts) // (256 * n * parts + 128 // group * 16 * rows * entry)
        chunk = min(steps, fit // sharing * sharing if fit >= sharing else fit)
        assert -(-steps // chunk) == want, (group, chunk)


@pytest.mark.parametrize("n,n_in,n_out,launches", LARGE_TILES)
def test_large_tiles(host, n, n_in, n_out, launches):  # noqa: F811
    got = eight(host, n, n_in, n_out, 0, T.BF16)
    assert len(got) == launches and "linear_fp8_quad_kernel 8 4" in got, got
