"""The grouped product on large tiles where its tiles have 192 rows and where they have 256, of few groups and of more than the 64 that a wavefront looks at
at a time, against 64 bits (tolerances as in test_gpu_linear)."""
import pytest
import torch

from paper_2501_10054_amd import tardis as T
from test_gpu_linear import check, grouped64, inside
from test_gpu_linear_tiles import _instances, _lib, ptr, tile

DEV = "cuda"
# (about a third of them empty, some with one row, and behind the 64th some that fill a tile of 256 rows)
MANY = [(0, 1, 250)[g % 3] if g < 64 else (250, 256, 0, 200, 193, 1)[g % 6] for g in range(88)] + [700, 0]
# rows of the groups, columns of tiles
GROUPS = {"one": ([8192], 8), "one, a row more": ([8193], 8), "even": ([512] * 8, 32), "nearly even": ([534, 490, 520, 512, 505, 531, 498, 506], 32), "many": (MANY, 1),
          "many, wide": (MANY, 3), "short": ([200, 250, 256, 193, 0, 129, 64], 1), "full": ([200, 250, 256, 193, 0, 129, 64] * 20, 2)}


def rows_of_a_full_tile(sizes, columns, m):
    """As the kernel decides: a round of the 256 CUs with tiles of 192 rows takes 7/8 of one with 256."""
    rounds = lambda rows: -(-sum(-(-s // rows) for s in sizes) * columns // 256)
    return 192 if m == 256 and rounds(192) * 7 < rounds(256) * 8 else m


def large():
    return [(d, s) for f32, d, s in _instances(grouped=1) if not f32 and d and s >= 16]


def test_both_numbers_of_rows_occur():
    """(on the CPU) in few groups and in many, and tiles of 256 rows with more than 192 of them."""
    steps = {name: rows_of_a_full_tile(sizes, columns, 256) for name, (sizes, columns) in GROUPS.items()}
    assert steps == {"one": 256, "one, a row more": 192, "even": 256, "nearly even": 192, "many": 192, "many, wide": 256, "short": 192, "full": 256}
    assert len(large()) == 3


@pytest.mark.gpu
@pytest.mark.parametrize("groups", GROUPS)
@pytest.mark.parametrize("direct,shape", large())
def test_large_tiles(direct, shape, groups):
    lib = _lib()
    m, n, sl = tile(lib, direct, shape)
    sizes, columns = GROUPS[groups]
    rows, n_out, n_in = sum(sizes), columns * n - 5, 2 * sl // 2 + 8
    gen = torch.Generator(device=DEV).manual_seed(shape + rows)
    offsets = torch.tensor([0] + sizes, device=DEV).cumsum(0).int()
    W = inside((len(sizes), n_out, n_in), torch.bfloat16, gen, std=2.0 / n_in ** 0.5)
    b = torch.randn(len(sizes), n_out, device=DEV, generator=gen).bfloat16()
    order = torch.randperm(rows, device=DEV, generator=gen).int()
    for x, o in ((inside((rows, n_in), torch.bfloat16, gen, gap=8), order), (inside((rows, n_in), torch.bfloat16, gen), None)):
        y = torch.full((rows + 1, n_out), 3.0, device=DEV)
        st = lib.linear_probe(0, direct, shape, ptr(x), rows, x.stride(0) * 2, ptr(W), ptr(b), None, ptr(y), rows, n_out, n_in * 2, T.ACT["gelu_erf"], 1, 1,
                              ptr(offsets), ptr(o), len(sizes), 1, torch.cuda.current_stream().cuda_stream)
        assert st == T.OK
        check(y[:-1], *grouped64(x, W, b, offsets, o, 1, rows, "gelu_erf"))
        assert (y[-1] == 3.0).all()
