"""How large a call of linear layers and experts may be, on the CPU: the library's host code on a runtime without a GPU."""
import ctypes as C
import random

import pytest

from host_runtime import hip, host  # noqa: F401  (fixtures)
from paper_2501_10054_amd import tardis as T
from test_linear_choice import OFFSETS, ORDER, W, WORK, X, Y, launched


def grouped(host, dtype, tokens, n_in, n_out, experts, k):  # noqa: F811
    """Status of the call and of the question for its working memory"""
    desc, lib = T.tardis_linear_desc(n_in, n_out, dtype, T.BF16, T.ACT["relu"], 0, W, None), host.lib
    lib.tardis_grouped_linear.argtypes = T.lib().tardis_grouped_linear.argtypes
    lib.tardis_grouped_linear_workspace.argtypes = T.lib().tardis_grouped_linear_workspace.argtypes
    asked = lib.tardis_grouped_linear_workspace(desc, experts, X, tokens, n_in, 1, tokens * k, C.c_int64())
    return lib.tardis_grouped_linear(desc, experts, X, tokens, n_in, OFFSETS, ORDER, k, tokens * k, Y, WORK, 1 << 40, None), asked


@pytest.mark.parametrize("dtype,tokens,n_in,n_out,experts", [(T.BF16, 65536, 8, 2048, 65536), (T.BF16, 4096, 8, 32768, 4096), (T.BF16, 16384, 8, 8192, 16384),
                                                             (T.BF16, 1 << 20, 8, 16384, 4096), (T.F32, 65536, 8, 2048, 65536)])
def test_groups_take_a_tile_that_a_launch_has_room_for(host, dtype, tokens, n_in, n_out, experts):  # noqa: F811
    """Many experts with few tokens each: the tile that would be fastest needs more blocks than a launch has, larger ones do not."""
    assert grouped(host, dtype, tokens, n_in, n_out, experts, 1) == (T.OK, T.OK)


def test_what_no_tile_has_room_for_is_refused_alike(host):  # noqa: F811
    """A launch has less than 2^21 tiles, of 256 columns and at least one for every expert with a token: the call and the question for
    its working memory give the same answer."""
    assert grouped(host, T.BF16, 65536, 8, 1 << 14, 65536, 1) == (T.ERR_SHAPE, T.ERR_SHAPE)
    lib = host.lib
    lib.tardis_linear_workspace.argtypes = T.lib().tardis_linear_workspace.argtypes
    big = T.tardis_linear_desc(64, 1 << 22, T.BF16, T.BF16, 0, 0, W, None)
    assert lib.tardis_linear_workspace(big, X, 1 << 30, 64, C.c_int64()) == T.ERR_SHAPE


def test_no_call_that_a_tile_fits_is_refused(host):  # noqa: F811
    rng = random.Random(5)
    tried = 0
    while tried < 3000:
        experts, tokens, n_in, n_out = (int(2 ** rng.uniform(*r)) for r in ((0, 16), (0, 20), (0, 13), (4, 17)))
        k, dtype = rng.randint(1, 4), rng.choice([T.BF16, T.F32])
        columns = 256 if dtype == T.BF16 else 128            # of the widest tiles for rows of any length, their rows: 192 and 128 or less
        tall = 192 if dtype == T.BF16 else 128
        positions = tokens * k
        tiles = min(positions, positions // tall + experts + 1) * -(-n_out // columns)
        if dtype == T.BF16 and (n_in * 2) % 16 and n_in * n_out * experts > 1 << 33:
            continue                                         # (rows that are copied first: not where the copy is larger than 16 GB)
        if tiles >= 1 << 21 or experts * n_out * n_in > 6 << 33 or positions * n_out > 6 << 33:
            continue
        tried += 1
        assert grouped(host, dtype, tokens, n_in, n_out, experts, k) == (T.OK, T.OK), (dtype, tokens, n_in, n_out, experts, k)


def test_no_launch_has_2_to_the_32_threads(hip):  # noqa: F811
    """Rows of an odd length that are copied first, and sums of experts, over more than 2^32 pieces of 16 bytes (64 GB: a card has 288)."""
    assert launched(hip, T.BF16, 4194309, 8191, 2048, 0, 0, 1) == ["linear_pack_kernel"] * 4 + ["linear_quad_kernel 0 8 8"]
    assert launched(hip, T.BF16, 4000000, 8191, 2048, 0, 0, 1) == ["linear_pack_kernel"] * 3 + ["linear_quad_kernel 0 8 8"]
    assert launched(hip, T.BF16, 2048, 4001, 8192, 0, 0, 1)[:2] == ["linear_pack_kernel"] * 2
    lib = hip.lib
    lib.tardis_moe_combine.argtypes = T.lib().tardis_moe_combine.argtypes
    for n, d, dtype, out, launches in ((1 << 21, 16384, T.BF16, T.BF16, 2), ((1 << 21) + 1, 16384, T.BF16, T.F32, 3), (1 << 20, 16384, T.F32, T.BF16, 2),
                                       ((1 << 20) - 1, 16384, T.BF16, T.BF16, 1), (8192, 4096, T.BF16, T.BF16, 1), (5000, 1 << 22, T.F32, T.F32, 3)):
        hip.launches()
        assert lib.tardis_moe_combine(X, 100, ORDER, OFFSETS, n, 4, d, dtype, None, Y, out, None) == T.OK
        assert len(hip.launches()) == launches
    assert lib.fake_refused() == 0


@pytest.mark.parametrize("gap", [1 << 22, 1 << 30, (1 << 40) + 3])
def test_one_row_has_no_distance_to_the_next(hip, gap):  # noqa: F811
    """The last token of a long prompt is a row of a tensor whose rows are a prompt apart: the distance says nothing, nor refuses or slows the call."""
    for experts in (0, 4):
        for n_in in (4096, 4097):
            assert launched(hip, T.BF16, 1, n_in, 4096, gap, experts, 2) == launched(hip, T.BF16, 1, n_in, 4096, 0, experts, 2)
    lib = hip.lib
    lib.tardis_linear_workspace.argtypes = T.lib().tardis_linear_workspace.argtypes
    need = []
    for pitch in (8191, 8191 + gap):
        need.append(C.c_int64())
        assert lib.tardis_linear_workspace(T.tardis_linear_desc(8191, 64, T.BF16, T.BF16, 0, 0, W, None), X, 1, pitch, need[-1]) == T.OK
    assert need[0].value == need[1].value


def test_the_router_s_question_and_call_have_the_same_limits():
    """2^30 slots at most."""
    from test_linear_host import route
    lib, P = T.lib(), C.c_void_p(0x4000)
    for n, k, status in ((1 << 30, 2, T.ERR_SHAPE), ((1 << 26) + 1, 16, T.ERR_SHAPE), ((1 << 30) + 1, 1, T.ERR_SHAPE)):
        need = C.c_int64(5)
        assert lib.tardis_moe_route_workspace(n, 64, k, need) == status
        assert route(n=n, experts=64, k=k, work=P, bytes_=1 << 40) == status
    need = C.c_int64()
    assert lib.tardis_moe_route_workspace(1 << 26, 64, 16, need) == T.OK and need.value > 0
