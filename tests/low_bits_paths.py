"""Calls of the layers in 8 and 4 bits that go through their kernels in other ways than low_bits_calls.py's: with several tokens, more steps than a ring has places,
more columns than LDS has room for; with a rest of K, ranges of K, few rows in a tile, tiles that end inside a row."""
from paper_2501_10054_amd.tardis import BF16, F32

# tokens, n_in, n_out, type of x, row tiles of a block, chunks of K for groups of 32, 64 and 128 columns
FEW_TOKENS = [
    (13, 4096, 11008, BF16, 4, (2, 2, 2)),
    (16, 2100, 16391, BF16, 4, (1, 1, 1)),
    (5, 4001, 5000, BF16, 2, (1, 1, 1)),
    (9, 9000, 5001, BF16, 2, (3, 2, 2)),
    (2, 16384, 16390, BF16, 2, (2, 2, 1)),
    (16, 9000, 17001, BF16, 4, (4, 4, 4)),
    (13, 3900, 11003, F32, 4, (4, 4, 4)),
    (16, 2100, 16400, F32, 4, (3, 3, 3)),
    (5, 4001, 5000, F32, 2, (2, 2, 2)),
    (2, 16384, 16390, F32, 2, (4, 3, 3)),
]

# tokens, n_in, n_out of tardis_linear_fp8 with outputs in bf16, launches (rows that are not whole pieces: two copies; ranges of K: the sum)
LARGE_TILES = [
    (96, 1040, 32768, 1),        # 96 rows of a tile, a rest of 16 columns
    (270, 4000, 16384, 1),       # tiles of 160 and 110 rows, a rest of 32
    (333, 4048, 11008, 1),       # a rest of 80
    (512, 1000, 11008, 3),       # copied, a rest of 112
    (150, 11008, 11008, 2),      # ranges of K
    (270, 11024, 2048, 2),       # ranges of K of which the last has a rest
    (1000, 11008, 4096, 2),      # full tiles, ranges of K
    (513, 8192, 4100, 2),        # outputs in whole 8 bytes, ranges of K
    (600, 4000, 9001, 1),        # outputs at odd places
    (700, 2050, 8190, 3),        # copied, a rest of 16
    (2048, 4112, 4096, 1),
]
