"""One call for each kernel of the layers in 8 and 4 bits and of the norm: the kernel (its template arguments), and the call's sizes."""
from paper_2501_10054_amd.tardis import BF16, F32, FP8_E4M3

# tokens, n_in, n_out, bytes between rows of x, type of y
EIGHT = [
    ("linear_fp8_kernel near 1 2 1 1 2 4 2 5", 40, 8192, 4096, 0, BF16),
    ("linear_fp8_kernel near 1 2 2 1 2 4 2 3", 128, 4096, 4096, 0, BF16),
    ("linear_fp8_kernel near 1 2 2 2 2 1 2 2", 84, 16, 18075, 0, BF16),
    ("linear_fp8_kernel near 1 2 2 2 2 2 2 5", 64, 4096, 11008, 0, BF16),
    ("linear_fp8_kernel near 1 2 4 2 2 2 2 3", 1, 4992, 18578, 0, BF16),
    ("linear_fp8_kernel near 1 4 2 2 2 2 2 3", 333, 11008, 4096, 0, BF16),
    ("linear_fp8_kernel near 1 4 4 2 2 1 2 2", 4368, 1, 1897, 0, BF16),
    ("linear_fp8_kernel near 1 4 4 2 2 2 2 2", 9866, 16, 271, 0, BF16),
    ("linear_fp8_kernel exact 0 1 1 1 1 8 1 6", 1, 1288, 1, 0, BF16),
    ("linear_fp8_kernel exact 0 2 1 1 2 4 1 4", 1, 129, 1, 3, BF16),
    ("linear_fp8_kernel exact 0 2 2 2 2 2 1 4", 1, 1, 8195, 0, BF16),
    ("linear_fp8_kernel exact 0 4 4 2 2 2 1 2", 83, 1, 17912, 0, BF16),
    ("linear_fp8_kernel exact 1 1 1 1 1 8 1 5", 1, 16384, 4096, 0, BF16),
    ("linear_fp8_kernel exact 1 1 1 1 1 8 2 5", 1, 528, 1, 16, BF16),
    ("linear_fp8_kernel exact 1 1 2 1 1 8 1 3", 1, 4096, 11008, 0, BF16),
    ("linear_fp8_kernel exact 1 2 2 1 2 4 2 3", 1706, 3008, 187, 0, F32),
    ("linear_fp8_kernel exact 1 2 2 2 2 1 2 2", 405, 16, 5164, 0, F32),
    ("linear_fp8_kernel exact 1 2 2 2 2 2 2 5", 10676, 3584, 33, 16, F32),
    ("linear_fp8_kernel exact 1 4 4 2 2 1 2 2", 2048, 4096, 4096, 0, F32),
    ("linear_fp8_quad_kernel 8 4", 700, 2048, 8192, 0, BF16),
]

# tokens, n_in, n_out, group, type of x
FOUR = []
for _group, _words in ((32, 1), (64, 2), (128, 4)):
    for _type, _parts, _name in ((BF16, 1, "bf16"), (F32, 3, "f32")):
        for _rows, _n_out in ((1, 1000), (2, 5000), (4, 16400)):
            FOUR.append((f"linear4_kernel {_name} {_words} {_rows}", 1, 300, _n_out, _group, _type))
        _deep = (6, 5, 3) if _parts == 1 else (2, 2, 2)
        FOUR.append((f"linear4_prepare_kernel {_name} {_words}", 70, 500, 300, _group, _type))
        FOUR.append((f"linear4_tile_kernel {_parts} {_words} 1 1 4 {_deep[0]}", 15, 16300, 70, _group, _type))
        FOUR.append((f"linear4_tile_kernel {_parts} {_words} 2 1 4 {_deep[1]}", 29, 1300, 130, _group, _type))
        FOUR.append((f"linear4_tile_kernel {_parts} {_words} 4 1 4 {_deep[2]}", 70, 900, 300, _group, _type))
        FOUR.append((f"linear4_tile_kernel {_parts} {_words} 4 4 4 2", 400, 300, 10000, _group, _type))

# rows, columns, type of x, type of y
NORM = [(f"rms_norm_kernel {name} {out} {each}", n, d, dtype, out) for name, dtype in (("bf16", BF16), ("f32", F32)) for out in (F32, BF16, FP8_E4M3)
        for each, n, d in ((1, 3, 4096), (2, 1021, 5137) if out == FP8_E4M3 else (2, 50, 16000), (4, 2048, 4096) if out == FP8_E4M3 else (4, 20, 30001), (8, 300, 40000),
                           (0, 2, 70001))]
