"""The listings of the linear layer's kernels: linear_quad_kernel issues its MFMAs as inline assembly, so that behind and before them the
waits of the hardware are read here; both kernels set m0 by hand for their loads to LDS; no register spills."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2501_10054_amd import build as B
from test_gemm_listing import AFTER_MFMA, BEFORE_MFMA, PACKED_OFF, _kernels, _walk
from test_gemm_quad_listing import _registers

SOURCES = ("linear_quad", "linear_bf16", "linear_f32")


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    if not (shutil.which("hipcc") or os.path.exists("/opt/rocm/bin/hipcc")):
        pytest.skip("no hipcc")
    tmp = str(tmp_path_factory.mktemp("listing"))

    def listing(job):
        name, packed = job
        flags, out = list(B.FLAGS), os.path.join(tmp, f"{name}_{packed}.s")
        if packed:
            at = next(i for i in range(len(flags)) if flags[i:i + 4] == PACKED_OFF)
            del flags[at:at + 4]
        subprocess.run([B._hipcc(), *flags, "--offload-device-only", "-S", os.path.join(B.CSRC, name + ".hip"), "-o", out], check=True, capture_output=True)
        with open(out) as f:
            return f.read()

    jobs = [(s, False) for s in SOURCES] + [("linear_quad", True)]
    with ThreadPoolExecutor(4) as ex:
        return dict(zip(jobs, ex.map(listing, jobs)))


@pytest.mark.parametrize("packed", [False, True])
def test_results_of_matrix_instructions_are_waited_for(listings, packed):
    kernels = _kernels(listings["linear_quad", packed], "linear_quad_kernel")
    assert len(kernels) == 6                        # 3 tiles, with and without groups
    for name, (code, labels) in kernels.items():
        operands = [[_registers(p) for p in re.split(r",\s*", rest)] if rest else [] for _, rest in code]
        every = [set().union(*o) if o else set() for o in operands]
        assert sum(op.startswith("v_mfma") for op, _ in code) >= 4 * 32, name
        for i, (op, rest) in enumerate(code):
            if op.startswith("v_mfma"):
                result = operands[i][0]
                for k in _walk(code, labels, i, AFTER_MFMA):
                    again = (code[k][0].startswith("v_mfma") and operands[k][0] == result == operands[k][3] and
                             not (operands[k][1] | operands[k][2]) & result)
                    assert again or not every[k] & result, (name, op, rest, code[k])
            elif op.startswith("v_") and operands[i] and operands[i][0]:
                for k in _walk(code, labels, i, BEFORE_MFMA):
                    if code[k][0].startswith("v_mfma"):
                        assert not operands[i][0] & set().union(*operands[k][1:4]), (name, op, rest, code[k])


def test_m0_belongs_to_the_loads_to_lds_of_large_tiles(listings):
    """Every load to LDS finds the m0 written for it, at least one instruction before, and nothing else uses m0."""
    for name, (code, _) in _kernels(listings["linear_quad", False], "linear_quad_kernel").items():
        written, loads = None, 0
        for i, (op, rest) in enumerate(code):
            if re.search(r"\bm0\b", rest):
                assert op == "s_add_u32" and rest.startswith("m0, s") and written is None, (name, op, rest)
                written = i
            elif op.startswith("buffer_load") and "lds" in rest:
                assert written is not None and i - written >= 2, (name, op, rest)
                written = None
                loads += 1
        assert loads > 0 and written is None, name


@pytest.mark.parametrize("source", ["linear_bf16", "linear_f32"])
def test_m0_belongs_to_the_loads_to_lds(listings, source):
    """m0 is written by the statement that loads to LDS and cannot be declared as overwritten: nothing else may use it."""
    kernels = _kernels(listings[source, False], "linear_kernel")
    assert len(kernels) == {"linear_bf16": 21 + 19, "linear_f32": 13 + 10}[source]      # without and with groups
    loads = 0
    for name, (code, _) in kernels.items():
        for i, (op, rest) in enumerate(code):
            if re.search(r"\bm0\b", rest):
                assert op == "s_mov_b32" and rest.startswith("m0, s"), (name, op, rest)
                assert [code[i + 1][0], code[i + 2][0]] == ["s_nop", "buffer_load_dwordx4"] and "lds" in code[i + 2][1], name
                loads += 1
    assert loads > 0


def test_nothing_spills(listings):
    seen = 0
    for text in listings.values():
        for part in re.split(r"\n  - \.agpr_count", text[text.index("amdhsa.kernels:"):])[1:]:
            name = re.search(r"\.name:\s+(\S+)", part)[1]
            seen += 1
            assert int(re.search(r"\.vgpr_spill_count:\s+(\d+)", part)[1]) == 0, name
            assert int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", part)[1]) == 0, name
    assert seen == 40 + 23 + 2 * 6


@pytest.mark.parametrize("source,kernel", [("linear_quad", "linear_quad_kernel"), ("linear_bf16", "linear_kernel"), ("linear_f32", "linear_kernel")])
def test_scalars_written_by_vector_instructions_are_waited_for(listings, source, kernel):
    """5 wait states between a vector instruction that writes a scalar register and a load that reads it: the loads are inline assembly, whose
    operands the compiler takes for ready."""
    def scalars(text):
        regs = set()
        for m in re.finditer(r"\bs(?:\[(\d+):(\d+)\]|(\d+)\b)", text):
            lo, hi = (int(m[1]), int(m[2])) if m[1] else (int(m[3]), int(m[3]))
            regs.update(range(lo, hi + 1))
        return regs

    for name, (code, labels) in _kernels(listings[source, False], kernel).items():
        for i, (op, rest) in enumerate(code):
            if not op.startswith(("v_readlane", "v_readfirstlane", "v_cmp")):
                continue
            written = scalars(rest.split(",")[0])
            for k in _walk(code, labels, i, 5):
                if code[k][0].startswith("buffer_load"):
                    assert not written & scalars(code[k][1]), (name, op, rest, code[k])
