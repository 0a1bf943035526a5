"""The listings of the kernels of layers in 8 and 4 bits: m0 belongs to their loads to LDS, the products in inline assembly are waited for, scalars that vector
instructions write are not read too early, and no register spills."""
import os
import re
import shutil
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2501_10054_amd import build as B
from test_gemm_listing import BEFORE_MFMA, _kernels, _walk
from test_gemm_quad_listing import _registers

# kernels and how many there are
SOURCES = {"linear_fp8": ("linear_fp8_kernel", 19), "linear_fp8_quad": ("linear_fp8_quad_kernel", 1), "linear_4bit": ("linear4_", 48)}
AFTER_WIDE_MFMA = 18       # wait states behind an instruction of 16 passes whose result is read


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    if not (shutil.which("hipcc") or os.path.exists("/opt/rocm/bin/hipcc")):
        pytest.skip("no hipcc")
    tmp = str(tmp_path_factory.mktemp("listing"))

    def listing(name):
        out = os.path.join(tmp, name + ".s")
        subprocess.run([B._hipcc(), *B.FLAGS, "--offload-device-only", "-S", os.path.join(B.CSRC, name + ".hip"), "-o", out], check=True, capture_output=True)
        with open(out) as f:
            return f.read()

    with ThreadPoolExecutor(4) as ex:
        return dict(zip(SOURCES, ex.map(listing, SOURCES)))


@pytest.mark.parametrize("source", SOURCES)
def test_nothing_spills(listings, source):
    text = listings[source]
    seen = 0
    for part in re.split(r"\n  - \.agpr_count", text[text.index("amdhsa.kernels:"):])[1:]:
        name = re.search(r"\.name:\s+(\S+)", part)[1]
        seen += 1
        assert int(re.search(r"\.vgpr_spill_count:\s+(\d+)", part)[1]) == 0, name
        assert int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", part)[1]) == 0, name
    assert seen == SOURCES[source][1]


@pytest.mark.parametrize("source", ["linear_fp8", "linear_fp8_quad", "linear_4bit"])
def test_m0_belongs_to_the_loads_to_lds(listings, source):
    loads = 0
    for name, (code, _) in _kernels(listings[source], SOURCES[source][0]).items():
        written = None
        for i, (op, rest) in enumerate(code):
            if re.search(r"\bm0\b", rest):
                assert op in ("s_add_u32", "s_mov_b32") and rest.startswith("m0, s") and written is None, (name, op, rest)
                written = i
            elif op.startswith("buffer_load") and "lds" in rest:
                assert written is not None and i - written >= 2, (name, op, rest)
                written = None
                loads += 1
        assert written is None, name
    assert loads > 0


@pytest.mark.parametrize("source", ["linear_fp8", "linear_fp8_quad", "linear_4bit"])
def test_scalars_written_by_vector_instructions_are_waited_for(listings, source):
    """5 wait states between a vector instruction that writes a scalar register and a load that reads it: the loads are inline assembly."""
    def scalars(text):
        regs = set()
        for m in re.finditer(r"\bs(?:\[(\d+):(\d+)\]|(\d+)\b)", text):
            lo, hi = (int(m[1]), int(m[2])) if m[1] else (int(m[3]), int(m[3]))
            regs.update(range(lo, hi + 1))
        return regs

    for name, (code, labels) in _kernels(listings[source], SOURCES[source][0]).items():
        for i, (op, rest) in enumerate(code):
            if not op.startswith(("v_readlane", "v_readfirstlane", "v_cmp")):
                continue
            written = scalars(rest.split(",")[0])
            for k in _walk(code, labels, i, 5):
                if code[k][0].startswith("buffer_load"):
                    assert not written & scalars(code[k][1]), (name, op, rest, code[k])


def test_results_of_matrix_instructions_are_waited_for(listings):
    for name, (code, labels) in _kernels(listings["linear_fp8_quad"], "linear_fp8_quad_kernel").items():
        operands = [[_registers(p) for p in re.split(r",\s*", rest)] if rest else [] for _, rest in code]
        every = [set().union(*o) if o else set() for o in operands]
        assert sum(op.startswith("v_mfma") for op, _ in code) >= 16, name
        for i, (op, rest) in enumerate(code):
            if op.startswith("v_mfma"):
                assert op == "v_mfma_f32_32x32x64_f8f6f4", op
                result = operands[i][0]
                for k in _walk(code, labels, i, AFTER_WIDE_MFMA):
                    again = (code[k][0].startswith("v_mfma") and operands[k][0] == result == operands[k][3] and
                             not (operands[k][1] | operands[k][2]) & result)
                    assert again or not every[k] & result, (name, op, rest, code[k])
            elif op.startswith("v_") and operands[i] and operands[i][0]:
                for k in _walk(code, labels, i, BEFORE_MFMA):
                    if code[k][0].startswith("v_mfma"):
                        assert not operands[i][0] & set().union(*operands[k][1:4]), (name, op, rest, code[k])


def test_codes_for_outputs_in_fp32_are_multiplied_as_bf16(listings):
    """The instructions that multiply codes drop products below 2^-13 of the largest: of kernels with exact sums none."""
    for name, (code, _) in _kernels(listings["linear_fp8"], "linear_fp8_kernel").items():
        ops = {op for op, _ in code if op.startswith("v_mfma")}
        assert ops == ({"v_mfma_f32_16x16x128_f8f6f4"} if "e4m3_near_t" in name else {"v_mfma_f32_16x16x32_bf16"}), (name, ops)
