"""The router's working memory may begin at any whole word: what the compiler is told (on the CPU), and that the call works there."""
import ctypes as C
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_2501_10054_amd import build as B
from paper_2501_10054_amd import tardis as T


def test_the_counts_are_read_as_words(tmp_path):
    """No load from global memory in the placing kernel is of a type that needs more than 4 bytes' alignment, but of the kernel's arguments."""
    if not (shutil.which("hipcc") or os.path.exists("/opt/rocm/bin/hipcc")):
        pytest.skip("no hipcc")
    out = str(tmp_path / "experts.ll")
    subprocess.run([B._hipcc(), *B.FLAGS, "--offload-device-only", "-emit-llvm", "-S", os.path.join(B.CSRC, "experts.hip"), "-o", out], check=True, capture_output=True)
    with open(out) as f:
        text = f.read()
    body = re.search(r"define [^\n]*route_place_kernel.*?\n}", text, re.S)[0]
    loads = re.findall(r"load [^\n]*addrspace\(1\)[^\n]*align (\d+)", body)
    assert loads and all(int(a) <= 4 for a in loads), loads


@pytest.mark.gpu
@pytest.mark.parametrize("experts,k", [(3, 2), (60, 4), (128, 8), (257, 3), (1024, 16)])
def test_memory_at_any_word(experts, k):
    gen = torch.Generator(device="cuda").manual_seed(experts)
    n = 5000
    logits = torch.randn(n, experts, device="cuda", generator=gen)
    want = T.tardis_moe_route(logits, k)
    need = C.c_int64()
    assert T.lib().tardis_moe_route_workspace(n, experts, k, need) == T.OK and need.value > 0
    for at in (4, 8, 12):
        work = torch.full((need.value + 32,), 77, dtype=torch.uint8, device="cuda")
        got = [torch.empty_like(t) for t in want]
        ids, weights, offsets, order, place = (t.data_ptr() for t in got)
        st = T.lib().tardis_moe_route(logits.data_ptr(), n, experts, k, T.F32, 1, ids, weights, offsets, order, place, work.data_ptr() + at, need.value,
                                      torch.cuda.current_stream().cuda_stream)
        assert st == T.OK
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert (work[:at] == 77).all() and (work[at + need.value:] == 77).all()
