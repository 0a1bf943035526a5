"""The tests that call the linear layer's kernels by their numbers are made from the built probe: none of them is lost where it has not been built."""
import os
import re
import shutil
import subprocess
import sys

import pytest

from paper_2501_10054_amd import build as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(not (shutil.which("hipcc") or os.path.exists("/opt/rocm/bin/hipcc")), reason="no hipcc")
def test_a_tree_without_the_probe_has_all_of_them(tmp_path):
    lost = shutil.ignore_patterns("__pycache__", os.path.basename(B.LINEAR_PROBE) + "*")
    for part in ("paper_2501_10054_amd", "tests", "include"):
        shutil.copytree(os.path.join(ROOT, part), tmp_path / part, ignore=lost)
    assert not (tmp_path / os.path.relpath(B.LINEAR_PROBE, ROOT)).exists()
    said = subprocess.run([sys.executable, "-m", "pytest", "--collect-only", "-q", "-p", "no:cacheprovider", "tests/test_gpu_linear_tiles.py"], cwd=tmp_path,
                          capture_output=True, text=True)
    assert said.returncode == 0, said.stdout + said.stderr
    names = re.findall(r"::(test_\w+)\[", said.stdout)
    # (24 tiles in bf16 and 13 in fp32, of which groups have 22 and 10)
    assert {n: names.count(n) for n in set(names)} == {"test_edges_of_a_tile": 37, "test_ranges_of_a_row": 37, "test_groups": 32}


def test_the_probe_is_there():
    assert os.path.exists(B.LINEAR_PROBE)


@pytest.mark.gpu
def test_the_probe_is_there_on_the_gpu():
    assert os.path.exists(B.LINEAR_PROBE)
