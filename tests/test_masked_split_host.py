"""CPU: requests of few rows get a launch of their own once they are 8 tiles a workgroup, on machines of any size."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def harness(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("split") / "masked_split_harness")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", os.path.join(ROOT, "tests", "masked_split_harness.cpp"),
                    "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("cus", [256, 128, 64, 32])
@pytest.mark.parametrize("hkv", [4, 8])
@pytest.mark.parametrize("rows,mid", [(8, 0), (32, 1)])
def test_few_rows_go_with_the_chunk_until_they_fill_the_machine(harness, rows, mid, hkv, cus):
    res = subprocess.run([harness, str(cus), str(hkv), str(rows), str(mid)], capture_output=True, text=True, check=True)
    own = [(0, 64) if mid else (16, 16), (0, 0)]  # (hi16, hi64): a launch of their own, or none
    for line in res.stdout.splitlines():
        n, hi16, hi64 = map(int, line.split())
        tiles = 32 * n * hkv  # 1000 keys are 32 tiles of 32 to each KV head
        assert (hi16, hi64) == own[tiles < 8 * 2 * cus], (n, hi16, hi64)  # (two workgroups a CU)
