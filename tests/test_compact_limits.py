"""Compaction of accepted drafts with counts and lists at the limits of their type: the arithmetic on the CPU, and one
call on the GPU."""
import os
import subprocess

import numpy as np
import pytest

from oracle import masked as M
from paper_2511_20982_amd import attn as A
from paper_2511_20982_amd import inputs as I

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_tokens_at_the_limits(tmp_path):
    exe = str(tmp_path / "compact_harness")
    subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", os.path.join(ROOT, "tests", "compact_harness.cpp"), "-o",
                    exe], check=True)
    res = subprocess.run([exe], capture_output=True, text=True)
    assert res.returncode == 0 and res.stdout.strip() == "ok", res.stdout + res.stderr


@pytest.mark.gpu
def test_the_longest_list(require_gpu):
    """2^31 - 1 accepted tokens by count and by list, of which two have places and sources in the page table."""
    import torch
    rng = np.random.default_rng(6)
    prefix, most, stride = np.array([30], np.int32), 2 ** 31 - 1, 8
    pt, pages = I.allocate_pages(rng, np.array([16 * stride]))
    k = rng.integers(0, 2 ** 15, (2, pages, 2, 16, 64)).astype(np.uint16)
    v = rng.integers(0, 2 ** 15, (2, pages, 2, 64, 16)).astype(np.uint16)
    path = torch.empty(most, dtype=torch.int32, device="cuda")
    path[:16 * stride] = 10 ** 6  # (past the table; what lies behind is not read)
    path[:2] = torch.tensor([1, 3], dtype=torch.int32)
    kd, vd = A.to_device(k), A.to_device(v)
    A.dopd_kv_compact(A.make_shape(2, 2, 64), 2, kd, vd, pages, A.to_device(pt), stride, A.to_device(prefix), path,
                      A.to_device(np.array([most], np.int32)), most, 1)
    torch.cuda.synchronize()
    want = M.compact(k, v, pt, prefix, np.array([[1, 3]]), [2])
    assert np.array_equal(A.to_host(kd), want[0]) and np.array_equal(A.to_host(vd), want[1])
