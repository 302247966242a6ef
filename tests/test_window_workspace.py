"""Workspaces of windowed attention: the split plans of random caches and lengths against
the size that a call is said to need (tests/sanitize/window_plans.cpp, host code under
AddressSanitizer and UBSan), and that size through the binding.  No GPU needed.
"""
import os
import shutil

import pytest

from paper_2607_16248_amd import kvq
from test_sanitizers import ENV, ROOT, SAN, _run


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_plans_fit_their_workspace(tmp_path):
    exe = str(tmp_path / "window_plans")
    san = os.path.join(ROOT, "tests", "sanitize")
    _run(["g++", "-std=c++17", "-Wno-return-type-c-linkage"] + SAN +
         ["-I", san, "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2607_16248_amd", "csrc"),
          os.path.join(san, "window_plans.cpp"), os.path.join(san, "hip_stub.cpp"), "-o", exe])
    assert "window plans ok" in _run([exe], env=ENV, timeout=300).stdout


@pytest.mark.parametrize("batch", [1, 4, 16, 64])
def test_long_chunks_of_large_batches(batch):
    # 1024 queries of 32 heads: a split's records are 17.3 MB; no more than 8 rounds of workgroups
    # (16 for several sequences) are ever split, 128 workgroups a split
    desc = kvq.make_desc(batch, 32, 8, 128, 32768, 32, 32, 128, [2] * batch, [2] * batch)
    h = kvq.kvq_cache_init(desc, 1 << 30, kvq.kvq_cache_bytes(desc))
    split = 32 * 1024 * 132 * 4
    for window in (4096, 1 << 30):
        assert 0 < kvq.kvq_window_workspace_bytes(h, 1024, window, 4) <= (16 if batch == 1 else 32) * split
    kvq.kvq_cache_destroy(h)
