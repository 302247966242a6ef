"""Block-scaled caches, rotated appends and truncation on the host: the split plans do
all work once and fit their workspaces, buffers are kept to, refusals change nothing
(tests/sanitize/block_plans.cpp under AddressSanitizer and UBSan; no GPU needed).
"""
import os
import shutil

import pytest

from test_sanitizers import ENV, ROOT, SAN, _run


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_block_plans_and_bookkeeping(tmp_path):
    exe = str(tmp_path / "block_plans")
    san, csrc = os.path.join(ROOT, "tests", "sanitize"), os.path.join(ROOT, "paper_2607_16248_amd", "csrc")
    _run(["g++", "-std=c++17", "-Wno-return-type-c-linkage"] + SAN + ["-I", san, "-I", os.path.join(ROOT, "include"), "-I", csrc]
         + [os.path.join(csrc, f) for f in ("kvq_api.cpp", "kvq_rotary.cpp", "dgap_adjust.cpp")]
         + [os.path.join(san, f) for f in ("hip_stub.cpp", "block_stub.cpp", "block_plans.cpp")] + ["-o", exe])
    assert "block plans ok" in _run([exe], env=ENV, timeout=500).stdout
