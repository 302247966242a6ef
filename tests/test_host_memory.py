"""No exception leaves the C interface: the attention calls with every one of their host
allocations failing in turn (tests/sanitize/host_memory.cpp; no GPU needed).
"""
import os
import shutil

import pytest

from test_sanitizers import ENV, ROOT, SAN, _run


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_calls_without_host_memory_return_a_status(tmp_path):
    exe = str(tmp_path / "host_memory")
    san = os.path.join(ROOT, "tests", "sanitize")
    csrc = os.path.join(ROOT, "paper_2607_16248_amd", "csrc")
    _run(["g++", "-std=c++17", "-Wno-return-type-c-linkage"] + SAN +
         ["-I", san, "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(csrc, "kvq_api.cpp"),
          os.path.join(san, "hip_stub.cpp"), os.path.join(san, "host_memory.cpp"), "-o", exe])
    assert "host memory ok" in _run([exe], env=ENV, timeout=300).stdout
