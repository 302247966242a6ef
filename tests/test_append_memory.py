"""No exception leaves the appends, whichever of their host allocations fails, and a call
that fails leaves the cache as it was (tests/sanitize/append_memory.cpp; no GPU needed).
"""
import os
import shutil

import pytest

from test_sanitizers import ENV, ROOT, SAN, _run


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_appends_without_host_memory_change_nothing(tmp_path):
    exe = str(tmp_path / "append_memory")
    san, csrc = os.path.join(ROOT, "tests", "sanitize"), os.path.join(ROOT, "paper_2607_16248_amd", "csrc")
    _run(["g++", "-std=c++17", "-Wno-return-type-c-linkage"] + SAN + ["-I", san, "-I", os.path.join(ROOT, "include"), "-I", csrc]
         + [os.path.join(csrc, f) for f in ("kvq_api.cpp", "kvq_block.cpp", "kvq_rotary.cpp")]
         + [os.path.join(san, f) for f in ("hip_stub.cpp", "block_stub.cpp", "append_memory.cpp")] + ["-o", exe])
    assert "append memory ok" in _run([exe], env=ENV, timeout=300).stdout
