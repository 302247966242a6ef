"""Block-scaled attention under forced splits of one block, over large batches and long
caches: no call of valid arguments is refused (tests/sanitize/block_limits.cpp; no GPU needed).
"""
import os
import shutil

import pytest

from test_sanitizers import ENV, ROOT, _run


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_plans_at_their_limits(tmp_path):
    exe = str(tmp_path / "block_limits")
    san, csrc = os.path.join(ROOT, "tests", "sanitize"), os.path.join(ROOT, "paper_2607_16248_amd", "csrc")
    _run(["g++", "-std=c++17", "-O2", "-g", "-fsanitize=undefined", "-fno-sanitize-recover=all", "-Wno-return-type-c-linkage",
          "-I", san, "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(csrc, "kvq_api.cpp")]
         + [os.path.join(san, f) for f in ("hip_stub.cpp", "block_stub.cpp", "block_limits.cpp")] + ["-o", exe])
    assert "block limits ok" in _run([exe], env=ENV, timeout=400).stdout
