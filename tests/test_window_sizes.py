"""Sizes of a windowed call that do not fit the C interface's 32 bits (no GPU needed):
refused, not cut to their lowest 32 bits, which would be another window.
"""
import pytest

from paper_2607_16248_amd import kvq

torch = pytest.importorskip("torch")

BIG = [1 << 31, 1 << 32, (1 << 32) + 64, 1 << 40, (1 << 63) - 1, -(1 << 32) + 64]


@pytest.mark.parametrize("big", BIG)
@pytest.mark.parametrize("name", ["n_q", "window", "sinks"])
def test_refused(name, big):
    desc = kvq.make_desc(2, 8, 2, 128, 512, 32, 32, 0, [2, 4], [2, 8])
    h = kvq.kvq_cache_init(desc, 1 << 30, kvq.kvq_cache_bytes(desc))
    sizes = {"n_q": 1, "window": 64, "sinks": 4, name: big}
    with pytest.raises(ValueError, match=f"{name} = "):
        kvq.kvq_window_workspace_bytes(h, **sizes)
    with pytest.raises(ValueError, match=f"{name} = "):
        kvq.kvq_window_attention(h, 1 << 30, sizes["n_q"], sizes["window"], sizes["sinks"], 1 << 30, 1 << 30, 1 << 40)
    assert kvq.kvq_window_workspace_bytes(h, 1, (1 << 31) - 1, (1 << 31) - 1) > 0
    kvq.kvq_cache_destroy(h)
