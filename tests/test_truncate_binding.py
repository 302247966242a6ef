"""kvq_truncate's binding: as many lengths as the cache has sequences (the call reads one for
each), no GPU needed."""
import pytest

from paper_2607_16248_amd import kvq
from test_block_boundary import handle


@pytest.mark.parametrize("batch", [1, 2, 5])
def test_lengths_of_every_sequence(batch):
    h = handle(batch=batch)
    try:
        for n in [k for k in range(batch + 3) if k != batch]:
            with pytest.raises(ValueError):
                kvq.kvq_truncate(h, [0] * n)
        kvq.kvq_truncate(h, [0] * batch)
        with pytest.raises(ValueError):
            kvq.kvq_truncate(h, [0] * (batch - 1) + [-1])
    finally:
        kvq.kvq_cache_destroy(h)


def test_a_cache_that_is_none():
    with pytest.raises(kvq.KvqError) as e:
        kvq.kvq_truncate(None, [0])
    assert e.value.status == kvq.ERR_ARG
