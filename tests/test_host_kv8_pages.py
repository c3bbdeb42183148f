"""What the 8-bit KV cache holds and hands out, without a GPU: its pages are its own, and what it grows by."""
import numpy as np
import pytest

from paper_2311_03285_amd import slora
from test_host_kv8 import refused


@pytest.fixture
def cache():
    pool = slora.pool_init(512, 200, slora.F16, None, 1, 16)
    c = slora.kv8_init(pool, 1, 2, 2, 64, 4, 100, None)
    yield pool, c
    slora.kv8_destroy(c)
    slora.pool_destroy(pool)


def test_pages_of_a_cache_are_nobody_elses(cache):
    """the caller's own KV pages can be given back; those that the cache took only by the cache"""
    pool, c = cache
    slora.pool_mark_kv(pool, [5, 6])
    slora.kv8_extend(c, [1], [20], [10, 11, 12, 13, 14, 15])
    for owned in (False, True):
        for pages in ([12], [5, 6, 15], [40, 10]):
            refused(slora.EBUSY, slora.pool_mark_kv, pool, pages, owned)
            assert slora.pool_free_pages(pool) == 200 - 8
    refused(slora.EBUSY, slora.adapter_load, pool, 1, 1, [12, 40])
    slora.pool_mark_kv(pool, [5, 6], False)
    slora.pool_mark_kv(pool, [5, 6])
    slora.kv8_truncate(c, [1], [8])  # the first block stays
    slora.pool_mark_kv(pool, [12, 13, 14, 15])
    slora.pool_mark_kv(pool, [12, 13, 14, 15], False)
    refused(slora.EBUSY, slora.pool_mark_kv, pool, [11], False)
    # pages of the library's choice, and another cache of the pool
    other = slora.kv8_init(pool, 1, 1, 1, 64, 1, 2000, None)
    slora.kv8_extend(other, [0], [190 * 8])
    assert slora.pool_free_pages(pool) == 200 - 2 - 2 - 190
    refused(slora.EBUSY, slora.pool_mark_kv, pool, [100], False)
    slora.kv8_destroy(other)
    slora.pool_mark_kv(pool, np.arange(100, 120))
    slora.pool_mark_kv(pool, np.arange(100, 120), False)
    assert slora.pool_free_pages(pool) == 200 - 2 - 2


def test_exponents_that_are_not_aligned(cache):
    pool, _ = cache
    refused(slora.EINVAL, slora.kv8_init, pool, 1, 2, 2, 64, 4, 100, 4097)
    slora.kv8_destroy(slora.kv8_init(pool, 1, 2, 2, 64, 4, 100, 4098))
