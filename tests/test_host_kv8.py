"""The 8-bit KV cache and the 4-bit products without a GPU: bookkeeping of a host-only pool, and every refusal - with its code, and
with nothing changed."""
import numpy as np
import pytest

from paper_2311_03285_amd import slora

H, D, LAYERS, KV = 512, 64, 2, 3
BLOCK = 8  # tokens of a page of 512 elements


@pytest.fixture
def cache():
    pool = slora.pool_init(H, 200, slora.F16, None, 1, 16)
    c = slora.kv8_init(pool, LAYERS, 6, KV, D, 4, 100, None)
    yield pool, c
    slora.kv8_destroy(c)
    slora.pool_destroy(pool)


def refused(code, call, *args, **kw):
    with pytest.raises(slora.SloraError) as e:
        call(*args, **kw)
    assert e.value.code == code, str(e.value)


def test_blocks_and_pages(cache):
    pool, c = cache
    per = LAYERS * KV
    assert slora.kv8_info(c) == {"block": BLOCK, "max_blocks": 13, "pages_per_block": per, "pages": 0}
    slora.kv8_extend(c, [0, 2], [1, 17])
    assert slora.kv8_info(c)["pages"] == (1 + 3) * per and slora.pool_free_pages(pool) == 200 - 4 * per
    slora.kv8_extend(c, [0], [7])  # fills the block
    assert slora.kv8_info(c)["pages"] == 4 * per
    slora.kv8_extend(c, [0, 1], [1, 0])
    assert slora.kv8_info(c)["pages"] == 5 * per
    assert slora.kv8_lengths(c, [2, 0, 1]).tolist() == [17, 9, 0]
    slora.kv8_truncate(c, [2, 0], [16, 9])
    assert slora.pool_free_pages(pool) == 200 - 4 * per
    slora.kv8_truncate(c, [2, 0], [0, 1], evicted=True)
    assert slora.pool_free_pages(pool) == 200 - per
    # adapters and cache draw from one pool
    slora.adapter_alloc(pool, 7, 16, 1)
    slora.adapter_alloc(pool, 8, 16, 1)
    refused(slora.ENOMEM, slora.kv8_extend, c, [3, 1], [100, 100])
    assert slora.kv8_lengths(c, [3, 1]).tolist() == [0, 0] and slora.kv8_info(c)["pages"] == per
    slora.adapter_unload(pool, 7)
    slora.adapter_unload(pool, 8)
    slora.kv8_extend(c, [3, 1], [100, 100])


def test_pages_by_name(cache):
    pool, c = cache
    per = LAYERS * KV
    pages = np.arange(per) * 3
    slora.pool_mark_kv(pool, [100])
    for bad, code in ((pages[:-1], slora.EINVAL), (np.append(pages, 190), slora.EINVAL), (np.where(pages == 3, 0, pages), slora.EBUSY),
                      (np.where(pages == 3, 100, pages), slora.EBUSY), (np.where(pages == 3, 200, pages), slora.ERANGE), (np.where(pages == 3, -1, pages), slora.ERANGE)):
        refused(code, slora.kv8_extend, c, [1], [5], bad)
        assert slora.pool_free_pages(pool) == 199 and slora.kv8_lengths(c, [1])[0] == 0
    slora.kv8_extend(c, [1], [5], pages)
    assert slora.pool_free_pages(pool) == 199 - per
    refused(slora.EBUSY, slora.adapter_load, pool, 1, 1, [0, 1])
    slora.kv8_truncate(c, [1], [0])
    slora.adapter_load(pool, 1, 1, [0, 1])


def test_sequences_out_of_order(cache):
    _, c = cache
    for call in (slora.kv8_extend, slora.kv8_truncate, slora.kv8_batch_plan):
        refused(slora.ERANGE, call, c, [0, 4], [0, 0])
        refused(slora.ERANGE, call, c, [-1], [0])
        refused(slora.EBUSY, call, c, [1, 0, 1], [0, 0, 0])
        with pytest.raises(ValueError):
            call(c, [0, 1], [0])
    refused(slora.ERANGE, slora.kv8_extend, c, [0], [101])
    refused(slora.ERANGE, slora.kv8_extend, c, [0], [-1])
    slora.kv8_extend(c, [0], [60])
    refused(slora.ERANGE, slora.kv8_extend, c, [0], [41])
    refused(slora.ERANGE, slora.kv8_truncate, c, [0], [61])
    refused(slora.ERANGE, slora.kv8_truncate, c, [0], [-1])
    refused(slora.ERANGE, slora.kv8_lengths, c, [4])
    refused(slora.EINVAL, slora.kv8_batch_plan, c, [0], [-1])
    refused(slora.EINVAL, slora.kv8_batch_plan, c, [0], [1], [-1])


def test_batches(cache):
    pool, c = cache
    slora.kv8_extend(c, [0, 1], [10, 20])
    b = slora.kv8_batch_plan(c, [0, 1], [1, 5], [4, 40])
    refused(slora.EBUSY, slora.kv8_destroy, c)
    refused(slora.EBUSY, slora.pool_destroy, pool)
    refused(slora.ERANGE, slora.kv8_append, b, LAYERS, 16, 192, 16, 192)
    refused(slora.ERANGE, slora.kv8_attend, b, -1, 16, 384, 16, 384, 1.0)
    # host-only: nothing runs
    refused(slora.EHIP, slora.kv8_append, b, 0, 16, 192, 16, 192)
    refused(slora.EHIP, slora.kv8_attend, b, 0, 16, 384, 16, 384, 1.0)
    refused(slora.EHIP, slora.kv8_evict, b, 0, 1, 16, 16, 16, 16)
    slora.kv8_extend(c, [0], [1])  # an older batch stays what it was
    refused(slora.EHIP, slora.kv8_append, b, 0, 16, 192, 16, 192)
    slora.kv8_truncate(c, [1], [19])
    refused(slora.EBUSY, slora.kv8_append, b, 0, 16, 192, 16, 192)
    slora.kv8_batch_destroy(b)
    slora.kv8_batch_destroy(slora.kv8_batch_plan(c, [], []))


@pytest.mark.parametrize("kw,code", [
    (dict(head_dim=48), slora.EINVAL), (dict(head_dim=128), slora.EINVAL), (dict(n_heads=7), slora.EINVAL), (dict(n_kv=0), slora.EINVAL),
    (dict(n_layers=0), slora.EINVAL), (dict(max_seqs=0), slora.EINVAL), (dict(max_tokens=0), slora.EINVAL),
    (dict(max_tokens=(1 << 27) + 1), slora.EINVAL), (dict(max_seqs=65535, max_tokens=1 << 27), slora.ERANGE)])
def test_caches_that_cannot_be(cache, kw, code):
    pool, _ = cache
    a = dict(n_layers=1, n_heads=6, n_kv=3, head_dim=64, max_seqs=4, max_tokens=100)
    a.update(kw)
    refused(code, slora.kv8_init, pool, a["n_layers"], a["n_heads"], a["n_kv"], a["head_dim"], a["max_seqs"], a["max_tokens"], None)


def test_4_bit_refusals():
    assert slora.w4_bytes(16, 128, 128) == 1024 + 16 * 3
    assert slora.w4_bytes(17, 136, 96) == 4 * 1024 + 4 * 4 * 16 * 3
    for shape in ((0, 128, 128), (16, 0, 32), (16, 12, 32), (16, 128, 16), (16, 128, 0), (16, 128, 48)):
        refused(slora.EINVAL, slora.w4_bytes, *shape)
        refused(slora.EINVAL, slora.w4_pack, *shape, slora.F16, 16, 16, None, 16)
    for args in ((2, 16, 16, None, 16), (0, None, 16, None, 16), (0, 16, None, None, 16), (0, 16, 16, None, None), (0, 16, 16, None, 24),
                 (0, 18, 16, None, 16), (0, 16, 17, None, 16)):
        refused(slora.EINVAL, slora.w4_pack, 16, 128, 32, *args)
    for call in (slora.w4_matmul, slora.w4_matmul_y16):
        refused(slora.EINVAL, call, [], [], 1, [])
        refused(slora.EINVAL, call, [None], [16], 1, [16])
        refused(slora.EINVAL, call, [None] * 9, [16] * 9, 1, list(range(16, 16 * 10, 16)))
        refused(slora.EINVAL, call, [None], [16], -1, [16])
        with pytest.raises(ValueError):
            call([None], [16, 16], 1, [16])
