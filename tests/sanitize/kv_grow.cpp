// A sequence that grows by a block at a time, as every decode step's does: its page list may not be copied each time.  With the stand-ins of kv_san.cpp.
#define main kv_san_main
#include "kv_san.cpp"
#undef main

int main()
{
    std::vector<uint16_t> mem(64 + 8);
    void *base = reinterpret_cast<void *>((reinterpret_cast<uintptr_t>(mem.data()) + 15) & ~uintptr_t(15));
    slora_pool *pool = nullptr;
    REQUIRE(slora_pool_init(&pool, 256, 40000, SLORA_F16, base, 1, 8) == SLORA_OK);
    slora_kv8 *cache = nullptr;
    REQUIRE(slora_kv8_init(&cache, pool, 2, 4, 4, 32, 2, 40000, base) == SLORA_OK);
    int64_t copied = 0;
    const int32_t seq = 1, block = cache->N;
    for (int k = 0; k < 4000; ++k) {
        const int32_t *before = cache->seqs[1].pages.data();
        const size_t held = cache->seqs[1].pages.size();
        REQUIRE(slora_kv8_extend(cache, 1, &seq, &block, nullptr, 0) == SLORA_OK);
        if (cache->seqs[1].pages.data() != before) copied += (int64_t)held;
    }
    if (copied > 2 * (int64_t)cache->seqs[1].pages.size()) {
        std::printf("kv_grow: %lld entries copied for a list of %zu\n", (long long)copied, cache->seqs[1].pages.size());
        return 1;
    }
    REQUIRE(slora_kv8_destroy(cache) == SLORA_OK);
    REQUIRE(slora_pool_destroy(pool) == SLORA_OK);
    std::puts("kv_grow OK");
    return 0;
}
