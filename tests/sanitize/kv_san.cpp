// Host logic of the 8-bit KV cache under AddressSanitizer / UndefinedBehaviorSanitizer, on the CPU only.
//
// pool.cpp, plan.cpp and kv8.cpp are compiled unchanged.  "Device" memory is host heap, copies are memcpy, events are always complete; the
// stand-in launchers check what the kernels assume of their lists - every page number that an item can reach, that appends and
// parts cover each token once, that parts fit the table in LDS - and touch every float of scratch that the kernels would.
// A seeded random sequence of calls runs, some of which must be refused.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <set>
#include <vector>

#include "kv8.hpp"

#define REQUIRE(c)                                                                \
    do {                                                                          \
        if (!(c)) {                                                               \
            std::fprintf(stderr, "kv_san: %s failed at line %d\n", #c, __LINE__); \
            std::abort();                                                         \
        }                                                                         \
    } while (0)

static bool g_fail_malloc = false;
static long g_tables = 0, g_appends = 0, g_attends = 0, g_joins = 0, g_evicts = 0, g_many = 0;

extern "C" {
hipError_t hipGetDevice(int *d) { *d = 0; return hipSuccess; }
hipError_t hipSetDevice(int) { return hipSuccess; }
hipError_t hipDeviceSynchronize(void) { return hipSuccess; }
hipError_t hipGetLastError(void) { return hipSuccess; }
const char *hipGetErrorString(hipError_t) { return "stand-in"; }
hipError_t hipMalloc(void **p, size_t n) { *p = g_fail_malloc ? nullptr : std::malloc(n ? n : 1); return *p ? hipSuccess : hipErrorOutOfMemory; }
hipError_t hipFree(void *p) { std::free(p); return hipSuccess; }
hipError_t hipHostMalloc(void **p, size_t n, unsigned) { *p = g_fail_malloc ? nullptr : std::malloc(n ? n : 1); return *p ? hipSuccess : hipErrorOutOfMemory; }
hipError_t hipHostFree(void *p) { std::free(p); return hipSuccess; }
hipError_t hipMemcpyAsync(void *d, const void *s, size_t n, hipMemcpyKind, hipStream_t) { std::memcpy(d, s, n); return hipSuccess; }
hipError_t hipEventCreateWithFlags(hipEvent_t *e, unsigned) { *e = (hipEvent_t)std::malloc(1); return hipSuccess; }
hipError_t hipEventDestroy(hipEvent_t e) { std::free((void *)e); return hipSuccess; }
hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return hipSuccess; }
hipError_t hipEventQuery(hipEvent_t) { return hipSuccess; }
hipError_t hipEventSynchronize(hipEvent_t) { return hipSuccess; }
hipError_t hipStreamCreateWithFlags(hipStream_t *s, unsigned) { *s = (hipStream_t)std::malloc(1); return hipSuccess; }
hipError_t hipStreamDestroy(hipStream_t s) { std::free((void *)s); return hipSuccess; }
hipError_t hipStreamWaitEvent(hipStream_t, hipEvent_t, unsigned) { return hipSuccess; }
hipError_t hipStreamIsCapturing(hipStream_t, hipStreamCaptureStatus *s) { *s = hipStreamCaptureStatusNone; return hipSuccess; }
hipError_t hipPointerGetAttributes(hipPointerAttribute_t *, const void *) { return hipErrorInvalidValue; }
}

namespace slora {

// the LoRA kernels are not called here
int32_t static_scratch_address(int, void **out) { static char s[16]; *out = s; return SLORA_OK; }
int32_t launch_write_pages(slora_pool *, const int32_t *, int64_t, const void *, void *, int32_t) { std::abort(); }
int32_t launch_copy(void *, const void *, size_t, void *) { std::abort(); }
bool stream_captures(void *);
int32_t launch_clear(void *, size_t, void *) { std::abort(); }
int32_t launch_gather(slora_pool *, int64_t, int32_t, void *, void *) { std::abort(); }
int32_t launch_shrink(slora_plan *, int32_t, const MultiArgs &, void *, const Route &) { std::abort(); }
int32_t launch_expand(slora_plan *, int32_t, const MultiArgs &, void *, bool, const Route &) { std::abort(); }
int32_t launch_chain(slora_plan *, int32_t, const MultiArgs &, void *, bool, const Route &) { std::abort(); }
int32_t launch_fused(slora_plan *, int32_t, const MultiArgs &, void *, bool, const Route &) { std::abort(); }

int32_t launch_kv_table(const slora_kv8_batch *b, void *)
{
    const slora_kv8 *c = b->cache;
    for (size_t i = 0; i < b->columns.size(); ++i)
        std::memcpy(c->d_table + (int64_t)b->d_columns[i] * c->per_block(), b->d_pages + i * c->per_block(), (size_t)c->per_block() * 4);
    g_tables++;
    return SLORA_OK;
}

static void check_page(const slora_kv8 *c, const KvShape &s, int32_t seq, int32_t block, int32_t head)
{
    REQUIRE(block >= 0 && block < c->blocks(c->seqs[(size_t)seq].len));
    const int32_t p = s.table[(((int64_t)seq * s.max_blocks + block) * s.n_layers + s.layer) * s.n_kv + head];
    REQUIRE(p >= 0 && p < c->pool->n_pages && c->pool->state[(size_t)p] == kKv);
    REQUIRE(p == c->seqs[(size_t)seq].pages[((size_t)block * s.n_layers + s.layer) * s.n_kv + head]);
}

int32_t launch_kv_append(const slora_kv8_batch *b, const KvShape &s, const KvAppend &, void *)
{
    std::set<std::pair<int, int>> done; // sequence, slot
    for (size_t i = 0; i < b->append.size(); ++i) {
        const KvItem &it = b->d_append[i];
        const KvSeq &q = b->d_seqs[it.s];
        REQUIRE(it.c > 0 && it.b >= 0 && it.b + it.c <= s.N && (it.a * s.N + it.b + it.c) <= q.len);
        for (int t = 0; t < it.c; ++t) {
            const int slot = it.a * s.N + it.b + t;
            REQUIRE(done.insert({it.s, slot}).second && slot >= q.len - q.rows);
            REQUIRE(it.d + t == q.row0 + slot - (q.len - q.rows));
        }
        for (int h = 0; h < s.n_kv; ++h) check_page(b->cache, s, q.seq, it.a, h);
    }
    REQUIRE((int32_t)done.size() == b->rows);
    g_appends++;
    return SLORA_OK;
}

int32_t launch_kv_attend(const slora_kv8_batch *b, const KvShape &s, const KvAttend &a, void *)
{
    std::vector<std::vector<int>> seen(b->seqs.size()); // of each column of each sequence: granules so far, in order
    for (size_t i = 0; i < b->seqs.size(); ++i) seen[i].assign((size_t)b->seqs[i].rows * s.G, 0);
    const int gpb = s.N / kKvGranule;
    std::vector<KvItem> all(b->d_few, b->d_few + b->few.size());
    for (size_t i = 0; i < b->few.size(); ++i) REQUIRE(b->d_few[i].b <= kKvFewCols);
    all.insert(all.end(), b->d_many, b->d_many + b->many.size());
    g_many += (long)b->many.size();
    std::stable_sort(all.begin(), all.end(), [](const KvItem &x, const KvItem &y) { return x.c < y.c; });
    for (const KvItem &it : all) {
        const KvSeq &q = b->d_seqs[it.s];
        REQUIRE(it.b > 0 && it.b <= kKvManyCols && it.a >= 0 && it.a + it.b <= q.rows * s.G && it.c >= 0 && it.d >= it.c);
        if (it.d > it.c) REQUIRE((it.d - 1) / gpb - it.c / gpb + 1 <= kKvPartBlocks);
        for (int c = it.a; c < it.a + it.b; ++c) {
            REQUIRE(seen[(size_t)it.s][(size_t)c] == it.c);
            seen[(size_t)it.s][(size_t)c] = it.d;
        }
        for (int g = it.c; g < it.d; ++g)
            for (int h = 0; h < s.n_kv; ++h) check_page(b->cache, s, q.seq, g / gpb, h);
        if (it.poff >= 0) {
            for (int64_t k = (int64_t)it.poff * s.n_kv; k < (int64_t)(it.poff + it.b) * s.n_kv; ++k) {
                for (int d = 0; d < s.D; ++d) a.part_o[k * s.D + d] = 1.0f;
                a.part_ml[2 * k] = a.part_ml[2 * k + 1] = 1.0f;
            }
        }
        if (q.score0 >= 0 && a.scores)
            for (int64_t k = 0; k < (int64_t)q.rows * s.G * s.n_kv * ((q.len + 7) / 8 * 8); ++k) a.scores[q.score0 + k] = 1.0f;
    }
    for (size_t i = 0; i < b->seqs.size(); ++i)
        for (int g : seen[i]) REQUIRE(g == (b->seqs[i].len + kKvGranule - 1) / kKvGranule);
    for (size_t i = 0; i < b->join.size(); ++i) {
        const KvItem &it = b->d_join[i];
        REQUIRE(it.c > 1 && it.c <= b->join_parts && it.b <= b->join_cols);
        for (int64_t k = it.poff; k < it.poff + (int64_t)it.c * it.b; ++k)
            for (int h = 0; h < s.n_kv; ++h) REQUIRE(a.part_ml[2 * (k * s.n_kv + h)] == 1.0f);
    }
    for (int64_t k = 0; k < (int64_t)b->rows * s.n_kv * s.G * 2; ++k) a.stat[k] = 0.0f;
    g_attends++;
    g_joins += (long)b->join.size();
    return SLORA_OK;
}

int32_t launch_kv_weights(const slora_kv8_batch *b, const KvShape &, const KvAttend &a, const KvWeights &, void *)
{
    for (const KvSeq &q : b->seqs) REQUIRE(q.len <= (q.score0 >= 0 ? b->longest_few : b->longest_many) && (q.score0 < 0 || q.rows == 0 || a.scores));
    return SLORA_OK;
}

int32_t launch_kv_evict(const slora_kv8_batch *b, const KvShape &s, const KvEvict &e, void *)
{
    int64_t moves = 0, firsts = 0;
    for (size_t i = 0; i < b->seqs.size(); ++i) {
        const KvSeq &q = b->d_seqs[i];
        REQUIRE(q.keep >= 0 && q.keep <= q.len && q.len - q.keep <= b->most_going && q.len <= b->longest);
        if (q.keep == q.len) continue;
        const int64_t most = std::min(q.keep, q.len - q.keep), blocks = (q.keep + s.N - 1) / s.N;
        REQUIRE(q.move0 == moves && q.first0 == firsts && blocks <= b->dest_blocks);
        for (int64_t k = 0; k < most * s.n_kv; ++k) e.src[q.move0 + k] = e.dst[q.move0 + k] = 1;
        for (int64_t k = 0; k < (blocks + 2) * s.n_kv; ++k) e.first[q.first0 + k] = 1;
        moves += most * s.n_kv;
        firsts += (blocks + 2) * s.n_kv;
        for (int h = 0; h < s.n_kv; ++h)
            for (int k = 0; k < b->cache->blocks(q.len); ++k) check_page(b->cache, s, q.seq, k, h);
    }
    g_evicts++;
    return SLORA_OK;
}

} // namespace slora

using namespace slora;

int main(int argc, char **argv)
{
    std::mt19937 rng(argc > 1 ? (unsigned)std::atoi(argv[1]) : 1);
    auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
    for (int round = 0; round < 6; ++round) {
        const int dims[] = {32, 64, 96, 128, 192, 256}, D = dims[pick(0, 5)];
        const int H = 8 * D + 8 * pick(0, 3 * D), kv = pick(1, 3), G = pick(1, 9), layers = pick(1, 2), seqs = pick(1, 6), most = pick(1, 9000);
        const int64_t n_pages = 60000;
        std::vector<uint16_t> mem(64 + 8); // the stand-in launchers do not touch pages
        void *base = reinterpret_cast<void *>((reinterpret_cast<uintptr_t>(mem.data()) + 15) & ~uintptr_t(15));
        slora_pool *pool = nullptr;
        REQUIRE(slora_pool_init(&pool, H, n_pages, round % 2, base, 1, 8) == SLORA_OK);
        slora_kv8 *cache = nullptr;
        g_fail_malloc = true;
        REQUIRE(slora_kv8_init(&cache, pool, layers, kv * G, kv, D, seqs, most, base) == SLORA_ENOMEM && !cache);
        g_fail_malloc = false;
        REQUIRE(slora_kv8_init(&cache, pool, layers, kv * G, kv, D, seqs, most, base) == SLORA_OK);
        std::vector<slora_kv8_batch *> old;
        for (int step = 0; step < 40; ++step) {
            std::vector<int32_t> ids, tokens, rows, keep, len((size_t)seqs);
            for (int s = 0; s < seqs; ++s)
                if (pick(0, 2)) ids.push_back(s);
            std::shuffle(ids.begin(), ids.end(), rng);
            len.resize(ids.size() + 1);
            REQUIRE(slora_kv8_lengths(cache, (int32_t)ids.size(), ids.data(), len.data()) == SLORA_OK);
            for (size_t i = 0; i < ids.size(); ++i) {
                const int room = most - len[i];
                tokens.push_back(std::min(room, pick(0, 3) ? pick(0, 3) : pick(0, 2500)));
            }
            const int32_t rc = slora_kv8_extend(cache, (int32_t)ids.size(), ids.data(), tokens.data(), nullptr, 0);
            REQUIRE(rc == SLORA_OK || rc == SLORA_ENOMEM);
            for (size_t i = 0; i < ids.size(); ++i) {
                rows.push_back(rc == SLORA_OK ? std::min(tokens[i], 600) : 0);
                keep.push_back(pick(0, most));
            }
            slora_kv8_batch *b = nullptr;
            REQUIRE(slora_kv8_batch_plan(cache, &b, (int32_t)ids.size(), ids.data(), rows.data(), pick(0, 1) ? keep.data() : nullptr) == SLORA_OK);
            void *streams[2] = {nullptr, reinterpret_cast<void *>(8)};
            alignas(16) static char row[16];
            const int64_t wide = (int64_t)kv * G * D;
            const int layer = pick(0, layers - 1);
            float *w = reinterpret_cast<float *>(row);
            int32_t *pos = reinterpret_cast<int32_t *>(row);
            REQUIRE(slora_kv8_append(b, layer, row, wide, row, wide, streams[pick(0, 1)]) == SLORA_OK);
            REQUIRE(slora_kv8_attend(b, layer, row, wide, row, wide, 1.0f, 1, pick(0, 1) ? w : nullptr, nullptr, nullptr, nullptr) != SLORA_OK || true);
            REQUIRE(slora_kv8_attend(b, layer, row, wide, row, wide, 1.0f, pick(0, 1), w, w, pos, streams[pick(0, 1)]) == SLORA_OK);
            REQUIRE(slora_kv8_attend(b, layer, row, wide, row, wide, 1.0f, 1, nullptr, nullptr, nullptr, streams[0]) == SLORA_OK);
            REQUIRE(slora_kv8_attend(b, layer, row, wide - 8, row, wide, 1.0f, 1, nullptr, nullptr, nullptr, nullptr) == (b->rows ? SLORA_EINVAL : SLORA_OK));
            const int32_t ev = slora_kv8_evict(b, layer, pick(0, 50), w, w, pos, pos, streams[0]);
            REQUIRE(ev == (b->has_keep ? SLORA_OK : SLORA_EINVAL));
            if (pick(0, 1) && !ids.empty()) {
                std::vector<int32_t> cut;
                REQUIRE(slora_kv8_lengths(cache, (int32_t)ids.size(), ids.data(), len.data()) == SLORA_OK);
                for (size_t i = 0; i < ids.size(); ++i) cut.push_back(pick(0, 3) ? pick(0, len[i]) : len[i]);
                REQUIRE(slora_kv8_truncate(cache, (int32_t)ids.size(), ids.data(), cut.data(), pick(0, 1)) == SLORA_OK);
                bool changed = false;
                for (size_t i = 0; i < ids.size(); ++i) changed |= cut[i] != len[i];
                REQUIRE(slora_kv8_append(b, layer, row, wide, row, wide, nullptr) == (changed ? SLORA_EBUSY : SLORA_OK));
            }
            old.push_back(b);
            if (pick(0, 1)) {
                REQUIRE(slora_kv8_batch_destroy(old.front()) == SLORA_OK);
                old.erase(old.begin());
            }
        }
        REQUIRE(old.empty() || slora_kv8_destroy(cache) == SLORA_EBUSY);
        for (slora_kv8_batch *b : old) REQUIRE(slora_kv8_batch_destroy(b) == SLORA_OK);
        REQUIRE(slora_pool_destroy(pool) == SLORA_EBUSY);
        REQUIRE(slora_kv8_destroy(cache) == SLORA_OK);
        int64_t free_pages = 0;
        REQUIRE(slora_pool_free_pages(pool, &free_pages) == SLORA_OK && free_pages == n_pages);
        REQUIRE(slora_pool_destroy(pool) == SLORA_OK);
    }
    REQUIRE(g_tables && g_appends && g_attends && g_joins && g_evicts && g_many);
    std::puts("kv_san OK");
    return 0;
}
