// Host logic of the 8-bit KV cache: which pages a sequence's blocks lie on, and the work lists of a
// batch.  No kernels here.
#include <hip/hip_runtime_api.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "kv8.hpp"

using namespace slora;

namespace {

int32_t hip_fail(hipError_t e, const char *what) { return fail(SLORA_EHIP, "%s: %s", what, hipGetErrorString(e)); }

int32_t check_seqs(const slora_kv8 *cache, int32_t n, const int32_t *seqs)
{
    if (!cache) return fail(SLORA_EINVAL, "cache is NULL");
    if (n < 0 || n > cache->max_seqs || (n > 0 && !seqs)) return fail(SLORA_EINVAL, "n=%d sequences of a cache for %d", n, cache->max_seqs);
    std::vector<uint8_t> seen;
    try {
        seen.assign((size_t)cache->max_seqs, 0);
    } catch (const std::bad_alloc &) {
        return fail(SLORA_ENOMEM, "out of host memory");
    }
    for (int32_t i = 0; i < n; ++i) {
        if (seqs[i] < 0 || seqs[i] >= cache->max_seqs) return fail(SLORA_ERANGE, "seqs[%d]=%d outside [0, %d)", i, seqs[i], cache->max_seqs);
        if (seen[(size_t)seqs[i]]++) return fail(SLORA_EBUSY, "sequence %d is listed twice", seqs[i]);
    }
    return SLORA_OK;
}

void release(slora_pool *pool, int32_t page)
{
    pool->in_cache[(size_t)page] = 0;
    pool->set_state(page, kFree);
}

// Workgroups that a launch of attention is cut into, if the sequences are long enough: twice three for every compute unit.  No one number is best for all.  us of append
// and attention, from two runs, with 768, 1024, 1536, 2048, 4096 (cached heads / heads that share one):
//   24 sequences of 200 - 1500 tokens (40 / 1)  65.3  61.2  60.4  59.2  63.3      six of 15000 - 25000 (8 / 8)   58.4  57.0  58.0  60.0  69.7
//   64 of 500 - 8000 (8 / 8)                     128   126   125   125   137       12 of 5000 (8 / 4)             31.4  34.1  34.3  33.3  42.2
//   two of 90000 - 131000 (8 / 8)                 88    88    86    91   108       one of 30000 (8 / 8)           25.1  27.2  33.5  38.2  38.2
//   100 of 300 - 1600 (8 / 4)                   47.0  46.6  46.7  48.2  55.1      three of 9000 (32 / 1)         45.5  49.0  47.1  47.7  50.0
// Fewer and longer parts spare the join where few sequences are cut, more even out sequences of different lengths.
constexpr int64_t kPartTarget = 1536;
// Prompts, two workgroups of which fit a compute unit: us a pass with 256, 512, 1024 workgroups: a chunk of 512 behind 30000 983 / 741 / 743, eight of 64 behind
// 4000 147 / 134 / 151, one of 2048 98 / 98 / 118; parts of at least 128, 256, 512 tokens, a prompt of 512: 37.5 / 35.7 / 33.8.
constexpr int64_t kManyTarget = 512;
constexpr int32_t kManyLeast = 64;
// Granules, a chunk for each of the four wavefronts.  us with parts of at least 8, 16, 32, 64: one sequence of 400 tokens (32 / 1) 12.2 / 12.0 / 12.7 / 11.7, of 1500 13.8 / 14.6 / 14.1
// / 15.5, of 2000 (8 / 4) 12.9 / 14.2 / 14.0 / 15.3; four of 1000 (8 / 4) 15.0 / 13.4 / 13.7 / 15.3; 40 of 100 - 400 (8 / 1) 16.1 / 13.5 / 13.6 / 12.2; eight of four drafted tokens
// behind 600 (4 / 4) 13.8 / 12.3 / 12.5 / 12.9.  Batches that fill the card uncut lose by being cut: 32 of 700 (8 / 8) 24.0 / 24.1 / 20.0 / 19.1, 128 of 64 - 500 (8 / 4) 29.5 / 29.6 / 27.5 / 24.8.
constexpr int32_t kPartLeast = 16;

} // namespace

int32_t slora_kv8_batch::upload()
{
    slora_pool *pool = cache->pool;
    if (!pool->dev_base || seqs.empty()) return SLORA_OK;
    const size_t per = (size_t)cache->per_block();
    const size_t items = append.size() + few.size() + many.size() + join.size();
    const size_t bytes = seqs.size() * sizeof(KvSeq) + items * sizeof(KvItem) + columns.size() * (1 + per) * sizeof(int32_t);
    int32_t rc = pool->take_set(&set, bytes, bytes);
    if (rc != SLORA_OK) return rc;
    unsigned char *at = static_cast<unsigned char *>(set->h);
    auto put = [&](const auto &v) {
        if (!v.empty()) std::memcpy(at, v.data(), v.size() * sizeof(v[0]));
        at += v.size() * sizeof(v[0]);
    };
    put(seqs);
    put(append);
    put(few);
    put(many);
    put(join);
    put(columns);
    for (int32_t c : columns) {
        const auto &pages = cache->seqs[(size_t)(c / cache->max_blocks)].pages;
        std::memcpy(at, pages.data() + (size_t)(c % cache->max_blocks) * per, per * sizeof(int32_t));
        at += per * sizeof(int32_t);
    }
    d_seqs = static_cast<KvSeq *>(set->d);
    d_append = reinterpret_cast<KvItem *>(d_seqs + seqs.size());
    d_few = d_append + append.size();
    d_many = d_few + few.size();
    d_join = d_many + many.size();
    d_columns = reinterpret_cast<int32_t *>(d_join + join.size());
    d_pages = d_columns + columns.size();
    void *up = nullptr;
    rc = pool->uploads(&up);
    hipError_t e = hipSuccess;
    if (rc == SLORA_OK) {
        e = hipMemcpyAsync(set->d, set->h, bytes, hipMemcpyHostToDevice, (hipStream_t)up);
        if (e == hipSuccess) e = hipEventRecord((hipEvent_t)set->order, (hipStream_t)up);
        if (e != hipSuccess) rc = hip_fail(e, "uploading the batch's lists");
    }
    last_stream = up;
    order_recorded = rc == SLORA_OK;
    return rc;
}

// Every call of the batch runs after its lists have arrived and after its earlier calls.
int32_t slora_kv8_batch::enter(void *stream)
{
    if (stream != last_stream) {
        hipError_t e = hipSuccess;
        if (!order_recorded) e = hipEventRecord((hipEvent_t)set->order, (hipStream_t)last_stream);
        if (e == hipSuccess) e = hipStreamWaitEvent((hipStream_t)stream, (hipEvent_t)set->order, 0);
        if (e != hipSuccess) return hip_fail(e, "ordering the batch's work between two streams");
        last_stream = stream;
        order_recorded = false;
    }
    if (!delivered) {
        // On the caller's stream: an entry that is given another page is written after the work of earlier batches, which
        // the caller has ordered before this one.
        if (!columns.empty()) {
            int32_t rc = launch_kv_table(this, stream);
            if (rc != SLORA_OK) return rc;
            for (int32_t c : columns) {
                auto &q = cache->seqs[(size_t)(c / cache->max_blocks)];
                q.on_device = std::max(q.on_device, c % cache->max_blocks + 1);
            }
        }
        delivered = true;
    }
    return SLORA_OK;
}

namespace {

int32_t check_batch(const slora_kv8_batch *b, int32_t layer)
{
    if (!b) return fail(SLORA_EINVAL, "batch is NULL");
    const slora_kv8 *c = b->cache;
    if (layer < 0 || layer >= c->n_layers) return fail(SLORA_ERANGE, "layer=%d outside [0, %d)", layer, c->n_layers);
    if (b->cuts_seen != c->cuts)
        for (size_t i = 0; i < b->seqs.size(); ++i)
            if ((uint32_t)b->cuts[i] != c->seqs[(size_t)b->seqs[i].seq].cuts)
                return fail(SLORA_EBUSY, "batch is stale: sequence %d was truncated after it was planned", b->seqs[i].seq);
    if (!c->pool->dev_base) return fail(SLORA_EHIP, "pool is host-only (dev_base == NULL)");
    return SLORA_OK;
}

int32_t check_rows(const char *name, const void *p, int64_t stride, int64_t width)
{
    if (!p) return fail(SLORA_EINVAL, "%s is NULL", name);
    if (reinterpret_cast<uintptr_t>(p) & 15) return fail(SLORA_EINVAL, "%s must be 16-byte aligned", name);
    if (stride < width || stride % 8) return fail(SLORA_EINVAL, "stride %lld of %s must be a multiple of 8 and at least %lld", (long long)stride, name, (long long)width);
    return SLORA_OK;
}

KvShape shape_of(const slora_kv8 *c, int32_t layer)
{
    KvShape s{};
    s.pool = static_cast<uint8_t *>(c->pool->dev_base);
    s.page_bytes = (int64_t)c->pool->H * 2;
    s.table = c->d_table;
    s.exps = c->exps;
    s.n_layers = c->n_layers;
    s.n_kv = c->n_kv;
    s.D = c->D;
    s.G = c->n_heads / c->n_kv;
    s.N = c->N;
    s.max_blocks = c->max_blocks;
    s.max_tokens = c->max_tokens;
    s.layer = layer;
    const uint32_t b = (uint32_t)(c->N / kKvGranule);
    s.div_b = b == 1 ? 0 : (uint32_t)(((uint64_t(1) << 32) + b - 1) / b);
    return s;
}

// Lists of the batch: see KvItem
void make_lists(slora_kv8_batch *b)
{
    const slora_kv8 *c = b->cache;
    const int32_t G = c->n_heads / c->n_kv, gpb = c->N / kKvGranule;
    // Sequences of few columns are cut into parts that make up kPartTarget workgroups, those of many columns (prompts), where a workgroup has
    // more to do, kManyTarget.
    auto is_many = [&](const KvSeq &q) { return (int64_t)q.rows * G >= kKvManyFrom; };
    int64_t work[2] = {0, 0}; // granules times tiles of columns
    for (const KvSeq &q : b->seqs) {
        const int64_t cols = (int64_t)q.rows * G, each = is_many(q) ? kKvManyCols : kKvFewCols;
        work[is_many(q)] += (cols + each - 1) / each * ((q.len + kKvGranule - 1) / kKvGranule) * c->n_kv;
    }
    int64_t part[2] = {std::max<int64_t>(kPartLeast, (work[0] + kPartTarget - 1) / kPartTarget), std::max<int64_t>(kManyLeast, (work[1] + kManyTarget - 1) / kManyTarget)};
    for (int64_t &p : part) p = std::min<int64_t>(p, (int64_t)(kKvPartBlocks - 12) * gpb); // (whole chunks may add seven granules, and begin inside a block)
    for (size_t i = 0; i < b->seqs.size(); ++i) {
        const KvSeq &q = b->seqs[i];
        for (int32_t t = std::max(q.len - q.rows, 0); t < q.len;) {
            const int32_t block = t / c->N, n = std::min(q.len, (block + 1) * c->N) - t;
            b->append.push_back({(int32_t)i, block, t % c->N, n, q.row0 + t - (q.len - q.rows), -1, {0, 0}});
            t += n;
        }
        const int64_t cols = (int64_t)q.rows * G;
        const int32_t granules = (q.len + kKvGranule - 1) / kKvGranule;
        const bool many = is_many(q);
        const int32_t each = many ? kKvManyCols : kKvFewCols, chunk = (many ? kKvManyTile : kKvChunk) / kKvGranule;
        auto &list = many ? b->many : b->few;
        for (int64_t c0 = 0; c0 < cols; c0 += each) {
            const int32_t nc = (int32_t)std::min<int64_t>(each, cols - c0);
            // parts of whole chunks, all of about the same length
            const int32_t n = (int32_t)std::max<int64_t>(1, (granules + part[many] - 1) / part[many]);
            const int32_t step = ((granules + n - 1) / n + chunk - 1) / chunk * chunk;
            const int32_t parts = step ? (granules + step - 1) / step : 1;
            if (parts > 1) b->join.push_back({(int32_t)i, (int32_t)c0, nc, parts, 0, (int32_t)b->part_cols, {0, 0}});
            for (int32_t k = 0; k < parts; ++k)
                list.push_back({(int32_t)i, (int32_t)c0, nc, k * step, std::min(granules, (k + 1) * step),
                                parts > 1 ? (int32_t)(b->part_cols + (int64_t)k * nc) : -1, {0, 0}});
            if (parts > 1) {
                b->part_cols += (int64_t)parts * nc;
                b->join_cols = std::max(b->join_cols, nc);
                b->join_parts = std::max(b->join_parts, parts);
            }
        }
    }
    // the longest first; of equal ones those of later columns, which see more
    auto granules_of = [&](const KvItem &x) {
        const KvSeq &q = b->seqs[(size_t)x.s];
        return std::min(x.d, (q.len - q.rows + (x.a + x.b - 1) / G + kKvGranule) / kKvGranule) - x.c;
    };
    std::stable_sort(b->many.begin(), b->many.end(), [&](const KvItem &x, const KvItem &y) { return granules_of(x) > granules_of(y); });
}

} // namespace

extern "C" {

int32_t slora_kv8_init(slora_kv8 **out, slora_pool *pool, int32_t n_layers, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                       int32_t max_seqs, int32_t max_tokens, void *dev_exps)
{
    clear_error();
    if (!out) return fail(SLORA_EINVAL, "out is NULL");
    *out = nullptr;
    if (!pool) return fail(SLORA_EINVAL, "pool is NULL");
    if (n_layers < 1 || n_layers > 4096) return fail(SLORA_EINVAL, "n_layers=%d must be in [1, 4096]", n_layers);
    if (n_kv_heads < 1 || n_kv_heads > 4096 || n_heads < n_kv_heads || n_heads > 65536 || n_heads % n_kv_heads)
        return fail(SLORA_EINVAL, "n_heads=%d must be a multiple of n_kv_heads=%d, which is in [1, 4096]", n_heads, n_kv_heads);
    if (head_dim != 32 && head_dim != 64 && head_dim != 96 && head_dim != 128 && head_dim != 192 && head_dim != 256)
        return fail(SLORA_EINVAL, "head_dim=%d must be 32, 64, 96, 128, 192 or 256", head_dim);
    if (pool->H < 8 * head_dim) return fail(SLORA_EINVAL, "a page of H=%d holds fewer than 8 tokens of head_dim=%d", pool->H, head_dim);
    if (max_seqs < 1 || max_seqs > 65535) return fail(SLORA_EINVAL, "max_seqs=%d must be in [1, 65535]", max_seqs);
    if (max_tokens < 1 || max_tokens > 1 << 27) return fail(SLORA_EINVAL, "max_tokens=%d must be in [1, 2^27]", max_tokens);
    if (pool->dev_base && !dev_exps) return fail(SLORA_EINVAL, "dev_exps is NULL");
    if (reinterpret_cast<uintptr_t>(dev_exps) & 1) return fail(SLORA_EINVAL, "dev_exps must be 2-byte aligned"); // (K's and V's are read together)
    slora_kv8 *c = new (std::nothrow) slora_kv8;
    if (!c) return fail(SLORA_ENOMEM, "out of host memory");
    c->pool = pool;
    c->n_layers = n_layers;
    c->n_heads = n_heads;
    c->n_kv = n_kv_heads;
    c->D = head_dim;
    c->max_seqs = max_seqs;
    c->max_tokens = max_tokens;
    c->N = kKvGranule * (pool->H / (kKvGranule * head_dim));
    c->max_blocks = c->blocks(max_tokens);
    c->exps = static_cast<int8_t *>(dev_exps);
    int32_t rc = SLORA_OK;
    // (columns of the table are counted in 32 bits)
    if ((int64_t)max_seqs * c->max_blocks >= int64_t(1) << 31)
        rc = fail(SLORA_ERANGE, "%d sequences of %d blocks are too many", max_seqs, c->max_blocks);
    if (rc == SLORA_OK) {
        try {
            c->seqs.resize((size_t)max_seqs);
            pool->in_cache.resize((size_t)pool->n_pages);
        } catch (const std::bad_alloc &) {
            rc = fail(SLORA_ENOMEM, "out of host memory");
        }
    }
    if (rc == SLORA_OK && pool->dev_base) {
        DeviceScope dev(pool->device);
        rc = dev.status();
        if (rc == SLORA_OK) {
            const hipError_t e = hipMalloc((void **)&c->d_table, (size_t)max_seqs * c->max_blocks * c->per_block() * sizeof(int32_t));
            if (e != hipSuccess) {
                (void)hipGetLastError();
                rc = fail(e == hipErrorOutOfMemory ? SLORA_ENOMEM : SLORA_EHIP, "hipMalloc(page table): %s", hipGetErrorString(e));
            }
        }
    }
    if (rc != SLORA_OK) {
        delete c;
        return rc;
    }
    pool->live_caches++;
    *out = c;
    return SLORA_OK;
}

int32_t slora_kv8_destroy(slora_kv8 *c)
{
    clear_error();
    if (!c) return SLORA_OK;
    if (c->live_batches) return fail(SLORA_EBUSY, "%lld batch(es) of this cache still exist", (long long)c->live_batches);
    if (c->d_table) {
        DeviceScope dev(c->pool->device);
        (void)hipDeviceSynchronize();
        (void)hipFree(c->d_table);
    }
    for (auto &q : c->seqs)
        for (int32_t p : q.pages) release(c->pool, p);
    c->pool->live_caches--;
    delete c;
    return SLORA_OK;
}

int32_t slora_kv8_info(const slora_kv8 *c, int64_t *out, int32_t n)
{
    clear_error();
    if (!c || !out || n < 0 || n > SLORA_KV8_INFO_N) return fail(SLORA_EINVAL, "bad arguments");
    const int64_t v[SLORA_KV8_INFO_N] = {c->N, c->max_blocks, c->per_block(), c->pages_held};
    for (int32_t k = 0; k < n; ++k) out[k] = v[k];
    return SLORA_OK;
}

int32_t slora_kv8_lengths(const slora_kv8 *c, int32_t n, const int32_t *seqs, int32_t *out)
{
    clear_error();
    if (!c || n < 0 || (n > 0 && (!seqs || !out))) return fail(SLORA_EINVAL, "bad arguments");
    for (int32_t i = 0; i < n; ++i)
        if (seqs[i] < 0 || seqs[i] >= c->max_seqs) return fail(SLORA_ERANGE, "seqs[%d]=%d outside [0, %d)", i, seqs[i], c->max_seqs);
    for (int32_t i = 0; i < n; ++i) out[i] = c->seqs[(size_t)seqs[i]].len;
    return SLORA_OK;
}

int32_t slora_kv8_extend(slora_kv8 *c, int32_t n, const int32_t *seqs, const int32_t *tokens, const int32_t *page_idx, int64_t n_idx)
{
    clear_error();
    int32_t rc = check_seqs(c, n, seqs);
    if (rc != SLORA_OK) return rc;
    if (n > 0 && !tokens) return fail(SLORA_EINVAL, "tokens is NULL");
    slora_pool *pool = c->pool;
    int64_t want = 0;
    for (int32_t i = 0; i < n; ++i) {
        const auto &q = c->seqs[(size_t)seqs[i]];
        if (tokens[i] < 0 || tokens[i] > c->max_tokens - q.len)
            return fail(SLORA_ERANGE, "%d more tokens for sequence %d, which holds %d of %d", tokens[i], seqs[i], q.len, c->max_tokens);
        if (tokens[i] > INT32_MAX - q.seen) return fail(SLORA_ERANGE, "sequence %d has no positions left", seqs[i]);
        want += (int64_t)(c->blocks(q.len + tokens[i]) - c->blocks(q.len)) * c->per_block();
    }
    if (page_idx ? n_idx != want : n_idx != 0) return fail(SLORA_EINVAL, "n_idx=%lld but %lld page(s) begin", (long long)n_idx, (long long)want);
    std::vector<int32_t> pages;
    try {
        pages.resize((size_t)want);
        for (int32_t i = 0; i < n; ++i) {
            auto &q = c->seqs[(size_t)seqs[i]];
            const size_t need = (size_t)c->blocks(q.len + tokens[i]) * c->per_block();
            if (need > q.pages.capacity()) q.pages.reserve(std::max(need, 2 * q.pages.capacity())); // (it grows by a block at a time)
        }
    } catch (const std::bad_alloc &) {
        return fail(SLORA_ENOMEM, "out of host memory");
    }
    if (page_idx) {
        const uint8_t kSeen = 0x80;
        int64_t i = 0;
        for (; i < want && rc == SLORA_OK; ++i) {
            const int64_t p = page_idx[i];
            if (p < 0 || p >= pool->n_pages)
                rc = fail(SLORA_ERANGE, "page_idx[%lld]=%lld outside [0, %lld)", (long long)i, (long long)p, (long long)pool->n_pages);
            else if (pool->state[(size_t)p] & kSeen)
                rc = fail(SLORA_EBUSY, "page %lld listed twice", (long long)p);
            else if (pool->state[(size_t)p] != kFree)
                rc = fail(SLORA_EBUSY, "page %lld is not free", (long long)p);
            else
                pool->state[(size_t)p] |= kSeen;
            if (rc != SLORA_OK) break;
        }
        for (int64_t k = 0; k < i; ++k) pool->state[(size_t)page_idx[k]] &= 0x7f;
        if (rc != SLORA_OK) return rc;
        for (int64_t k = 0; k < want; ++k) {
            pages[(size_t)k] = page_idx[k];
            pool->set_state(page_idx[k], kKv);
        }
    } else {
        rc = pool->take(want, kKv, pages.data());
        if (rc != SLORA_OK) return rc;
    }
    for (int32_t p : pages) pool->in_cache[(size_t)p] = 1;
    const int32_t *at = pages.data();
    for (int32_t i = 0; i < n; ++i) {
        auto &q = c->seqs[(size_t)seqs[i]];
        const int64_t m = (int64_t)(c->blocks(q.len + tokens[i]) - c->blocks(q.len)) * c->per_block();
        q.pages.insert(q.pages.end(), at, at + m);
        at += m;
        q.len += tokens[i];
        q.seen += tokens[i];
    }
    c->pages_held += want;
    return SLORA_OK;
}

int32_t slora_kv8_truncate(slora_kv8 *c, int32_t n, const int32_t *seqs, const int32_t *lengths, int32_t evicted)
{
    clear_error();
    int32_t rc = check_seqs(c, n, seqs);
    if (rc != SLORA_OK) return rc;
    if (n > 0 && !lengths) return fail(SLORA_EINVAL, "lengths is NULL");
    for (int32_t i = 0; i < n; ++i) {
        const auto &q = c->seqs[(size_t)seqs[i]];
        if (lengths[i] < 0 || lengths[i] > q.len) return fail(SLORA_ERANGE, "length %d of sequence %d, which holds %d", lengths[i], seqs[i], q.len);
    }
    for (int32_t i = 0; i < n; ++i) {
        auto &q = c->seqs[(size_t)seqs[i]];
        if (lengths[i] == q.len) continue;
        const size_t stay = (size_t)c->blocks(lengths[i]) * c->per_block();
        for (size_t k = stay; k < q.pages.size(); ++k) release(c->pool, q.pages[k]);
        c->pages_held -= (int64_t)(q.pages.size() - stay);
        q.pages.resize(stay);
        if (!evicted) q.seen -= q.len - lengths[i];
        q.len = lengths[i];
        if (q.len == 0) q.seen = 0;
        q.on_device = std::min(q.on_device, c->blocks(q.len));
        q.cuts++;
        c->cuts++;
    }
    return SLORA_OK;
}

int32_t slora_kv8_batch_plan(slora_kv8 *c, slora_kv8_batch **out, int32_t n, const int32_t *seqs, const int32_t *rows, const int32_t *keep)
{
    clear_error();
    if (!out) return fail(SLORA_EINVAL, "out is NULL");
    *out = nullptr;
    int32_t rc = check_seqs(c, n, seqs);
    if (rc != SLORA_OK) return rc;
    if (n > 0 && !rows) return fail(SLORA_EINVAL, "rows is NULL");
    int64_t total = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (rows[i] < 0) return fail(SLORA_EINVAL, "rows[%d]=%d is negative", i, rows[i]);
        if (keep && keep[i] < 0) return fail(SLORA_EINVAL, "keep[%d]=%d is negative", i, keep[i]);
        total += rows[i];
    }
    if (total * c->n_heads >= int64_t(1) << 31) return fail(SLORA_ERANGE, "%lld rows of %d heads are too many for one batch", (long long)total, c->n_heads);
    slora_kv8_batch *b = new (std::nothrow) slora_kv8_batch;
    if (!b) return fail(SLORA_ENOMEM, "out of host memory");
    b->cache = c;
    try {
        for (int32_t i = 0; i < n; ++i) {
            const auto &q = c->seqs[(size_t)seqs[i]];
            KvSeq s{};
            s.seq = seqs[i];
            s.len = q.len;
            s.rows = rows[i];
            s.row0 = b->rows;
            s.seen = q.seen;
            s.keep = keep ? std::min(keep[i], q.len) : q.len;
            b->rows += rows[i];
            b->longest = std::max(b->longest, q.len);
            b->short_rows |= rows[i] > q.len;
            if (b->moves > INT32_MAX || b->firsts > INT32_MAX) {
                delete b;
                return fail(SLORA_ERANGE, "the batch's evictions are too many");
            }
            s.move0 = (int32_t)b->moves;
            s.first0 = (int32_t)b->firsts;
            b->most_going = std::max(b->most_going, s.len - s.keep);
            if (s.keep < s.len) {
                b->moves += (int64_t)std::min(s.keep, s.len - s.keep) * c->n_kv;
                b->firsts += (int64_t)(c->blocks(s.keep) + 2) * c->n_kv;
                b->dest_blocks = std::max(b->dest_blocks, c->blocks(s.keep));
            }
            const int64_t cols = (int64_t)rows[i] * (c->n_heads / c->n_kv);
            s.score0 = cols <= kKvFewCols ? b->scores : -1;
            if (cols <= kKvFewCols) {
                b->scores += cols * c->n_kv * (((int64_t)q.len + 7) / 8 * 8);
                b->longest_few = std::max(b->longest_few, q.len);
            } else {
                b->longest_many = std::max(b->longest_many, q.len);
            }
            b->seqs.push_back(s);
            b->cuts.push_back((int32_t)q.cuts);
            for (int32_t k = q.on_device; k < c->blocks(q.len); ++k) b->columns.push_back(seqs[i] * c->max_blocks + k);
        }
        make_lists(b);
    } catch (const std::bad_alloc &) {
        delete b;
        return fail(SLORA_ENOMEM, "out of host memory");
    }
    b->has_keep = keep != nullptr;
    b->cuts_seen = c->cuts;
    // (kernels count work by 32 bits)
    const int64_t most = (int64_t)std::max({b->few.size(), b->many.size(), b->append.size(), b->join.size(), (size_t)1}) * c->n_kv;
    if (most >= int64_t(1) << 31 || b->part_cols * c->n_kv >= int64_t(1) << 31 || b->moves > INT32_MAX || b->firsts > INT32_MAX) {
        delete b;
        return fail(SLORA_ERANGE, "the batch is too large");
    }
    {
        DeviceScope dev(c->pool->device);
        rc = dev.status();
        if (rc == SLORA_OK) rc = b->upload();
        if (rc != SLORA_OK) {
            const std::string text = last_error_cstr();
            if (b->set) c->pool->give_set(b->set, b->last_stream);
            delete b;
            return fail(rc, "%s", text.c_str());
        }
    }
    c->live_batches++;
    *out = b;
    return SLORA_OK;
}

int32_t slora_kv8_batch_destroy(slora_kv8_batch *b)
{
    clear_error();
    if (!b) return SLORA_OK;
    if (b->set) {
        DeviceScope dev(b->cache->pool->device);
        b->cache->pool->give_set(b->set, b->last_stream);
    }
    b->cache->live_batches--;
    delete b;
    return SLORA_OK;
}

int32_t slora_kv8_append(slora_kv8_batch *b, int32_t layer, const void *k, int64_t k_stride, const void *v, int64_t v_stride, void *stream)
{
    clear_error();
    int32_t rc = check_batch(b, layer);
    if (rc != SLORA_OK) return rc;
    if (b->short_rows) return fail(SLORA_EINVAL, "a sequence of the batch has fewer tokens than rows");
    if (b->rows == 0) return SLORA_OK;
    const slora_kv8 *c = b->cache;
    const int64_t width = (int64_t)c->n_kv * c->D;
    if ((rc = check_rows("k", k, k_stride, width)) != SLORA_OK || (rc = check_rows("v", v, v_stride, width)) != SLORA_OK) return rc;
    DeviceScope dev(c->pool->device);
    if (dev.status() != SLORA_OK) return dev.status();
    rc = b->enter(stream);
    if (rc != SLORA_OK) return rc;
    KvAppend a{};
    a.x[0] = static_cast<const uint16_t *>(k);
    a.x[1] = static_cast<const uint16_t *>(v);
    a.stride[0] = k_stride;
    a.stride[1] = v_stride;
    return launch_kv_append(b, shape_of(c, layer), a, stream);
}

int32_t slora_kv8_attend(slora_kv8_batch *b, int32_t layer, const void *q, int64_t q_stride, void *out, int64_t out_stride, float scale,
                         int32_t causal, const float *weights_in, float *weights_out, int32_t *pos, void *stream)
{
    clear_error();
    int32_t rc = check_batch(b, layer);
    if (rc != SLORA_OK) return rc;
    const bool weights = weights_in || weights_out || pos;
    if (weights && (!weights_in || !weights_out || !pos)) return fail(SLORA_EINVAL, "weights_in, weights_out and pos go together");
    if (weights && ((reinterpret_cast<uintptr_t>(weights_in) | reinterpret_cast<uintptr_t>(weights_out) | reinterpret_cast<uintptr_t>(pos)) & 3))
        return fail(SLORA_EINVAL, "weights_in, weights_out and pos must be 4-byte aligned");
    const float by = scale * 1.44269504088896340736f; // (scores are powers of two)
    if (!std::isfinite(by)) return fail(SLORA_EINVAL, "scale must be finite, and its product with log2 e");
    const slora_kv8 *c = b->cache;
    const int64_t width = (int64_t)c->n_heads * c->D;
    if (b->rows > 0 && ((rc = check_rows("q", q, q_stride, width)) != SLORA_OK || (rc = check_rows("out", out, out_stride, width)) != SLORA_OK)) return rc;
    if (b->seqs.empty() || (b->rows == 0 && !weights)) return SLORA_OK;
    DeviceScope dev(c->pool->device);
    if (dev.status() != SLORA_OK) return dev.status();
    const size_t o_floats = (size_t)b->part_cols * c->n_kv * c->D, ml_floats = (size_t)b->part_cols * c->n_kv * 2;
    const size_t stat_floats = (size_t)b->rows * c->n_heads * 2;
    // (scores first: their rows are 32-byte aligned)
    const size_t score_floats = weights ? (size_t)b->scores : 0;
    rc = c->pool->grow_v(b->set, score_floats + o_floats + ml_floats + stat_floats, 0, stream);
    if (rc == SLORA_OK) rc = b->enter(stream);
    if (rc != SLORA_OK) return rc;
    KvAttend a{};
    a.q = static_cast<const uint16_t *>(q);
    a.out = static_cast<uint16_t *>(out);
    a.q_stride = q_stride;
    a.out_stride = out_stride;
    a.scale = by;
    a.causal = causal != 0;
    a.scores = weights ? b->set->v : nullptr;
    a.part_o = b->set->v + score_floats;
    a.part_ml = a.part_o + o_floats;
    a.stat = a.part_ml + ml_floats;
    const KvShape s = shape_of(c, layer);
    if (b->rows > 0) rc = launch_kv_attend(b, s, a, stream);
    if (rc == SLORA_OK && weights) rc = launch_kv_weights(b, s, a, {weights_in, weights_out, pos}, stream);
    return rc;
}

int32_t slora_kv8_evict(slora_kv8_batch *b, int32_t layer, int32_t recent, const float *weights_in, float *weights_out, const int32_t *pos_in,
                        int32_t *pos_out, void *stream)
{
    clear_error();
    int32_t rc = check_batch(b, layer);
    if (rc != SLORA_OK) return rc;
    if (!b->has_keep) return fail(SLORA_EINVAL, "the batch was planned without keep");
    if (recent < 0) return fail(SLORA_EINVAL, "recent=%d is negative", recent);
    if (!weights_in || !weights_out || !pos_in || !pos_out) return fail(SLORA_EINVAL, "weights and positions are needed");
    if ((reinterpret_cast<uintptr_t>(weights_in) | reinterpret_cast<uintptr_t>(weights_out) | reinterpret_cast<uintptr_t>(pos_in) |
         reinterpret_cast<uintptr_t>(pos_out)) & 3)
        return fail(SLORA_EINVAL, "weights and positions must be 4-byte aligned");
    if (b->longest == 0) return SLORA_OK;
    const slora_kv8 *c = b->cache;
    DeviceScope dev(c->pool->device);
    if (dev.status() != SLORA_OK) return dev.status();
    rc = c->pool->grow_v(b->set, (size_t)(2 * b->moves + b->firsts), 0, stream);
    if (rc == SLORA_OK) rc = b->enter(stream);
    if (rc != SLORA_OK) return rc;
    KvEvict e{};
    e.w_in = weights_in;
    e.w_out = weights_out;
    e.pos_in = pos_in;
    e.pos_out = pos_out;
    e.recent = recent;
    e.src = reinterpret_cast<int32_t *>(b->set->v);
    e.dst = e.src + b->moves;
    e.first = e.dst + b->moves;
    return launch_kv_evict(b, shape_of(c, layer), e, stream);
}

} // extern "C"
