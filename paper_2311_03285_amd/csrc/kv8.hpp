// The 8-bit KV cache: what its host logic (kv8.cpp) and its kernels (kv8_kernels.hip) share.
#pragma once

#include "slora_internal.hpp"

namespace slora {

constexpr int kKvGranule = 8;        // tokens of a granule: 8 * D bytes of K, [token][element], then of V, [element][token]
constexpr int kKvLowest = -60;       // least exponent of a block
constexpr int kKvPoison = 127;       // exponent of a block that was given an infinity or NaN
constexpr int kKvFewCols = 16;       // columns (rows x heads that share a head of the cache) of a tile of the matrix instruction
constexpr int kKvFewThreads = 256;   // 4 wavefronts, which take turns at chunks of 32 tokens
constexpr int kKvChunk = 32;
constexpr int kKvManyTile = 64;      // tokens that a workgroup of prompts takes at a time
constexpr int kKvManyCols = 128, kKvManyThreads = 256; // columns of a workgroup of prompts: 32 for each of four wavefronts
// Columns of a sequence from which it is one.  us a pass, tiles of 16 / of 128: 24 columns of 8 sequences, 32 cached heads, behind 1000 tokens 41 / 35, 48 there 52 / 45;
// 32 columns of 32 sequences, 8 cached heads, behind 2000 48 / 57, 64 there 64 / 67: with 33 neither loses more than a sixth.
constexpr int kKvManyFrom = 33;
constexpr int kKvPartBlocks = 512;   // most blocks of a part of a sequence: their page numbers are held in LDS

// Arrays of bins that an eviction's digits are counted in.  With one barrier a turn, the wavefronts count into array a before it and read a behind it,
// and clear the array of the next turn before it: that one was last read behind the barrier before the last, so it has to be neither a nor
// the array before a, which a slow wavefront may still be reading.
constexpr int kKvBinArrays = 3;
constexpr int kv_next_bins(int a) { return a + 1 == kKvBinArrays ? 0 : a + 1; }

// a sequence of the batch
struct KvSeq {
    int32_t seq, len;  // its number, tokens it holds
    int32_t rows, row0; // query rows, the first one's number in the batch
    int32_t seen;      // positions given out
    int32_t keep;      // tokens that an eviction leaves
    int32_t move0;     // first entry of its list of moves, for head 0 (each head has min(keep, len - keep) of them)
    int32_t first0;    // first entry of its counts of moves before each block, for head 0 (blocks + 2 each)
    int64_t score0;    // first of its scores, [head][column][token] with tokens rounded up to 8; -1: more columns than have them kept
    int64_t pad;
};
static_assert(sizeof(KvSeq) == 48, "KvSeq must stay 48 bytes");

// work of one workgroup, for each head of the cache
struct KvItem {
    int32_t s;    // sequence of the batch
    int32_t a, b; // append: block, first slot in it;     attend and join: first column (row * G + head of those that share), columns
    int32_t c, d; // append: slots, first row of the batch; attend: granules [c, d);  join: parts
    int32_t poff; // attend, join: first column of the (first) part's sums in the scratch; -1: the only part, which writes its rows itself
    int32_t pad[2];
};
static_assert(sizeof(KvItem) == 32, "KvItem must stay 32 bytes");

// what the kernels know of the cache
struct KvShape {
    uint8_t *pool;
    int64_t page_bytes;
    const int32_t *table; // [sequence][block][layer][head]
    int8_t *exps;         // ... [K, V]
    int32_t n_layers, n_kv, D, G, N, max_blocks, max_tokens, layer;
    uint32_t div_b;       // ceil(2^32 / granules per block), see kv_div
};

struct KvAppend {
    const uint16_t *x[2]; // K, V
    int64_t stride[2];
};

struct KvAttend {
    const uint16_t *q;
    uint16_t *out;
    int64_t q_stride, out_stride;
    float scale;    // times log2(e)
    int32_t causal;
    float *part_o;  // averages of V of parts: [column][head][D]
    float *part_ml; // ... [column][head] {m, l}: their scores' sums l * 2^m
    float *stat;    // [row][query head] {maximum, 1 / sum}
    float *scores;  // see KvSeq; NULL: not wanted
};

struct KvWeights {
    const float *w_in;
    float *w_out;
    int32_t *pos;
};

struct KvEvict {
    const float *w_in;
    float *w_out;
    const int32_t *pos_in;
    int32_t *pos_out;
    int32_t recent;
    int32_t *src, *dst; // moves: from, to
    int32_t *first;     // moves before each block, all moves, exponents of the block about the budget
};

} // namespace slora

struct slora_kv8 {
    slora_pool *pool = nullptr;
    int32_t n_layers = 0, n_heads = 0, n_kv = 0, D = 0, max_seqs = 0, max_tokens = 0;
    int32_t N = 0, max_blocks = 0;
    int8_t *exps = nullptr;
    int32_t *d_table = nullptr;
    struct Seq {
        int32_t len = 0, seen = 0;
        int32_t on_device = 0;       // leading blocks whose pages are in the device table
        uint32_t cuts = 0;           // truncations so far
        std::vector<int32_t> pages;  // [block][layer][head]
    };
    std::vector<Seq> seqs;
    uint64_t cuts = 0;               // ... of all sequences
    int64_t live_batches = 0, pages_held = 0;
    int32_t per_block() const { return n_layers * n_kv; }
    int32_t blocks(int32_t tokens) const { return (int32_t)(((int64_t)tokens + N - 1) / N); }
};

struct slora_kv8_batch {
    slora_kv8 *cache = nullptr;
    std::vector<slora::KvSeq> seqs;
    std::vector<slora::KvItem> append, few, many, join;
    std::vector<int32_t> cuts; // of each sequence when the batch was planned
    std::vector<int32_t> columns; // sequence * max_blocks + block: pages that the first call brings into the table
    uint64_t cuts_seen = 0;
    bool has_keep = false, short_rows = false, delivered = false;
    int32_t rows = 0, longest = 0, dest_blocks = 0, join_cols = 0, join_parts = 0; // (the last two: most of a join item)
    int32_t most_going = 0; // most tokens that an eviction drops from a sequence
    int32_t longest_few = 0, longest_many = 0; // of sequences of up to kKvFewCols columns, whose scores weights are taken from, and of others
    int64_t part_cols = 0, moves = 0, firsts = 0, scores = 0; // scratch; part_cols for each head of the cache

    slora::Buffers *set = nullptr;
    slora::KvSeq *d_seqs = nullptr;
    slora::KvItem *d_append = nullptr, *d_few = nullptr, *d_many = nullptr, *d_join = nullptr;
    int32_t *d_columns = nullptr, *d_pages = nullptr;
    void *last_stream = nullptr;
    bool order_recorded = false;
    int32_t upload();
    int32_t enter(void *stream);
};

namespace slora {

// kv8_kernels.hip
int32_t launch_kv_table(const slora_kv8_batch *b, void *stream);
int32_t launch_kv_append(const slora_kv8_batch *b, const KvShape &shape, const KvAppend &a, void *stream);
int32_t launch_kv_attend(const slora_kv8_batch *b, const KvShape &shape, const KvAttend &a, void *stream);
int32_t launch_kv_weights(const slora_kv8_batch *b, const KvShape &shape, const KvAttend &a, const KvWeights &w, void *stream);
int32_t launch_kv_evict(const slora_kv8_batch *b, const KvShape &shape, const KvEvict &e, void *stream);

} // namespace slora
