// Shared by the host side of the paged key-value cache (kv_cache.cpp) and its kernels: the records of a batch's lists
// and the launchers.  include/lora_kv.h has the contract and the layout of the pages.
#pragma once

#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "lora_kv.h"

namespace lora {

constexpr int KV_ROW_ITEM = 16;   // rows of a row item: the query side of one 16 x 16 x k product
constexpr int KV_TILE = 128;      // rows of a tile item
constexpr int KV_TURNS_TILE = 256; // ... where two groups of wavefronts take turns (attn_kernels.hip), which there is for
constexpr bool kv_turns(int dtype, int dim) { return dtype == LORA_BF16 && dim == 128; }
// How a batch's tiles are worked on (attn_kernels.hip): four wavefronts to a tile and two blocks on a compute unit, three blocks, or two groups of four wavefronts to a tile; all three
// with tiles of KV_TILE rows; two groups in turns
enum KvTiles { KV_TILES_PLAIN = LORA_KV_TILES_PLAIN, KV_TILES_MANY = LORA_KV_TILES_MANY, KV_TILES_PAIRS = LORA_KV_TILES_PAIRS, KV_TILES_TURNS = LORA_KV_TILES_TURNS };
constexpr bool kv_many(int dtype, int dim) { return dtype == LORA_BF16 && dim == 128; }
constexpr bool kv_pairs(int dtype, int dim) { return dtype == LORA_BF16 && dim == 64; }
constexpr int KV_MAX_MOVES = 128; // page copies of one launch (they travel as its arguments)
constexpr int KV_MAX_READS = 440; // pages read back by one launch (likewise)
// Pages of 8 bits: exponents are held with this added, and lie from -117 (the smallest value above 0 is normal in bf16) to 120 (of the largest fp32 values)
constexpr int KV_EXP_BIAS = 127, KV_EXP_MIN = -117, KV_EXP_MAX = 120;

// One new token: where it stands and the page it lies in.
struct KvToken {
    int32_t pos, page;
};

// Up to u new tokens (u: tokens of a chunk of values) of one sequence that share their chunks: tokens tok .. tok + n - 1 of the packed
// batch at positions pos .. pos + n - 1 of page `page`.
struct KvGroup {
    int32_t tok, pos, n, page;
};

// One piece of the attention, for every key-value head: rows row0 .. row0 + n_rows - 1 of a segment over tokens kv0 .. kv1 - 1 of its
// sequence.  Row r is query head kv_head * g + r % g of the segment's token r / g.
struct AttnItem {
    int32_t tok0;   // the segment's first token in the packed batch; of rows that share a prefix: where their tokens are listed
    int32_t ctx;    // its position; KV_SHARED, KV_EXACT: the rows of several segments, which see all the tokens
    int32_t page0;  // the sequence's first entry of the page list
    int32_t row0, n_rows;
    int32_t kv0, kv1;
    int32_t part;   // -1: writes its rows of the output; else where its partial results go, in rows: head h, row r at part + h * n_rows + r (of a
                    // tile n_rows rounded up to 32)
};

constexpr int KV_SHARED = LORA_KV_MAX_TOKENS;  // (no segment's first token stands there)
constexpr int KV_EXACT = KV_SHARED + 1;        // ... and a tile of them keeps its weights to 16 bits as row items do: some of the segments have no more rows than those

// Batches with shared prefixes: every part of what a row attends to -- prefixes, the segment's own tokens -- is a source of partial results, which lie in
// blocks of rows: row r of the source is row (row0 + r) % rows of block block0 + (row0 + r) / rows.  A join puts together rows first .. first + n_rows - 1 of its sources (KV_JOIN_ROWS at
// most), which are rows row0 + first .. of a segment.
struct SharedSource {
    int32_t row0, block0, rows, tile;  // tile: laid out as a tile's
};
struct SharedBlock {
    int32_t part, n_parts, stride, n_rows;
};
struct SharedJoin {
    int32_t tok0, row0, first, n_rows, source0, n_sources;
};
constexpr int KV_JOIN_ROWS = 16;

// Rows whose pieces are joined: n_parts pieces, `stride` rows of partial results apart.
struct JoinItem {
    int32_t tok0, row0, n_rows, part, n_parts, stride;
};

struct KvMoves {
    int32_t from[KV_MAX_MOVES], to[KV_MAX_MOVES];
};

// Lists on their way up from pinned memory: n pieces of 16 bytes
struct KvLists {
    void *to;
    const void *from;
    uint32_t n;
};

struct AppendArgs {
    const void *q, *k, *v;
    void *q_out;
    int64_t q_stride, q_out_stride, k_stride, v_stride;
    const float *rope;
    char *pages;  // of this layer
    int64_t page_stride;
    const KvToken *tokens;
    const KvGroup *groups;
    int32_t n_tokens, n_groups, n_heads, n_kv, dim, page_shift, rope_dim, neighbours;
};

// ... with norms of heads; weights may be null
struct AppendHeadsArgs {
    AppendArgs a;
    const float *q_norm, *k_norm;
    int32_t q_norm_stride, k_norm_stride;
    double eps;
};

struct ReadArgs {
    const char *pages;  // of this layer
    int64_t page_stride;
    void *k, *v;
    int64_t k_stride, v_stride;
    int32_t n_kv, dim, page_shift, n_reads;
    // read i: tokens off[i] .. of page page[i], rows row[i] .. row[i + 1] - 1
    int32_t page[KV_MAX_READS], row[KV_MAX_READS + 1];
    uint8_t off[KV_MAX_READS];
};
static_assert(sizeof(ReadArgs) <= 4096, "a kernel's arguments");

struct AttnArgs {
    const void *q;
    void *out;
    int64_t q_stride, out_stride;
    const char *pages;  // of this layer
    int64_t page_stride;
    const int32_t *page_list, *row_tokens;
    const AttnItem *tiles, *rows;
    float *part_o, *part_ml;
    float scale_log2;  // scale * log2(e)
    int32_t n_tiles, n_rows, n_short, n_kv, group, page_shift;  // n_short: items behind the n_rows that a wavefront takes alone
    bool prefixes, exact;  // some of the items are rows of several segments; some of the tiles are KV_EXACT
};

struct JoinArgs {
    void *out;
    int64_t out_stride;
    const JoinItem *items;
    const float *part_o, *part_ml;
    int32_t n_items, n_kv, group, max_rows;
};

struct SharedJoinArgs {
    void *out;
    int64_t out_stride;
    const SharedJoin *items;
    const SharedSource *sources;
    const SharedBlock *blocks;
    const float *part_o, *part_ml;
    int32_t n_items, n_kv, group, max_rows;
};

hipError_t prepare_attn_kernels();  // once for the current device
hipError_t prepare_attn_e4m3_kernels();
hipError_t launch_append(const AppendArgs &a, int dtype, hipStream_t st);
hipError_t launch_append_heads(const AppendHeadsArgs &a, int dtype, bool e4m3, hipStream_t st);
hipError_t launch_read(const ReadArgs &a, int dtype, bool e4m3, hipStream_t st);
hipError_t launch_moves(const KvMoves &m, int n, char *pages, int64_t page_stride, const KvLists &lists, hipStream_t st, hipEvent_t done);
hipError_t launch_attn(const AttnArgs &a, int dtype, int dim, KvTiles way, int n_cu, hipStream_t st);
hipError_t launch_attn_e4m3(const AttnArgs &a, int dim, KvTiles way, int n_cu, hipStream_t st);
hipError_t launch_attn_join(const JoinArgs &a, int dtype, int dim, bool tiles, hipStream_t st);

hipError_t launch_shared_join(const SharedJoinArgs &a, int dtype, int dim, hipStream_t st);

}  // namespace lora
