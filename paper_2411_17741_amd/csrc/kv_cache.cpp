// Host side of the paged key-value cache: sequences and their pages, batches and how their attention is cut up.
// include/lora_kv.h has the contract; the kernels are in kv_kernels.hip and attn_kernels.hip.
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <cstring>
#include <mutex>
#include <new>
#include <unordered_map>
#include <vector>

#include "kv_internal.h"
#include "lora_internal.h"

namespace {

#define KV_TRY(expr)                           \
    do {                                       \
        hipError_t e_ = (expr);                \
        if (e_ != hipSuccess) {                \
            (void)hipGetLastError();           \
            lora::set_last_hip((int)e_);       \
            return LORA_E_HIP;                 \
        }                                      \
    } while (0)

constexpr size_t ALIGN = 256;
constexpr size_t align_up(size_t n) { return (n + ALIGN - 1) / ALIGN * ALIGN; }

// Memory for partial results of attention over parts of a cache.  A batch whose pieces would need more is cut into fewer.
constexpr size_t PART_BYTES = (size_t)64 << 20;
// Lists of a batch that was destroyed may still be on their way up: that many more of them than batches alive.
constexpr int SPARE_BATCHES = 2;
// The attention over long caches with few rows is cut along the cache until about so many blocks have work, in pieces of no fewer tokens.
constexpr int ROW_BLOCKS = 512, ROW_MIN_TOKENS = 512;
// Tokens times head_dim up to which a wavefront may have an item to itself.
constexpr int ROW_SHORT_VALUES = 16384;
// ... in pages of 8 bits.  Heads of 128, 16384 -> this: 512 requests of about 100 tokens with 32 / 8 heads 39.9 -> 37.8 us, 128 of 120 19.0 -> 17.8, 256 of 400 56.2 -> 55.2; but 512 of 600 135 -> 138.
constexpr int ROW_SHORT_E4M3 = 32768;
// Tiles are cut into pieces of no fewer tokens than join work is worth -- fp32 products take 8 times as long --, or of half of that where there are few tiles.  Measured for fp32, 512 -> these:
// prompts of 300, 1 and 77 tokens with 32 / 8 heads of 128, append and attention of two layers, 111 -> 76 us, with 6 / 2 108 -> 56, with 32 / 8 heads of 64 65 -> 56.
constexpr int tile_min_tokens(const lora_kv_config_t &c) { return c.dtype == LORA_BF16 ? 512 : c.head_dim == 64 ? 256 : 128; }
constexpr int PIECE_STEP = 64;  // pieces begin at multiples of it: a whole number of every kernel's steps, in one page or at the start of one
constexpr int MAX_EXTRA = 2048;  // pieces beyond one for each block of rows
// Of how many prefixes of prefixes a segment may have a part; tokens' places in all of them together (times max_batch_tokens); tokens of a piece of a prefix with few rows
constexpr int SHARED_DEPTH = 7, SHARED_TOKENS = 2, SHARED_ROW_MIN_TOKENS = 256;
// Behind how many prefixes without room, one behind the other, fewer segments are still looked for that share more: 2000 requests, each a fork of the one before it, would otherwise take 23 ms.
constexpr int SHARED_MISSES = 16;
// A prefix is worth it if the segments but one are spared more bytes of keys and values than these, and so many for each row of each head of 128, whose parts are written and read again.  (The bytes
// that are spared would mostly have come out of caches.)  Measured, one by one -> shared, us, heads of 128, each request 100 tokens of its own behind the prefix, with a deviation of the logarithm of 0.4 (in
// brackets: 100 for all): 64 requests with 32 / 8 heads and 600 tokens, 148 MB, 27.9 -> 20.0 (19.3 -> 20.1), 1024 tokens 35.4 -> 24.9 (26.1 -> 24.9), 512 tokens, 132 MB, 25.1 -> 23.2 (17.3 -> 23.4); with 64 / 8 heads 800
// tokens 33.2 -> 23.6 (23.4 -> 23.4), 640 29.2 -> 21.5 (19.8 -> 21.6).  256 requests with 32 / 8 heads and 256 tokens, 267 MB, 41.8 -> 35.4, 128 tokens 35.5 -> 36.7; 20 of 1800, 140 MB, 22.1 -> 20.0, 1500 20.1 -> 21.0; 5 of
// 8000 28.1 -> 23.1, 5000 21.0 -> 21.7; 60 with 40 / 40 and 200 46.4 -> 35.9.  In 8 bits 64 with 32 / 8 and 2000 31.6 -> 26.2, 1500 25.9 -> 26.1, 1024 20.9 -> 25.6.  Of few rows: 2 requests with 40 / 40 heads and 1024
// tokens, 21 MB, 14.2 -> 13.0, 512 tokens 12.5 -> 12.5.  The rule counts bytes alone, and not the pieces that either way cuts: it loses with 64 requests and 512 or 640 tokens of lengths that differ, with 128 of 320
// (25.5 -> 22.3) and with 20 of 300 with 40 / 40 heads (25.0 -> 20.9).
constexpr int64_t SHARED_FEW_BYTES = 16 << 20, SHARED_BYTES = 112 << 20, SHARED_ROW_BYTES = 14 << 10;
// Few blocks are as fast as the compute unit that has most of them: a block takes its tokens and EVEN_BLOCK more, and of rows each over two for a compute unit waits, EVEN_WAIT.  Pieces of an even share of all
// tokens -> so cut, us.  Rows in 8 bits: 4 tokens of 30000 with 64 / 8 heads of 128 57.3 -> 49.9 (544 blocks, 512), 3 of about 50000 80 -> 70, 20 of 4000 with 32 / 8 38.4 -> 35.0, one of 131071 with 64 / 8
// 56.2 -> 54.2; 2 of 1500 with 40 / 40 17.2 -> 17.8.  Tiles in 8 bits: 128 tokens behind 20000 with 32 / 8 72 -> 63.6, 500 behind 2000 with 40 / 40 54 -> 45, 256 behind 5000 with 16 / 4 heads of 256 69 -> 48,
// 1500 44 -> 41.  Prefixes: 4 requests behind 9000 tokens with 32 / 8 heads 20.3 -> 15.9, 8 behind 1500 with 40 / 40 16.5 -> 14.1 (without EVEN_WAIT 16.9), 10 behind 1200 with 32 / 32 15.4 -> 15.3; in tiles, 200 behind
// 20000 with 40 / 40 332 -> 271, 16 behind 40000 with 48 / 6 56 -> 52, 30 behind 30000 with 32 / 8 heads of 256 110 -> 89; tiles beside them,
// 3 x 180 and 20 tokens behind 4000 with 32 / 8 74 -> 64, 2 x 100 and 8 behind 6000 55 -> 44; 30 tokens, 40, 7 and 150 behind 2000 30.1 -> 29.3.  (Pages that are not of 8 bits, and share nothing, are cut as they always were.)
constexpr int64_t EVEN_ROUNDS = 4, EVEN_BLOCK = 128, EVEN_WAIT = 3;

struct Seq {
    int64_t id = 0;
    int32_t n_tokens = 0;
    bool alive = false;
    std::vector<int32_t> pages;
};

// A batch's lists, of which a cache has n_batches and a few; `name` is what the caller holds of a batch, 0 if the lists are nobody's.
struct Batch {
    uint64_t name = 0;
    bool stale = false, upload_pending = false;
    int64_t freed_at = 0;  // order in which lists became free
    char *dev = nullptr, *pinned = nullptr;
    const char *pinned_dev = nullptr;
    hipEvent_t uploaded = nullptr;
    lora_kv_batch_info_t info{};
    int32_t max_pos = -1;  // of the batch's tokens
    bool exact = false;    // some of its tiles are KV_EXACT
    int32_t n_joins = 0, n_tile_joins = 0, join_rows = 0;  // join_rows: the most rows of a join of row items
    int32_t n_shared_joins = 0, shared_rows = 0;  // segments with prefixes; the most rows of one
    lora_kv_prefix_info_t prefixes{};
    size_t off_row_tokens = 0, off_sources = 0, off_blocks = 0, off_shared_joins = 0;
    size_t off_tokens = 0, off_groups = 0, off_pages = 0, off_rows = 0, off_tiles = 0, off_joins = 0, off_tile_joins = 0;
    std::vector<uint8_t> member;  // by sequence slot
    bool alive() const { return name != 0; }
};

// Batches are known by numbers that are given once in the life of the process: which lists of their cache, below, and a count.  So a batch that was destroyed, or is another
// cache's, is never taken for one that is alive.  The lock guards the count, the list of caches and the names and infos of their batches for lora_kv_batch_info, which is told
// no cache.
constexpr int NAME_BITS = 11;
std::mutex g_lock;
uint64_t g_names = 0;
lora_kv *g_caches = nullptr;

}  // namespace

struct lora_kv {
    lora_kv_config_t cfg{};
    bool host_only = false;
    char *pages = nullptr, *work = nullptr;
    size_t layer_bytes = 0, page_bytes = 0, list_cap = 0;
    float *part_o = nullptr, *part_ml = nullptr;
    int64_t part_rows = 0;
    int page_shift = 0, n_cu = 256, device = 0;

    std::vector<Seq> seqs;
    std::vector<int32_t> free_seqs;
    std::unordered_map<int64_t, int32_t> slot_of;
    std::vector<int32_t> refs;     // holders of a page
    std::vector<uint64_t> free_bits;
    int32_t limit = 0, free_pages = 0, used_pages = 0;
    size_t free_from = 0;  // no free page in the words before this one
    int64_t copied = 0;
    std::vector<uint32_t> seen;  // by sequence slot: the call that named it last
    uint32_t call = 0;

    std::vector<Batch> batches;
    lora_kv *next = nullptr, *before = nullptr;  // in g_caches
    int64_t tick = 0;
    int32_t alive_batches = 0;

    bool any_stream = false;
    hipStream_t last = nullptr;
    hipEvent_t order_ev = nullptr;

    bool e4m3() const { return cfg.flags & LORA_KV_PAGES_E4M3; }
    int row_chunk() const { return cfg.dtype == LORA_BF16 ? 8 : 4; }  // values of 16 bytes: of queries, keys, values and outputs,
    int chunk() const { return e4m3() ? 16 : row_chunk(); }          // ... and of the pages
    int group() const { return cfg.n_heads / cfg.n_kv_heads; }
    bool page_free(int32_t p) const { return (free_bits[(size_t)p >> 6] >> (p & 63)) & 1; }
    void give_back(int32_t p)
    {
        if (--refs[p]) return;
        --used_pages;
        ++free_pages;  // (a page in use lies below the limit)
        free_bits[(size_t)p >> 6] |= (uint64_t)1 << (p & 63);
        free_from = std::min(free_from, (size_t)p >> 6);
    }
    int32_t take()  // the free page with the lowest number; there is one
    {
        while (!free_bits[free_from]) ++free_from;
        const int32_t p = (int32_t)(free_from * 64 + __builtin_ctzll(free_bits[free_from]));
        free_bits[free_from] &= free_bits[free_from] - 1;
        refs[p] = 1;
        --free_pages;
        ++used_pages;
        return p;
    }
    Seq *find(int64_t id)
    {
        const auto it = slot_of.find(id);
        return it == slot_of.end() ? nullptr : &seqs[it->second];
    }
    int32_t slot(const Seq &s) const { return (int32_t)(&s - seqs.data()); }
    void next_call()
    {
        if (++call == 0) {
            std::fill(seen.begin(), seen.end(), 0u);
            call = 1;
        }
    }
    bool first_time(const Seq &s)  // in this call
    {
        uint32_t &c = seen[slot(s)];
        if (c == call) return false;
        c = call;
        return true;
    }
    void drop_batches_with(const Seq &s)
    {
        for (auto &b : batches)
            if (b.alive() && b.member[slot(s)]) b.stale = true;
    }
};

namespace {

using lora::AttnItem;
using lora::JoinItem;
using lora::KvGroup;
using lora::KvToken;
using lora::SharedBlock;
using lora::SharedJoin;
using lora::SharedSource;

static_assert(1024 + SPARE_BATCHES <= 1 << NAME_BITS, "the most batches of a cache");

Batch *find_batch(lora_kv &kv, const lora_kv_batch_t *handle)
{
    const uint64_t name = reinterpret_cast<uintptr_t>(handle), at = name & ((1 << NAME_BITS) - 1);
    return name && at < kv.batches.size() && kv.batches[at].name == name ? &kv.batches[at] : nullptr;
}

size_t elem_bytes(int32_t dtype) { return dtype == LORA_BF16 ? 2 : 4; }

constexpr size_t MAX_PAGE_BYTES = ((size_t)1 << 32) - 1;  // the kernels multiply a page's number by 32 bits

size_t layer_bytes(const lora_kv_config_t &c)
{
    const size_t rows = (size_t)2 * c.n_kv_heads * c.page_tokens;
    return c.flags & LORA_KV_PAGES_E4M3 ? rows * (c.head_dim + 1) : rows * c.head_dim * elem_bytes(c.dtype);
}

bool good(const lora_kv_config_t *c)
{
    if (!c || c->n_layers < 1 || c->n_kv_heads < 1 || c->n_heads < c->n_kv_heads || c->n_heads % c->n_kv_heads) return false;
    if (c->head_dim != 64 && c->head_dim != 128 && c->head_dim != 256) return false;
    if (c->page_tokens != 32 && c->page_tokens != 64 && c->page_tokens != 128 && c->page_tokens != 256) return false;
    if (c->n_pages < 1 || c->max_seqs < 1 || c->max_batch_seqs < 1 || c->max_batch_tokens < 1 || c->max_batch_pages < 1 || c->n_batches < 1)
        return false;
    if ((int64_t)c->max_batch_tokens * (c->n_heads / c->n_kv_heads) > LORA_KV_MAX_TOKENS) return false;
    if (c->n_heads > 4096 || c->n_layers > 65536 || c->n_batches > 1024 || c->max_batch_tokens > LORA_KV_MAX_TOKENS) return false;
    if ((c->dtype != LORA_BF16 && c->dtype != LORA_F32) || (c->flags & ~(LORA_KV_HOST_ONLY | LORA_KV_PAGES_E4M3))) return false;
    if ((c->flags & LORA_KV_PAGES_E4M3) && c->dtype != LORA_BF16) return false;
    return layer_bytes(*c) <= MAX_PAGE_BYTES / (size_t)c->n_layers;
}

int64_t max_items(const lora_kv_config_t &c)
{
    const int64_t g = c.n_heads / c.n_kv_heads;
    return (int64_t)c.max_batch_tokens * g / lora::KV_TILE + c.max_batch_seqs + MAX_EXTRA;
}

// Of segments with prefixes, fewer rows than a tile's each, and of blocks that are cut beside them
int64_t max_shared_joins(const lora_kv_config_t &c)
{
    const int64_t g = c.n_heads / c.n_kv_heads;
    return (int64_t)c.max_batch_tokens * g / lora::KV_JOIN_ROWS + c.max_batch_seqs + MAX_EXTRA;
}

size_t list_bytes(const lora_kv_config_t &c)
{
    const size_t T = c.max_batch_tokens;
    return align_up(T * sizeof(KvToken)) + align_up(T * sizeof(KvGroup)) + align_up((size_t)c.max_batch_pages * 4) +
           align_up((size_t)max_items(c) * sizeof(AttnItem)) + align_up((size_t)MAX_EXTRA * sizeof(JoinItem)) + 3 * ALIGN +
           align_up(T * SHARED_TOKENS * 4) + align_up((size_t)max_items(c) * sizeof(SharedBlock)) + align_up(((size_t)c.max_batch_seqs * (SHARED_DEPTH + 1) + MAX_EXTRA) * sizeof(SharedSource)) +
           align_up((size_t)max_shared_joins(c) * sizeof(SharedJoin));
}

// The cache's device is the current one as long as this lives: events, the default stream and kernels are the current device's.
class OnDevice {
    int back_ = -1;

public:
    explicit OnDevice(const lora_kv &kv)
    {
        int now = 0;
        if (!kv.host_only && hipGetDevice(&now) == hipSuccess && now != kv.device && hipSetDevice(kv.device) == hipSuccess) back_ = now;
    }
    ~OnDevice()
    {
        if (back_ >= 0) (void)hipSetDevice(back_);
    }
    OnDevice(const OnDevice &) = delete;
};

// Work of a call on a stream waits for the work of the one before it on another; asked for before a call changes anything.  Nothing can wait for a stream that is
// being captured without becoming part of the capture, so calls on others are refused meanwhile.
int in_order(lora_kv &kv, hipStream_t st)
{
    if (kv.any_stream && kv.last == st) return LORA_OK;
    hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
    KV_TRY(hipStreamIsCapturing(st, &cs));
    if (cs != hipStreamCaptureStatusNone) return LORA_OK;  // the caller's to order
    if (kv.any_stream) {
        KV_TRY(hipStreamIsCapturing(kv.last, &cs));
        if (cs != hipStreamCaptureStatusNone) return LORA_E_STATE;
        KV_TRY(hipEventRecord(kv.order_ev, kv.last));
        KV_TRY(hipStreamWaitEvent(st, kv.order_ev, 0));
    }
    kv.last = st;
    kv.any_stream = true;
    return LORA_OK;
}

int refuse_capture(hipStream_t st)
{
    hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
    KV_TRY(hipStreamIsCapturing(st, &cs));
    return cs == hipStreamCaptureStatusNone ? LORA_OK : LORA_E_STATE;
}

// Copies pages; `lists` (16-byte pieces, n may be 0) go up with the last of the launches, or in one of their own, which `done` is recorded with.
int copy_pages(lora_kv &kv, const std::vector<int32_t> &from, const std::vector<int32_t> &to, hipStream_t st, const lora::KvLists &lists = {}, hipEvent_t done = nullptr)
{
    for (size_t at = 0; at < from.size(); at += lora::KV_MAX_MOVES) {
        lora::KvMoves m;
        const int n = (int)std::min(from.size() - at, (size_t)lora::KV_MAX_MOVES);
        std::copy_n(from.begin() + at, n, m.from);
        std::copy_n(to.begin() + at, n, m.to);
        const bool last = at + n == from.size();
        KV_TRY(lora::launch_moves(m, n, kv.pages, (int64_t)kv.page_bytes, last ? lists : lora::KvLists{}, st, last ? done : nullptr));
    }
    if (from.empty()) KV_TRY(lora::launch_upload(lists.to, lists.from, (size_t)lists.n * 16, st, done));
    return LORA_OK;
}

// Sequences that get tokens in one call: found, checked, the pages they will need counted; nothing is changed.
struct Growth {
    std::vector<Seq *> seqs;
    std::vector<int32_t> n_tokens;
    std::vector<int32_t> from, to;  // page copies, filled by grow()
};

int check_growth(lora_kv &kv, int32_t n, const int64_t *ids, const int32_t *counts, const int32_t *offsets, Growth &g)
{
    g.seqs.resize(n);
    g.n_tokens.resize(n);
    std::unordered_map<int32_t, int32_t> leaving;  // holders of a shared page that will have a copy
    int64_t need = 0;
    kv.next_call();
    for (int32_t i = 0; i < n; ++i) {
        Seq *s = kv.find(ids[i]);
        if (!s) return LORA_E_NOTFOUND;
        if (!kv.first_time(*s)) return LORA_E_INVAL;
        const int64_t add = counts ? counts[i] : (int64_t)offsets[i + 1] - offsets[i];
        if (add < 0) return LORA_E_INVAL;
        if (s->n_tokens + add > LORA_KV_MAX_TOKENS) return LORA_E_NOMEM;
        g.seqs[i] = s;
        g.n_tokens[i] = (int32_t)add;
        need += ((s->n_tokens + add + kv.cfg.page_tokens - 1) >> kv.page_shift) - (int64_t)s->pages.size();
        if (add && (s->n_tokens & (kv.cfg.page_tokens - 1))) {
            const int32_t p = s->pages.back();
            if (kv.refs[p] > 1) {
                int32_t &l = leaving[p];
                if (kv.refs[p] - l > 1) {
                    ++l;
                    ++need;
                }
            }
        }
    }
    return need > kv.free_pages ? LORA_E_NOMEM : LORA_OK;
}

void grow(lora_kv &kv, Growth &g)
{
    for (size_t i = 0; i < g.seqs.size(); ++i) {
        Seq &s = *g.seqs[i];
        if (!g.n_tokens[i]) continue;
        if ((s.n_tokens & (kv.cfg.page_tokens - 1)) && kv.refs[s.pages.back()] > 1) {
            kv.drop_batches_with(s);  // they name the page that is left to the others
            const int32_t old = s.pages.back();
            s.pages.back() = kv.take();
            kv.give_back(old);
            g.from.push_back(old);
            g.to.push_back(s.pages.back());
            ++kv.copied;
        }
        s.n_tokens += g.n_tokens[i];
        const size_t want = ((size_t)s.n_tokens + kv.cfg.page_tokens - 1) >> kv.page_shift;
        while (s.pages.size() < want) s.pages.push_back(kv.take());
    }
}

// Room that grow() will need, taken before anything is changed (it must not run out of host memory midway).
void reserve(const lora_kv &kv, Growth &g)
{
    for (size_t i = 0; i < g.seqs.size(); ++i) {
        std::vector<int32_t> &p = g.seqs[i]->pages;
        const size_t want = ((size_t)g.seqs[i]->n_tokens + g.n_tokens[i] + kv.cfg.page_tokens - 1) >> kv.page_shift;
        if (want > p.capacity()) p.reserve(std::max(want, 2 * p.size()));
    }
    g.from.reserve(g.seqs.size());
    g.to.reserve(g.seqs.size());
}

// A prefix: entries [from, to) of the page lists of its segments, which they have in common, and as many rows as the segments have together.
struct Prefix {
    int32_t from, to;
    std::vector<int32_t> segs;
    int64_t rows;
    bool exact;  // tiles of it keep weights to 16 bits
};

// How the attention of a batch is cut up.
struct Cut {
    std::vector<Prefix> prefixes;
    std::vector<int32_t> own;  // by segment: the pages that are its prefixes' (empty: none has one)
    std::vector<int32_t> row_tokens;
    std::vector<SharedSource> sources;
    std::vector<SharedBlock> blocks;
    std::vector<SharedJoin> shared_joins;
    bool exact = false;  // some of the prefixes' tiles are KV_EXACT
    int32_t prefix_row_items = 0, prefix_tile_items = 0, prefix_segments = 0;
    int32_t extra_joins = 0;  // blocks that share nothing and are joined with the others
    lora::KvTiles way = lora::KV_TILES_PLAIN;
    int32_t n_short = 0;  // of the rows' items, at the list's end
    std::vector<AttnItem> rows, tiles;
    std::vector<JoinItem> joins, tile_joins;
    std::vector<int32_t> page0;  // by segment
};

// A block of rows over tokens [0, kv_len), in pieces of at most `piece` tokens and about the same length
void cut_block(AttnItem base, int32_t kv_len, int32_t piece, int32_t rows, int32_t n_kv, std::vector<AttnItem> &items, std::vector<JoinItem> &joins, int64_t &part)
{
    int32_t n = (kv_len + piece - 1) / piece;
    base.part = -1;
    if (n <= 1) {
        base.kv0 = 0;
        base.kv1 = kv_len;
        items.push_back(base);
        return;
    }
    const int32_t each = ((kv_len + n - 1) / n + PIECE_STEP - 1) / PIECE_STEP * PIECE_STEP, stride = rows * n_kv;  // stride: partial results of a piece
    n = (kv_len + each - 1) / each;
    joins.push_back({base.tok0, base.row0, base.n_rows, (int32_t)part, n, stride});
    for (int32_t i = 0; i < n; ++i) {
        base.kv0 = i * each;
        base.kv1 = std::min(kv_len, (i + 1) * each);
        base.part = (int32_t)part;
        part += stride;
        items.push_back(base);
    }
}

// How many pieces of at most `piece` tokens the cuts here make of `tokens`
int64_t pieces_of(int64_t tokens, int64_t piece)
{
    const int64_t n = std::max((tokens + piece - 1) / piece, (int64_t)1), each = ((tokens + n - 1) / n + PIECE_STEP - 1) / PIECE_STEP * PIECE_STEP;
    return n == 1 ? 1 : (tokens + each - 1) / each;
}

// `piece`, or up to twice as much where compute units then have their blocks more evenly.  blocks(piece): blocks of a piece each, and all of them with those beside.
template <typename F>
int64_t even_piece(int64_t piece, int64_t n_cu, F blocks)
{
    int64_t best = piece, least = INT64_MAX;
    for (int64_t p = piece; p <= 2 * piece; p += std::max(piece / 16 / PIECE_STEP, (int64_t)1) * PIECE_STEP) {
        const auto [n, all] = blocks(p);
        if (p == piece && n > EVEN_ROUNDS * n_cu) break;
        const int64_t time = (n + n_cu - 1) / n_cu * (p + EVEN_BLOCK) + std::max(all - 2 * n_cu, (int64_t)0) * EVEN_WAIT;
        if (time < least) least = time, best = p;
    }
    return best;
}

// What segments of few rows have in common.  Larger ones fill tiles of their own: the products take as long, and there is nothing to join.  (Called before the
// sequences grow: pages that are full by then stay as they are.)
void find_prefixes(const lora_kv &kv, const Growth &g, int32_t min_tokens, Cut &cut)
{
    const int32_t grp = kv.group();
    const int64_t token_bytes = (int64_t)(kv.layer_bytes / kv.cfg.page_tokens);  // keys and values
    const auto worth = [&](int64_t shared, int64_t segs, int64_t rows) {
        if (min_tokens) return shared >= min_tokens;
        return (segs - 1) * shared * token_bytes >= (rows <= lora::KV_ROW_ITEM ? SHARED_FEW_BYTES : SHARED_BYTES) + rows * kv.cfg.n_kv_heads * SHARED_ROW_BYTES * kv.cfg.head_dim / 128;
    };
    struct Set {
        int32_t at, base, depth, misses;  // pages that the segments have in common; those of them that are in prefixes already; how many these are; and how many had no room since the last
        std::vector<int32_t> segs;
    };
    const auto full = [&](int32_t i) { return g.seqs[i]->n_tokens >> kv.page_shift; };
    const auto page = [&](int32_t i, int32_t at) { return g.seqs[i]->pages[at]; };
    std::vector<Set> sets(1);
    for (size_t i = 0; i < g.seqs.size(); ++i)
        if (g.n_tokens[i] && (int64_t)g.n_tokens[i] * grp < lora::KV_TILE) sets[0].segs.push_back((int32_t)i);
    sets[0].at = sets[0].base = sets[0].depth = sets[0].misses = 0;
    cut.own.assign(g.seqs.size(), 0);
    int64_t room = (int64_t)kv.cfg.max_batch_tokens * SHARED_TOKENS;
    while (!sets.empty() && room >= 2) {  // (a prefix has two segments at least)
        Set set = std::move(sets.back());
        sets.pop_back();
        if (set.depth == SHARED_DEPTH) continue;
        std::vector<int32_t> &segs = set.segs;
        segs.erase(std::remove_if(segs.begin(), segs.end(), [&](int32_t i) { return full(i) <= set.at || kv.refs[page(i, set.at)] < 2; }), segs.end());
        std::sort(segs.begin(), segs.end(), [&](int32_t a, int32_t b) { return page(a, set.at) != page(b, set.at) ? page(a, set.at) < page(b, set.at) : a < b; });
        for (size_t first = 0, last; first < segs.size(); first = last) {
            for (last = first + 1; last < segs.size() && page(segs[last], set.at) == page(segs[first], set.at);) ++last;
            if (last - first < 2) continue;
            Set part{full(segs[first]), set.base, set.depth, set.misses, {segs.begin() + first, segs.begin() + last}};
            const int32_t *const p = g.seqs[segs[first]]->pages.data();
            int64_t tokens = 0;
            for (const int32_t i : part.segs) {
                part.at = std::min(part.at, full(i));
                part.at = (int32_t)(std::mismatch(p + set.at, p + part.at, g.seqs[i]->pages.data() + set.at).first - p);
                tokens += g.n_tokens[i];
            }
            const int32_t to = part.at & ~(std::max(PIECE_STEP >> kv.page_shift, 1) - 1);  // (what is behind a prefix begins where pieces may)
            if (to > part.base && worth((int64_t)(to - part.base) << kv.page_shift, (int64_t)part.segs.size(), tokens * grp)) {
                if (tokens > room) {  // left out; fewer segments that share more may have room
                    if (++part.misses > SHARED_MISSES) continue;
                    sets.push_back(std::move(part));
                    continue;
                }
                part.misses = 0;
                room -= tokens;
                // in bf16 the weights of few rows have 16 bits: they must not lose them by sharing
                const bool exact = tokens * grp > lora::KV_ROW_ITEM && kv.cfg.dtype == LORA_BF16 &&
                                   std::any_of(part.segs.begin(), part.segs.end(), [&](int32_t i) { return (int64_t)g.n_tokens[i] * grp <= lora::KV_ROW_ITEM; });
                cut.exact = cut.exact || exact;
                cut.prefixes.push_back({part.base, to, part.segs, tokens * grp, exact});
                for (const int32_t i : part.segs) cut.own[i] = to;
                part.base = to;
                ++part.depth;
            }
            sets.push_back(std::move(part));
        }
    }
    if (cut.prefixes.empty()) cut.own.clear();
}

// The same into pieces whose results are always joined, from token `from` on; where they lie is noted as a block of rows
void cut_shared(AttnItem base, int32_t from, int32_t to, int32_t piece, int32_t rows, int32_t n_kv, std::vector<AttnItem> &items, std::vector<SharedBlock> &blocks, int64_t &part)
{
    int32_t n = std::max((to - from + piece - 1) / piece, 1);
    const int32_t each = ((to - from + n - 1) / n + PIECE_STEP - 1) / PIECE_STEP * PIECE_STEP, stride = rows * n_kv;
    n = (to - from + each - 1) / each;
    blocks.push_back({(int32_t)part, n, stride, base.n_rows});
    for (int32_t i = 0; i < n; ++i) {
        base.kv0 = from + i * each;
        base.kv1 = std::min(to, from + (i + 1) * each);
        base.part = (int32_t)part;
        part += stride;
        items.push_back(base);
    }
}

// false: the results of the prefixes' pieces have no room
bool cut_attention(const lora_kv &kv, const Growth &g, const int32_t *offsets, Cut &cut)
{
    const auto from_of = [&](size_t i) { return cut.own.empty() ? (int64_t)0 : (int64_t)cut.own[i] << kv.page_shift; };
    const auto tokens_of = [&](const Prefix &p) { return (int64_t)(p.to - p.from) << kv.page_shift; };
    const int32_t grp = kv.group(), n_kv = kv.cfg.n_kv_heads, tile_min = tile_min_tokens(kv.cfg);
    int64_t row_tokens = 0, tile_tokens = 0, n_tiles = 0, longest = 0, part = 0, tile = lora::KV_TURNS_TILE;
    const auto tile_end = [&tile, grp](int64_t ctx, int64_t rows, int64_t row0) {  // tokens that the tile's last row sees
        return (int32_t)(ctx + (std::min(rows, row0 + tile) - 1) / grp + 1);
    };
    // Two groups of wavefronts in turns, 256 rows at a time, where every compute unit gets two such blocks at least and they are long (1024 tokens in the
    // mean).  Measured, tiles of 128 rows -> turns: 16384 tokens with 64 / 8 heads 3985 -> 3650 us, 8192 with 32 / 8 537 -> 499, 4096 150 -> 136, 2048 + 2048 81.3 -> 76.9, 4096 with 32 / 32
    // heads 152 -> 143.  The rule does not ask for a gain where it takes few rounds of blocks: 2048 + 2048 with 32 / 32 heads 85.1 -> 85.5, 3 x 1500 behind 600 with 40 / 40 155.5 -> 160.
    if (lora::kv_turns(kv.cfg.dtype, kv.cfg.head_dim)) {
        int64_t tokens = 0;
        for (size_t i = 0; i < g.seqs.size(); ++i) {
            const int64_t n = g.n_tokens[i], rows = n * grp, ctx = g.seqs[i]->n_tokens - n;
            if (rows > lora::KV_ROW_ITEM)
                for (int64_t r = 0; r < rows; r += tile) tokens += tile_end(ctx, rows, r) - from_of(i), ++n_tiles;
        }
        for (const Prefix &p : cut.prefixes)
            if (p.rows > lora::KV_ROW_ITEM) tokens += (p.rows + tile - 1) / tile * tokens_of(p), n_tiles += (p.rows + tile - 1) / tile;
        if (n_tiles * n_kv >= 2 * kv.n_cu && tokens >= 1024 * n_tiles) cut.way = lora::KV_TILES_TURNS;
        // Prefixes, of which there are few tiles: as many pieces as compute units where each is long enough and the tiles' rows are there.  32 requests behind 100000 tokens with 64 / 8 heads
        // 180 -> 162 us.
        int64_t large = 0, small = 0;
        for (const Prefix &p : cut.prefixes)
            if (p.rows > lora::KV_ROW_ITEM) large += (p.rows + tile - 1) / tile * tokens_of(p), small += (p.rows + lora::KV_TILE - 1) / lora::KV_TILE * tokens_of(p);
        if (large * n_kv >= 1024 * kv.n_cu && large * 2 <= small * 5 / 4) cut.way = lora::KV_TILES_TURNS;
    }
    if (cut.way != lora::KV_TILES_TURNS) tile = lora::KV_TILE;
    n_tiles = 0;
    for (size_t i = 0; i < g.seqs.size(); ++i) {
        const int64_t n = g.n_tokens[i], rows = n * grp, ctx = g.seqs[i]->n_tokens - n;
        if (!n) continue;
        if (rows <= lora::KV_ROW_ITEM) row_tokens += ctx + n - from_of(i);
        else
            for (int64_t r = 0; r < rows; r += tile, ++n_tiles) {
                const int64_t end = tile_end(ctx, rows, r) - from_of(i);
                tile_tokens += end;
                longest = std::max(longest, end);
            }
    }
    for (const Prefix &p : cut.prefixes) {
        if (p.rows <= lora::KV_ROW_ITEM) {
            row_tokens += tokens_of(p);
            continue;
        }
        const int64_t tiles = (p.rows + tile - 1) / tile;
        n_tiles += tiles;
        tile_tokens += tiles * tokens_of(p);
        longest = std::max(longest, tokens_of(p));
    }
    const int32_t short_tokens = (kv.e4m3() ? ROW_SHORT_E4M3 : ROW_SHORT_VALUES) / kv.cfg.head_dim;
    const auto at_least = [](int64_t tokens, int64_t least) { return (int32_t)std::min(std::max(tokens, least), (int64_t)LORA_KV_MAX_TOKENS); };
    int32_t row_piece = at_least(row_tokens * n_kv / ROW_BLOCKS, ROW_MIN_TOKENS);
    // A tile that takes longer than all of a compute unit's share is cut, into pieces of half of that: two at a time are worked on
    const int64_t share = tile_tokens * n_kv / kv.n_cu;
    int32_t tile_piece = at_least(share / 2, tile_min), tile_whole = at_least(share, tile_min);
    // Prefixes are joined anyway, and cut into as many pieces; but not into shorter ones than the rows beside them keep the machine busy with, three quarters of whose tokens for a compute unit
    // take a tile about as long (256 requests of 350 tokens behind 2000 with 32 / 8 heads: 4 pieces 94.3 us, 2 85.0, 1 83.8).
    int32_t prefix_row_piece = at_least(row_tokens * n_kv / ROW_BLOCKS, SHARED_ROW_MIN_TOKENS);
    int32_t prefix_tile_piece = at_least(cut.way == lora::KV_TILES_TURNS ? share : share / 2, tile_min);
    if (cut.way != lora::KV_TILES_TURNS) prefix_tile_piece = std::max(prefix_tile_piece, at_least(row_tokens * n_kv / kv.n_cu * 3 / 4, 0));
    // The same, evenly for the compute units: prefixes in tiles, tiles, rows of batches that have nothing else
    const auto evenly = [&](int32_t piece, auto blocks) { return at_least(even_piece(piece, kv.n_cu, blocks), 0); };
    const auto prefix_blocks = [&](bool tiles, int64_t piece) {
        int64_t n = 0;
        for (const Prefix &p : cut.prefixes)
            if ((p.rows > lora::KV_ROW_ITEM) == tiles) n += (tiles ? (p.rows + tile - 1) / tile : 1) * pieces_of(tokens_of(p), piece) * n_kv;
        return n;
    };
    const auto own_rows = [&](int64_t piece) {  // blocks of rows: that a wavefront may do alone or not
        int64_t n[2] = {0, 0};
        for (size_t i = 0; i < g.seqs.size(); ++i)
            if (g.n_tokens[i]) n[g.seqs[i]->n_tokens - from_of(i) > short_tokens] += pieces_of(g.seqs[i]->n_tokens - from_of(i), piece) * n_kv;
        return std::pair(n[0], n[1]);
    };
    const auto own_tiles = [&](int64_t piece) {
        int64_t n = 0;
        for (size_t i = 0; i < g.seqs.size(); ++i) {
            const int64_t rows = (int64_t)g.n_tokens[i] * grp, ctx = g.seqs[i]->n_tokens - g.n_tokens[i];
            for (int64_t r = 0; rows > lora::KV_ROW_ITEM && r < rows; r += tile) {
                const int64_t end = tile_end(ctx, rows, r) - from_of(i);
                n += (from_of(i) || end > std::max((int64_t)tile_whole, piece) ? pieces_of(end, piece) : 1) * n_kv;
            }
        }
        return n;
    };
    const bool few_rows = !n_tiles && (int64_t)g.seqs.size() * n_kv <= EVEN_ROUNDS * kv.n_cu;
    if (!cut.prefixes.empty()) prefix_tile_piece = evenly(prefix_tile_piece, [&](int64_t piece) { return std::pair(prefix_blocks(true, piece), (int64_t)0); });
    if (n_tiles && (kv.e4m3() || !cut.prefixes.empty()) && n_tiles * n_kv <= EVEN_ROUNDS * kv.n_cu) {
        const int64_t beside = prefix_blocks(true, prefix_tile_piece);
        if (own_tiles(tile_piece)) tile_piece = evenly(tile_piece, [&](int64_t piece) { return std::pair(own_tiles(piece) + beside, (int64_t)0); });
        tile_whole = std::max(tile_whole, tile_piece);
    } else if (few_rows && !cut.prefixes.empty()) {
        const auto [alone, others] = own_rows(row_piece);
        const int64_t beside = others + (alone > 4 * kv.n_cu ? alone / 4 : alone);
        prefix_row_piece = evenly(prefix_row_piece, [&](int64_t piece) {
            const int64_t n = prefix_blocks(false, piece);
            return std::pair(n, n + beside);
        });
    } else if (few_rows && kv.e4m3()) {
        row_piece = evenly(row_piece, [&](int64_t piece) {
            const auto [alone, others] = own_rows(piece);
            return std::pair(alone + others, (int64_t)0);
        });
    }
    // No more blocks than compute units and no tile of over 1024 tokens: for heads of 64, whose steps are mostly instructions of one wavefront after the other, two groups of
    // wavefronts share a tile's tokens, and tiles stay whole (700 tokens with 32 heads 16.5 -> 12.5 us, with 32 / 8 heads 15.3 -> 12.3).  Longer ones, and heads of 128, do as well
    // or better with pieces.
    if (cut.way == lora::KV_TILES_PLAIN && cut.prefixes.empty() && lora::kv_pairs(kv.cfg.dtype, kv.cfg.head_dim) && n_tiles && n_tiles * n_kv <= kv.n_cu && longest <= 2 * tile_min) {
        cut.way = lora::KV_TILES_PAIRS;
        tile_whole = 2 * tile_min;
    }
    // Where tiles are cut anyway, and pieces of fewer tokens still find a compute unit each (a quarter more than the share: not all pieces are whole), the last is done earlier: 213 + 752 tokens
    // with 6 / 2 heads 17.6 -> 13.9 us, 1072 18.6 -> 16.8, 1000 with 8 / 1 heads of 256 29.1 -> 24.5.
    if (cut.way == lora::KV_TILES_PLAIN && longest > tile_min) {
        const int32_t piece = at_least(share * 5 / 4, tile_min / 2);
        if (piece < tile_min) tile_piece = tile_whole = piece;
    }
    for (;;) {
        cut.rows.clear();
        cut.tiles.clear();
        cut.joins.clear();
        cut.tile_joins.clear();
        cut.row_tokens.clear();
        cut.sources.clear();
        cut.blocks.clear();
        cut.shared_joins.clear();
        cut.prefix_segments = 0;
        part = 0;
        cut.extra_joins = 0;
        const auto put_joins = [&](int32_t tok0, int32_t row0, int32_t rows_of, int32_t n_sources) {
            for (int32_t r = 0; r < rows_of; r += lora::KV_JOIN_ROWS)
                cut.shared_joins.push_back({tok0, row0, r, std::min(rows_of - r, (int32_t)lora::KV_JOIN_ROWS), (int32_t)cut.sources.size(), n_sources});
        };
        // prefixes first, then the segments' own tokens: what of a prefix a segment's rows are, by prefix and segment
        std::vector<std::vector<SharedSource>> of_segment(cut.own.size());
        for (const Prefix &p : cut.prefixes) {
            const bool tiles = p.rows > lora::KV_ROW_ITEM;
            const int32_t rows_of = tiles ? (int32_t)tile : lora::KV_ROW_ITEM, block0 = (int32_t)cut.blocks.size(), list0 = (int32_t)cut.row_tokens.size();
            int64_t row = 0;
            for (const int32_t i : p.segs) {
                of_segment[i].push_back({(int32_t)row, block0, rows_of, tiles});
                for (int32_t t = 0; t < g.n_tokens[i]; ++t) cut.row_tokens.push_back(offsets[i] + t);
                row += (int64_t)g.n_tokens[i] * grp;
            }
            AttnItem it{list0, p.exact ? lora::KV_EXACT : lora::KV_SHARED, cut.page0[p.segs[0]], 0, 0, 0, 0, -1};
            for (int64_t r = 0; r < p.rows; r += rows_of) {
                it.row0 = (int32_t)r;
                it.n_rows = (int32_t)std::min(p.rows - r, (int64_t)rows_of);
                cut_shared(it, p.from << kv.page_shift, p.to << kv.page_shift, tiles ? prefix_tile_piece : prefix_row_piece, tiles ? (it.n_rows + 31) & ~31 : it.n_rows, n_kv, tiles ? cut.tiles : cut.rows,
                           cut.blocks, part);
            }
        }
        cut.prefix_row_items = (int32_t)cut.rows.size();
        cut.prefix_tile_items = (int32_t)cut.tiles.size();
        for (size_t i = 0; i < g.seqs.size(); ++i) {
            const int64_t n = g.n_tokens[i], rows = n * grp, ctx = g.seqs[i]->n_tokens - n;
            if (!n) continue;
            AttnItem it{offsets[i], (int32_t)ctx, cut.page0[i], 0, (int32_t)rows, 0, 0, -1};
            if (from_of(i)) {  // (fewer rows than a tile has)
                const bool tiles = rows > lora::KV_ROW_ITEM;
                of_segment[i].push_back({0, (int32_t)cut.blocks.size(), lora::KV_TILE, tiles});
                cut_shared(it, (int32_t)from_of(i), (int32_t)(ctx + n), tiles ? tile_piece : row_piece, tiles ? (it.n_rows + 31) & ~31 : it.n_rows, n_kv, tiles ? cut.tiles : cut.rows, cut.blocks,
                           part);
                put_joins(offsets[i], 0, (int32_t)rows, (int32_t)of_segment[i].size());
                ++cut.prefix_segments;
                cut.sources.insert(cut.sources.end(), of_segment[i].begin(), of_segment[i].end());
                continue;
            }
            // what is cut beside segments with prefixes is joined by their launch
            const auto cut_one = [&](int32_t end, int32_t piece, int32_t block_rows, std::vector<AttnItem> &items, std::vector<JoinItem> &joins, bool tiles) {
                if (cut.prefixes.empty() || end <= piece) return cut_block(it, end, piece, block_rows, n_kv, items, joins, part);
                put_joins(it.tok0, it.row0, it.n_rows, 1);
                ++cut.extra_joins;
                cut.sources.push_back({0, (int32_t)cut.blocks.size(), (int32_t)tile, tiles});
                cut_shared(it, 0, end, piece, block_rows, n_kv, items, cut.blocks, part);
            };
            if (rows <= lora::KV_ROW_ITEM) {
                cut_one((int32_t)(ctx + n), row_piece, it.n_rows, cut.rows, cut.joins, false);
                continue;
            }
            for (int64_t r = 0; r < rows; r += tile) {
                it.row0 = (int32_t)r;
                it.n_rows = (int32_t)std::min(rows - r, tile);
                const int32_t end = tile_end(ctx, rows, r);
                cut_one(end, end > tile_whole ? tile_piece : end, (it.n_rows + 31) & ~31, cut.tiles, cut.tile_joins, true);
            }
        }
        if (cut.way == lora::KV_TILES_PAIRS && (int64_t)(cut.tiles.size() + cut.rows.size()) * n_kv > kv.n_cu) {
            cut.way = lora::KV_TILES_PLAIN;
            tile_whole = at_least(share, tile_min);
            continue;
        }
        if (part <= kv.part_rows && (int64_t)(cut.joins.size() + cut.tile_joins.size()) + cut.extra_joins <= MAX_EXTRA && (int64_t)cut.shared_joins.size() <= max_shared_joins(kv.cfg) && (int64_t)(cut.rows.size() + cut.tiles.size()) <= max_items(kv.cfg)) break;
        if (!cut.prefixes.empty() && row_piece == LORA_KV_MAX_TOKENS && tile_piece == LORA_KV_MAX_TOKENS && prefix_row_piece == LORA_KV_MAX_TOKENS && prefix_tile_piece == LORA_KV_MAX_TOKENS) return false;
        row_piece = at_least((int64_t)row_piece * 2, 0);
        tile_piece = at_least((int64_t)tile_piece * 2, 0);
        prefix_row_piece = at_least((int64_t)prefix_row_piece * 2, 0);
        prefix_tile_piece = at_least((int64_t)prefix_tile_piece * 2, 0);
        tile_whole = std::max(tile_whole, tile_piece);
    }
    // Three blocks on a compute unit, where the tiles fill more than three for each, or more than two and are short (256 tokens in the mean): bf16 heads of 128, two blocks -> three,
    // 8 x 500 tokens with 32 heads 42.6 -> 39.2 us, 6 x 300 24.4 -> 17.3; but 2048 with 40 heads 68.2 -> 74.5.
    if (cut.way == lora::KV_TILES_PLAIN && !kv.e4m3() && !cut.exact && lora::kv_many(kv.cfg.dtype, kv.cfg.head_dim)) {
        int64_t blocks = (int64_t)cut.tiles.size() * n_kv, tokens = 0;
        for (const AttnItem &t : cut.tiles) tokens += t.kv1 - t.kv0;
        if (blocks > 3 * kv.n_cu || (blocks > 2 * kv.n_cu && tokens < 256 * (int64_t)cut.tiles.size())) cut.way = lora::KV_TILES_MANY;
    }
    // the longest first: what starts last is short
    const auto longer = [](const AttnItem &a, const AttnItem &b) { return a.kv1 - a.kv0 > b.kv1 - b.kv0; };
    std::stable_sort(cut.rows.begin(), cut.rows.end(), longer);
    std::stable_sort(cut.tiles.begin(), cut.tiles.end(), longer);
    // Where there are more items than blocks fit on the machine, a wavefront has a short one to itself: a block on it is mostly waiting for its first
    // loads and its last stores.  Measured: 512 requests of 20 tokens with 32 heads of 128 96 -> 51 us, 256 of 120 94 -> 78 us; with 200 to 450 tokens, and
    // with half as many for heads of 256, nothing is gained.  Beside prefixes, whose parts are there to be worked on, from twice as many on: 128 requests with 20 tokens of their own behind 2000 with 32 / 8
    // heads 29.2 -> 27.8 us, 20 of 50 with 40 / 40 26.9 -> 25.4.
    size_t n_short = 0;
    const auto is_short = [&](const AttnItem &it) { return (it.part < 0 || !cut.prefixes.empty()) && it.kv1 - it.kv0 <= short_tokens; };
    while (n_short < cut.rows.size() && is_short(cut.rows[cut.rows.size() - 1 - n_short])) ++n_short;
    cut.n_short = (int64_t)n_short * n_kv > (cut.prefixes.empty() ? 2 : 4) * kv.n_cu ? (int32_t)n_short : 0;
    // Tiles are worked on two at a time on a compute unit, block b beside block b + n_cu: the longest go with the shortest of the first two rounds
    // (2048 tokens with 32 / 8 heads: 70 -> 55 us).
    const size_t round = ((size_t)kv.n_cu + n_kv - 1) / n_kv;
    if (cut.way != lora::KV_TILES_TURNS && cut.tiles.size() > round) std::reverse(cut.tiles.begin() + round, cut.tiles.begin() + std::min(cut.tiles.size(), 2 * round));
    return true;
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

template <typename F> int guarded(F f)  // no exception leaves a C entry
{
    try {
        return f();
    } catch (const std::bad_alloc &) {
        return LORA_E_NOMEM;
    } catch (...) {
        return LORA_E_NOMEM;
    }
}

}  // namespace

extern "C" {

size_t lora_kv_page_bytes(const lora_kv_config_t *cfg) { return good(cfg) ? layer_bytes(*cfg) * cfg->n_layers : 0; }
size_t lora_kv_pages_bytes(const lora_kv_config_t *cfg) { return lora_kv_page_bytes(cfg) * (good(cfg) ? cfg->n_pages : 0); }
size_t lora_kv_work_bytes(const lora_kv_config_t *cfg)
{
    return good(cfg) ? list_bytes(*cfg) * (cfg->n_batches + SPARE_BATCHES) + PART_BYTES : 0;
}

int lora_kv_create(const lora_kv_config_t *cfg, void *dev_pages, size_t pages_bytes, void *dev_work, size_t work_bytes, lora_kv_t **out)
{
    if (!out) return LORA_E_INVAL;
    *out = nullptr;
    if (!good(cfg)) return LORA_E_INVAL;
    const bool host_only = cfg->flags & LORA_KV_HOST_ONLY;
    if (!host_only) {
        if (!dev_pages || !dev_work || ((reinterpret_cast<uintptr_t>(dev_pages) | reinterpret_cast<uintptr_t>(dev_work)) & (ALIGN - 1))) return LORA_E_INVAL;
        if (pages_bytes < lora_kv_pages_bytes(cfg) || work_bytes < lora_kv_work_bytes(cfg)) return LORA_E_NOMEM;
    }
    return guarded([&]() -> int {
        lora_kv *kv = new lora_kv;
        struct Guard {
            lora_kv *kv;
            ~Guard() { if (kv) lora_kv_destroy(kv); }
        } guard{kv};
        kv->cfg = *cfg;
        kv->host_only = host_only;
        kv->pages = static_cast<char *>(dev_pages);
        kv->work = static_cast<char *>(dev_work);
        kv->layer_bytes = layer_bytes(*cfg);
        kv->page_bytes = lora_kv_page_bytes(cfg);
        kv->list_cap = list_bytes(*cfg);
        kv->page_shift = __builtin_ctz((unsigned)cfg->page_tokens);
        kv->seqs.resize(cfg->max_seqs);
        kv->seen.assign(cfg->max_seqs, 0u);
        kv->free_seqs.resize(cfg->max_seqs);
        for (int32_t i = 0; i < cfg->max_seqs; ++i) kv->free_seqs[i] = cfg->max_seqs - 1 - i;
        kv->slot_of.reserve(cfg->max_seqs);
        kv->refs.assign(cfg->n_pages, 0);
        kv->limit = kv->free_pages = cfg->n_pages;
        kv->free_bits.assign(((size_t)cfg->n_pages + 63) / 64, ~(uint64_t)0);
        if (cfg->n_pages & 63) kv->free_bits.back() = ((uint64_t)1 << (cfg->n_pages & 63)) - 1;
        kv->batches.resize(cfg->n_batches + SPARE_BATCHES);
        for (auto &b : kv->batches) b.member.assign(cfg->max_seqs, 0);
        if (!host_only) {
            KV_TRY(lora::prepare_attn_kernels());
            KV_TRY(lora::prepare_attn_e4m3_kernels());
            int n = 0;
            KV_TRY(hipGetDevice(&kv->device));
            KV_TRY(hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, kv->device));
            if (n > 0) kv->n_cu = n;
            char *at = kv->work;
            for (auto &b : kv->batches) {
                b.dev = at;
                at += kv->list_cap;
                KV_TRY(hipHostMalloc(reinterpret_cast<void **>(&b.pinned), kv->list_cap, hipHostMallocMapped));
                KV_TRY(hipHostGetDevicePointer(reinterpret_cast<void **>(const_cast<char **>(&b.pinned_dev)), b.pinned, 0));
                KV_TRY(hipEventCreateWithFlags(&b.uploaded, hipEventDisableTiming));
            }
            KV_TRY(hipEventCreateWithFlags(&kv->order_ev, hipEventDisableTiming));
            // of a row: head_dim sums, and its maximum and weight
            kv->part_rows = (int64_t)(PART_BYTES / ((size_t)(cfg->head_dim + 2) * 4));
            kv->part_o = reinterpret_cast<float *>(at);
            kv->part_ml = kv->part_o + kv->part_rows * cfg->head_dim;
        }
        {
            std::lock_guard<std::mutex> lock(g_lock);
            kv->next = g_caches;
            if (g_caches) g_caches->before = kv;
            g_caches = kv;
        }
        guard.kv = nullptr;
        *out = kv;
        return LORA_OK;
    });
}

int lora_kv_destroy(lora_kv_t *kv)
{
    if (!kv) return LORA_E_INVAL;
    {
        std::lock_guard<std::mutex> lock(g_lock);
        if (kv->next) kv->next->before = kv->before;
        if (kv->before) kv->before->next = kv->next;
        else if (g_caches == kv) g_caches = kv->next;
    }
    for (auto &b : kv->batches) {
        if (b.pinned) (void)hipHostFree(b.pinned);
        if (b.uploaded) (void)hipEventDestroy(b.uploaded);
    }
    if (kv->order_ev) (void)hipEventDestroy(kv->order_ev);
    delete kv;
    return LORA_OK;
}

// ---- sequences ----------------------------------------------------------------------------

static int add_sequences(lora_kv_t *kv, int32_t n, const int64_t *ids, const Seq *parent, int32_t n_tokens)
{
    if (n > (int32_t)kv->free_seqs.size()) {
        return LORA_E_NOMEM;
    }
    const size_t shared = parent ? ((size_t)n_tokens + kv->cfg.page_tokens - 1) >> kv->page_shift : 0;
    for (int32_t i = 0; i < n; ++i)
        if (kv->slot_of.count(ids[i])) return LORA_E_STATE;
    // the sequences are made aside: nothing has changed if an id comes twice or host memory runs out
    std::unordered_map<int64_t, int32_t> fresh;
    std::vector<std::vector<int32_t>> pages(n);
    for (int32_t i = 0; i < n; ++i) {
        if (!fresh.emplace(ids[i], i).second) return LORA_E_STATE;
        if (parent) pages[i].assign(parent->pages.begin(), parent->pages.begin() + shared);
    }
    kv->slot_of.reserve(kv->slot_of.size() + n);
    int32_t done = 0;
    try {
        for (; done < n; ++done) kv->slot_of.emplace(ids[done], kv->free_seqs[kv->free_seqs.size() - 1 - done]);
    } catch (...) {
        while (done--) kv->slot_of.erase(ids[done]);
        throw;
    }
    for (int32_t i = 0; i < n; ++i) {
        Seq &s = kv->seqs[kv->free_seqs.back()];
        kv->free_seqs.pop_back();
        s.id = ids[i];
        s.alive = true;
        s.n_tokens = parent ? n_tokens : 0;
        s.pages = std::move(pages[i]);
        for (int32_t p : s.pages) ++kv->refs[p];
    }
    return LORA_OK;
}

int lora_kv_seq_add(lora_kv_t *kv, int32_t n, const int64_t *ids)
{
    if (!kv || n < 0 || (n && !ids)) return LORA_E_INVAL;
    return guarded([&] { return add_sequences(kv, n, ids, nullptr, 0); });
}

int lora_kv_seq_fork(lora_kv_t *kv, int64_t parent, int32_t n, const int64_t *ids, int32_t n_tokens)
{
    if (!kv || n < 0 || (n && !ids) || n_tokens < -1) return LORA_E_INVAL;
    return guarded([&]() -> int {
        const Seq *p = kv->find(parent);
        if (!p) return LORA_E_NOTFOUND;
        if (n_tokens > p->n_tokens) return LORA_E_INVAL;
        return add_sequences(kv, n, ids, p, n_tokens < 0 ? p->n_tokens : n_tokens);
    });
}

int lora_kv_seq_extend(lora_kv_t *kv, int32_t n, const int64_t *ids, const int32_t *n_tokens, void *stream)
{
    if (!kv || n < 0 || (n && (!ids || !n_tokens))) return LORA_E_INVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return guarded([&]() -> int {
        const OnDevice on(*kv);
        Growth g;
        if (const int rc = check_growth(*kv, n, ids, n_tokens, nullptr, g)) return rc;
        reserve(*kv, g);
        if (!kv->host_only) {
            if (const int rc = refuse_capture(st)) return rc;
            if (const int rc = in_order(*kv, st)) return rc;  // (also where nothing is copied: what the caller puts into the pages must not overtake work that reads them)
        }
        grow(*kv, g);
        return g.from.empty() || kv->host_only ? LORA_OK : copy_pages(*kv, g.from, g.to, st);
    });
}

int lora_kv_seq_truncate(lora_kv_t *kv, int32_t n, const int64_t *ids, const int32_t *n_tokens)
{
    if (!kv || n < 0 || (n && (!ids || !n_tokens))) return LORA_E_INVAL;
    kv->next_call();
    for (int32_t i = 0; i < n; ++i) {
        const Seq *s = kv->find(ids[i]);
        if (!s) return LORA_E_NOTFOUND;
        if (!kv->first_time(*s) || n_tokens[i] < 0 || n_tokens[i] > s->n_tokens) return LORA_E_INVAL;
    }
    for (int32_t i = 0; i < n; ++i) {
        Seq &s = *kv->find(ids[i]);
        if (s.n_tokens == n_tokens[i]) continue;
        kv->drop_batches_with(s);
        s.n_tokens = n_tokens[i];
        const size_t keep = ((size_t)s.n_tokens + kv->cfg.page_tokens - 1) >> kv->page_shift;
        while (s.pages.size() > keep) {
            kv->give_back(s.pages.back());
            s.pages.pop_back();
        }
    }
    return LORA_OK;
}

int lora_kv_seq_free(lora_kv_t *kv, int32_t n, const int64_t *ids)
{
    if (!kv || n < 0 || (n && !ids)) return LORA_E_INVAL;
    kv->next_call();
    for (int32_t i = 0; i < n; ++i) {
        const Seq *s = kv->find(ids[i]);
        if (!s) return LORA_E_NOTFOUND;
        if (!kv->first_time(*s)) return LORA_E_INVAL;
    }
    for (int32_t i = 0; i < n; ++i) {
        Seq &s = *kv->find(ids[i]);
        kv->drop_batches_with(s);
        for (int32_t p : s.pages) kv->give_back(p);
        s.pages.clear();
        s.n_tokens = 0;
        s.alive = false;
        kv->free_seqs.push_back(kv->slot(s));  // (never more than it held at first)
        kv->slot_of.erase(ids[i]);
    }
    return LORA_OK;
}

int lora_kv_seq_info(const lora_kv_t *kv, int64_t id, lora_kv_seq_info_t *out)
{
    if (!kv || !out) return LORA_E_INVAL;
    const Seq *s = const_cast<lora_kv_t *>(kv)->find(id);
    if (!s) return LORA_E_NOTFOUND;
    *out = {s->n_tokens, (int32_t)s->pages.size(), 0};
    for (int32_t p : s->pages) out->n_shared += kv->refs[p] > 1;
    return LORA_OK;
}

int lora_kv_seq_pages(const lora_kv_t *kv, int64_t id, int32_t *pages, int32_t cap, int32_t *n)
{
    if (!kv || !n || cap < 0) return LORA_E_INVAL;
    const Seq *s = const_cast<lora_kv_t *>(kv)->find(id);
    if (!s) return LORA_E_NOTFOUND;
    *n = (int32_t)s->pages.size();
    if (pages) std::copy_n(s->pages.begin(), std::min(*n, cap), pages);
    return LORA_OK;
}

int lora_kv_seq_read(lora_kv_t *kv, int32_t n, const int64_t *ids, const int32_t *first, const int32_t *n_tokens, int32_t layer, void *k, int64_t k_stride, void *v, int64_t v_stride,
                     int64_t n_rows, void *stream)
{
    if (!kv || n < 0 || (n && !ids) || layer < 0 || layer >= kv->cfg.n_layers || n_rows < 0 || n_rows > INT32_MAX) return LORA_E_INVAL;
    if (kv->host_only) return LORA_E_STATE;
    const lora_kv_config_t &c = kv->cfg;
    return guarded([&]() -> int {
        struct Part {
            const Seq *seq;
            int32_t pos, end;
        };
        std::vector<Part> parts(n);
        int64_t tokens = 0;
        for (int32_t i = 0; i < n; ++i) {
            const Seq *s = kv->find(ids[i]);
            if (!s) return LORA_E_NOTFOUND;
            const int64_t pos = first ? first[i] : 0, end = n_tokens ? pos + n_tokens[i] : s->n_tokens;
            if (pos < 0 || end < pos || end > s->n_tokens) return LORA_E_INVAL;
            parts[i] = {s, (int32_t)pos, (int32_t)end};
            tokens += end - pos;
        }
        if (tokens != n_rows) return LORA_E_INVAL;
        if (!tokens) return LORA_OK;
        const int64_t row = (int64_t)c.n_kv_heads * c.head_dim, u = kv->row_chunk();
        const auto bad = [&](const void *p, int64_t stride) { return !p || !aligned16(p) || stride < row || stride % u || stride > ((int64_t)1 << 40); };
        if (bad(k, k_stride) || bad(v, v_stride)) return LORA_E_INVAL;
        hipStream_t st = static_cast<hipStream_t>(stream);
        const OnDevice on(*kv);
        if (const int rc = in_order(*kv, st)) return rc;
        lora::ReadArgs a;
        a.pages = kv->pages + kv->layer_bytes * layer;
        a.page_stride = (int64_t)kv->page_bytes;
        a.k = k, a.v = v, a.k_stride = k_stride, a.v_stride = v_stride;
        a.n_kv = c.n_kv_heads, a.dim = c.head_dim, a.page_shift = kv->page_shift, a.n_reads = 0;
        int32_t at = 0;
        for (const Part &p : parts)
            for (int32_t pos = p.pos; pos < p.end;) {
                const int32_t off = pos & (c.page_tokens - 1), m = std::min(p.end - pos, c.page_tokens - off);
                a.page[a.n_reads] = p.seq->pages[pos >> kv->page_shift];
                a.off[a.n_reads] = (uint8_t)off;
                a.row[a.n_reads] = at;
                a.row[++a.n_reads] = at += m;
                pos += m;
                if (a.n_reads == lora::KV_MAX_READS || at == tokens) {
                    KV_TRY(lora::launch_read(a, c.dtype, kv->e4m3(), st));
                    a.n_reads = 0;
                }
            }
        return LORA_OK;
    });
}

// ---- pages ---------------------------------------------------------------------------------

int lora_kv_compact(lora_kv_t *kv, void *stream, int32_t *moved)
{
    if (!kv) return LORA_E_INVAL;
    if (moved) *moved = 0;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return guarded([&]() -> int {
        const OnDevice on(*kv);
        std::vector<int32_t> from, to;
        int32_t hole = 0;
        for (int32_t p = kv->used_pages; p < kv->limit; ++p) {
            if (!kv->refs[p]) continue;
            while (kv->refs[hole]) ++hole;  // as many free pages below used_pages as pages in use above it
            from.push_back(p);
            to.push_back(hole++);
        }
        std::vector<int32_t> where(kv->cfg.n_pages);
        if (!kv->host_only) {
            if (const int rc = refuse_capture(st)) return rc;
            if (const int rc = in_order(*kv, st)) return rc;  // (also where nothing moves: the free pages may be put to another use next, behind a limit)
        }
        if (from.empty()) return LORA_OK;
        if (!kv->host_only)
            if (const int rc = copy_pages(*kv, from, to, st)) return rc;
        for (int32_t p = 0; p < kv->cfg.n_pages; ++p) where[p] = p;
        const auto mark = [&](int32_t p, bool is_free) {
            const uint64_t bit = (uint64_t)1 << (p & 63);
            if (is_free) kv->free_bits[(size_t)p >> 6] |= bit;
            else kv->free_bits[(size_t)p >> 6] &= ~bit;
        };
        for (size_t i = 0; i < from.size(); ++i) {
            where[from[i]] = to[i];
            std::swap(kv->refs[from[i]], kv->refs[to[i]]);
            mark(from[i], true);
            mark(to[i], false);
        }
        for (auto &s : kv->seqs)
            for (int32_t &p : s.pages) p = where[p];
        for (auto &b : kv->batches) b.stale = b.stale || b.alive();
        kv->free_from = 0;
        kv->copied += (int64_t)from.size();
        if (moved) *moved = (int32_t)from.size();
        return LORA_OK;
    });
}

int lora_kv_set_limit(lora_kv_t *kv, int32_t limit)
{
    if (!kv || limit < 0 || limit > kv->cfg.n_pages) return LORA_E_INVAL;
    for (int32_t p = limit; p < kv->limit; ++p)
        if (kv->refs[p]) return LORA_E_STATE;
    for (int32_t p = std::min(limit, kv->limit); p < std::max(limit, kv->limit); ++p) kv->free_bits[(size_t)p >> 6] ^= (uint64_t)1 << (p & 63);
    kv->free_pages += limit - kv->limit;
    kv->limit = limit;
    kv->free_from = 0;
    return LORA_OK;
}

int lora_kv_stats(const lora_kv_t *kv, lora_kv_stats_t *out)
{
    if (!kv || !out) return LORA_E_INVAL;
    *out = {kv->limit, kv->used_pages, kv->free_pages, 0, 0, (int32_t)kv->slot_of.size(), kv->copied};
    for (int32_t p = 0; p < kv->limit; ++p) {
        out->pages_shared += kv->refs[p] > 1;
        if (kv->refs[p]) out->pages_end = p + 1;
    }
    return LORA_OK;
}

// ---- batches --------------------------------------------------------------------------------

static int create_batch(lora_kv_t *kv, int32_t n_seg, const int64_t *seg_seq, const int32_t *seg_offsets, void *stream, int32_t shared, lora_kv_batch_t **out)
{
    if (!out) return LORA_E_INVAL;
    *out = nullptr;
    if (!kv || n_seg < 0 || !seg_offsets || (n_seg && !seg_seq) || seg_offsets[0] != 0) return LORA_E_INVAL;
    if (kv->host_only) return LORA_E_STATE;
    if (n_seg > kv->cfg.max_batch_seqs) return LORA_E_NOMEM;
    for (int32_t i = 0; i < n_seg; ++i)
        if (seg_offsets[i + 1] < seg_offsets[i]) return LORA_E_INVAL;
    const int32_t T = seg_offsets[n_seg];
    if (T > kv->cfg.max_batch_tokens) return LORA_E_NOMEM;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return guarded([&]() -> int {
        const OnDevice on(*kv);
        if (kv->alive_batches >= kv->cfg.n_batches) return LORA_E_NOMEM;
        Growth g;
        if (const int rc = check_growth(*kv, n_seg, seg_seq, nullptr, seg_offsets, g)) return rc;
        int64_t n_pages = 0;
        for (int32_t i = 0; i < n_seg; ++i)
            if (g.n_tokens[i]) n_pages += ((int64_t)g.seqs[i]->n_tokens + g.n_tokens[i] + kv->cfg.page_tokens - 1) >> kv->page_shift;
        if (n_pages > kv->cfg.max_batch_pages) return LORA_E_NOMEM;
        if (const int rc = refuse_capture(st)) return rc;

        // the lists that have been free for longest: their last upload is over or nearly so
        Batch *b = nullptr;
        for (auto &x : kv->batches)
            if (!x.alive() && (!b || x.freed_at < b->freed_at)) b = &x;
        reserve(*kv, g);
        Cut cut;
        cut.page0.resize(n_seg);
        cut.rows.reserve(n_seg + MAX_EXTRA);
        cut.joins.reserve(MAX_EXTRA);
        if (const int rc = in_order(*kv, st)) return rc;
        if (b->upload_pending) {
            KV_TRY(hipEventSynchronize(b->uploaded));
            b->upload_pending = false;
        }

        std::vector<KvGroup> groups;
        groups.reserve((size_t)T / kv->chunk() + 2 * (size_t)n_seg);
        int32_t page0 = 0;
        for (int32_t i = 0; i < n_seg; ++i) {
            cut.page0[i] = page0;
            if (g.n_tokens[i]) page0 += (int32_t)(((int64_t)g.seqs[i]->n_tokens + g.n_tokens[i] + kv->cfg.page_tokens - 1) >> kv->page_shift);
        }
        if (shared >= 0) find_prefixes(*kv, g, shared, cut);
        // cut_attention sees the lengths after the growth; they are put back if it runs out of host memory
        for (int32_t i = 0; i < n_seg; ++i) g.seqs[i]->n_tokens += g.n_tokens[i];
        try {
            if (!cut_attention(*kv, g, seg_offsets, cut)) {
                cut.prefixes.clear();
                cut.own.clear();
                cut.exact = false;
                cut.way = lora::KV_TILES_PLAIN;
                (void)cut_attention(*kv, g, seg_offsets, cut);
            }
        } catch (...) {
            for (int32_t i = 0; i < n_seg; ++i) g.seqs[i]->n_tokens -= g.n_tokens[i];
            throw;
        }
        for (int32_t i = 0; i < n_seg; ++i) g.seqs[i]->n_tokens -= g.n_tokens[i];
        grow(*kv, g);

        std::fill(b->member.begin(), b->member.end(), 0);
        size_t at = 0;
        const auto place = [&](size_t bytes) {
            const size_t here = at;
            at += align_up(bytes);
            return here;
        };
        b->off_tokens = place((size_t)T * sizeof(KvToken));
        b->off_pages = place((size_t)n_pages * 4);
        b->off_rows = place(cut.rows.size() * sizeof(AttnItem));
        b->off_tiles = place(cut.tiles.size() * sizeof(AttnItem));
        b->off_joins = place(cut.joins.size() * sizeof(JoinItem));
        b->off_tile_joins = place(cut.tile_joins.size() * sizeof(JoinItem));
        b->off_row_tokens = place(cut.row_tokens.size() * 4);
        b->off_sources = place(cut.sources.size() * sizeof(SharedSource));
        b->off_blocks = place(cut.blocks.size() * sizeof(SharedBlock));
        b->off_shared_joins = place(cut.shared_joins.size() * sizeof(SharedJoin));
        KvToken *tokens = reinterpret_cast<KvToken *>(b->pinned + b->off_tokens);
        int32_t *pages = reinterpret_cast<int32_t *>(b->pinned + b->off_pages);
        b->max_pos = -1, b->exact = cut.exact;
        const int u = kv->chunk();
        for (int32_t i = 0; i < n_seg; ++i) {
            const Seq &s = *g.seqs[i];
            b->member[kv->slot(s)] = 1;
            if (!g.n_tokens[i]) continue;
            std::copy(s.pages.begin(), s.pages.end(), pages + cut.page0[i]);
            b->max_pos = std::max(b->max_pos, s.n_tokens - 1);
            const int32_t ctx = s.n_tokens - g.n_tokens[i];
            int32_t open = -1;  // chunk of the latest group
            for (int32_t t = 0; t < g.n_tokens[i]; ++t) {
                const int32_t pos = ctx + t, page = s.pages[pos >> kv->page_shift];
                tokens[seg_offsets[i] + t] = {pos, page};
                if (pos / u != open) {
                    open = pos / u;
                    groups.push_back({seg_offsets[i] + t, pos, 0, page});
                }
                ++groups.back().n;
            }
        }
        b->off_groups = place(groups.size() * sizeof(KvGroup));
        std::copy(groups.begin(), groups.end(), reinterpret_cast<KvGroup *>(b->pinned + b->off_groups));
        std::copy(cut.rows.begin(), cut.rows.end(), reinterpret_cast<AttnItem *>(b->pinned + b->off_rows));
        std::copy(cut.tiles.begin(), cut.tiles.end(), reinterpret_cast<AttnItem *>(b->pinned + b->off_tiles));
        std::copy(cut.joins.begin(), cut.joins.end(), reinterpret_cast<JoinItem *>(b->pinned + b->off_joins));
        std::copy(cut.tile_joins.begin(), cut.tile_joins.end(), reinterpret_cast<JoinItem *>(b->pinned + b->off_tile_joins));
        std::copy(cut.row_tokens.begin(), cut.row_tokens.end(), reinterpret_cast<int32_t *>(b->pinned + b->off_row_tokens));
        std::copy(cut.sources.begin(), cut.sources.end(), reinterpret_cast<SharedSource *>(b->pinned + b->off_sources));
        std::copy(cut.blocks.begin(), cut.blocks.end(), reinterpret_cast<SharedBlock *>(b->pinned + b->off_blocks));
        std::copy(cut.shared_joins.begin(), cut.shared_joins.end(), reinterpret_cast<SharedJoin *>(b->pinned + b->off_shared_joins));
        b->n_shared_joins = (int32_t)cut.shared_joins.size(), b->shared_rows = 0;
        for (const SharedJoin &j : cut.shared_joins) b->shared_rows = std::max(b->shared_rows, j.n_rows);
        b->n_joins = (int32_t)cut.joins.size(), b->n_tile_joins = (int32_t)cut.tile_joins.size();
        b->join_rows = 0;
        for (const JoinItem &j : cut.joins) b->join_rows = std::max(b->join_rows, j.n_rows);
        if (const int rc = copy_pages(*kv, g.from, g.to, st, {b->dev, b->pinned_dev, (uint32_t)((at + 15) / 16)}, b->uploaded)) return rc;
        b->upload_pending = true;
        b->stale = false;
        ++kv->alive_batches;
        std::lock_guard<std::mutex> lock(g_lock);
        b->info = {T, n_seg, (int32_t)n_pages, (int32_t)groups.size(), (int32_t)cut.rows.size(), (int32_t)cut.tiles.size(), (int32_t)(cut.joins.size() + cut.tile_joins.size()) + cut.extra_joins,
                   cut.n_short, (int32_t)cut.way};
        b->prefixes = {(int32_t)cut.prefixes.size(), cut.prefix_segments, cut.prefix_row_items, cut.prefix_tile_items, 0};
        for (const Prefix &p : cut.prefixes) b->prefixes.n_tokens += (int64_t)(p.to - p.from) << kv->page_shift;
        b->name = ++g_names << NAME_BITS | (uint64_t)(b - kv->batches.data());
        *out = reinterpret_cast<lora_kv_batch_t *>((uintptr_t)b->name);
        return LORA_OK;
    });
}

int lora_kv_batch_create(lora_kv_t *kv, int32_t n_seg, const int64_t *seg_seq, const int32_t *seg_offsets, void *stream, lora_kv_batch_t **out)
{
    return create_batch(kv, n_seg, seg_seq, seg_offsets, stream, -1, out);
}

int lora_kv_batch_create_shared(lora_kv_t *kv, int32_t n_seg, const int64_t *seg_seq, const int32_t *seg_offsets, int32_t min_tokens, void *stream, lora_kv_batch_t **out)
{
    if (out) *out = nullptr;
    return min_tokens < 0 ? LORA_E_INVAL : create_batch(kv, n_seg, seg_seq, seg_offsets, stream, min_tokens, out);
}

int lora_kv_batch_destroy(lora_kv_t *kv, lora_kv_batch_t *handle)
{
    Batch *const batch = kv ? find_batch(*kv, handle) : nullptr;
    if (!batch) return LORA_E_INVAL;
    batch->freed_at = ++kv->tick;
    --kv->alive_batches;
    std::lock_guard<std::mutex> lock(g_lock);
    batch->name = 0;
    return LORA_OK;
}

int lora_kv_batch_info(const lora_kv_batch_t *handle, lora_kv_batch_info_t *out)
{
    if (!handle || !out) return LORA_E_INVAL;
    std::lock_guard<std::mutex> lock(g_lock);
    for (lora_kv *kv = g_caches; kv; kv = kv->next)
        if (const Batch *const batch = find_batch(*kv, handle)) {
            *out = batch->info;
            return LORA_OK;
        }
    return LORA_E_INVAL;
}

int lora_kv_batch_prefixes(const lora_kv_batch_t *handle, lora_kv_prefix_info_t *out)
{
    if (!handle || !out) return LORA_E_INVAL;
    std::lock_guard<std::mutex> lock(g_lock);
    for (lora_kv *kv = g_caches; kv; kv = kv->next)
        if (const Batch *const batch = find_batch(*kv, handle)) {
            *out = batch->prefixes;
            return LORA_OK;
        }
    return LORA_E_INVAL;
}

int lora_kv_append(lora_kv_t *kv, lora_kv_batch_t *handle, int32_t layer, const lora_kv_append_t *a, void *stream) { return lora_kv_append_norm(kv, handle, layer, a, nullptr, stream); }

int lora_kv_append_norm(lora_kv_t *kv, lora_kv_batch_t *handle, int32_t layer, const lora_kv_append_t *a, const lora_kv_norm_t *norm, void *stream)
{
    Batch *const batch = kv ? find_batch(*kv, handle) : nullptr;
    if (!batch || !a || layer < 0 || layer >= kv->cfg.n_layers) return LORA_E_INVAL;
    if (batch->stale) return LORA_E_STATE;
    const lora_kv_config_t &c = kv->cfg;
    const int64_t row = (int64_t)c.n_kv_heads * c.head_dim, q_row = (int64_t)c.n_heads * c.head_dim, u = kv->row_chunk();
    const auto bad = [&](const void *p, int64_t stride, int64_t least) { return !p || !aligned16(p) || stride < least || stride % u || stride > ((int64_t)1 << 40); };
    if (batch->info.n_tokens) {
        if (bad(a->k, a->k_stride, row) || bad(a->v, a->v_stride, row)) return LORA_E_INVAL;
        if (a->q ? bad(a->q, a->q_stride, q_row) || bad(a->q_out, a->q_out_stride, q_row) : a->q_out != nullptr) return LORA_E_INVAL;
        if (a->q && a->q == a->q_out && a->q_stride != a->q_out_stride) return LORA_E_INVAL;
        if (a->rope && (!aligned16(a->rope) || a->rope_dim < 16 || a->rope_dim > c.head_dim || a->rope_dim % 16 || a->rope_positions <= batch->max_pos))
            return LORA_E_INVAL;
        const auto bad_weights = [&](const float *w, int32_t stride) { return w && (!aligned16(w) || stride % 4 || (stride && stride < c.head_dim)); };
        if (norm && (bad_weights(norm->q, norm->q_stride) || bad_weights(norm->k, norm->k_stride) || (norm->q && !a->q))) return LORA_E_INVAL;
    }
    if (norm && !(norm->eps >= FLT_MIN && std::isfinite(norm->eps))) return LORA_E_INVAL;
    if (a->rope && a->rope_pairs != LORA_ROPE_HALVES && a->rope_pairs != LORA_ROPE_NEIGHBOURS) return LORA_E_INVAL;
    if (!batch->info.n_tokens) return LORA_OK;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const OnDevice on(*kv);
    if (const int rc = in_order(*kv, st)) return rc;
    lora::AppendArgs k{};
    k.q = a->q, k.k = a->k, k.v = a->v, k.q_out = a->q_out;
    k.q_stride = a->q_stride, k.q_out_stride = a->q_out_stride, k.k_stride = a->k_stride, k.v_stride = a->v_stride;
    k.rope = a->rope;
    k.rope_dim = a->rope ? a->rope_dim : 0;
    k.neighbours = a->rope_pairs == LORA_ROPE_NEIGHBOURS;
    k.pages = kv->pages + kv->layer_bytes * layer;
    k.page_stride = (int64_t)kv->page_bytes;
    k.tokens = reinterpret_cast<const KvToken *>(batch->dev + batch->off_tokens);
    k.groups = reinterpret_cast<const KvGroup *>(batch->dev + batch->off_groups);
    k.n_tokens = batch->info.n_tokens, k.n_groups = batch->info.n_groups;
    k.n_heads = c.n_heads, k.n_kv = c.n_kv_heads, k.dim = c.head_dim, k.page_shift = kv->page_shift;
    if (kv->e4m3() || (norm && (norm->q || norm->k))) {
        lora::AppendHeadsArgs h{k, nullptr, nullptr, 0, 0, 1.0};
        if (norm) h = {k, norm->q, norm->k, norm->q_stride, norm->k_stride, norm->eps};
        KV_TRY(lora::launch_append_heads(h, c.dtype, kv->e4m3(), st));
    } else {
        KV_TRY(lora::launch_append(k, c.dtype, st));
    }
    return LORA_OK;
}

int lora_kv_attend(lora_kv_t *kv, lora_kv_batch_t *handle, int32_t layer, const void *q, int64_t q_stride, void *out, int64_t out_stride, float scale,
                   void *stream)
{
    Batch *const batch = kv ? find_batch(*kv, handle) : nullptr;
    if (!batch || layer < 0 || layer >= kv->cfg.n_layers) return LORA_E_INVAL;
    if (batch->stale) return LORA_E_STATE;
    const lora_kv_config_t &c = kv->cfg;
    const float scale_log2 = scale * 1.44269504088896340736f;
    if (!(scale > 0.f) || !std::isfinite(scale_log2)) return LORA_E_INVAL;
    if (!batch->info.n_tokens) return LORA_OK;
    const int64_t row = (int64_t)c.n_heads * c.head_dim, u = kv->row_chunk();
    const auto bad = [&](const void *p, int64_t stride) { return !p || !aligned16(p) || stride < row || stride % u || stride > ((int64_t)1 << 40); };
    if (bad(q, q_stride) || bad(out, out_stride) || (q == out && q_stride != out_stride)) return LORA_E_INVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    const OnDevice on(*kv);
    if (const int rc = in_order(*kv, st)) return rc;
    lora::AttnArgs a{};
    a.q = q, a.out = out, a.q_stride = q_stride, a.out_stride = out_stride;
    a.pages = kv->pages + kv->layer_bytes * layer;
    a.page_stride = (int64_t)kv->page_bytes;
    a.page_list = reinterpret_cast<const int32_t *>(batch->dev + batch->off_pages);
    a.row_tokens = reinterpret_cast<const int32_t *>(batch->dev + batch->off_row_tokens);
    a.prefixes = batch->n_shared_joins != 0, a.exact = batch->exact;
    a.part_o = kv->part_o, a.part_ml = kv->part_ml;
    a.scale_log2 = scale_log2;
    a.n_kv = c.n_kv_heads, a.group = kv->group(), a.page_shift = kv->page_shift;
    a.tiles = reinterpret_cast<const AttnItem *>(batch->dev + batch->off_tiles);
    a.rows = reinterpret_cast<const AttnItem *>(batch->dev + batch->off_rows);
    a.n_tiles = batch->info.n_tile_items;
    a.n_rows = batch->info.n_row_items - batch->info.n_short_items;
    a.n_short = batch->info.n_short_items;
    const lora::KvTiles way = (lora::KvTiles)batch->info.tiles_way;
    if (kv->e4m3()) KV_TRY(lora::launch_attn_e4m3(a, c.head_dim, way, kv->n_cu, st));
    else KV_TRY(lora::launch_attn(a, c.dtype, c.head_dim, way, kv->n_cu, st));
    lora::JoinArgs j{};
    j.out = out, j.out_stride = out_stride;
    j.part_o = kv->part_o, j.part_ml = kv->part_ml;
    j.n_kv = c.n_kv_heads, j.group = kv->group();
    if (batch->n_joins) {
        j.items = reinterpret_cast<const JoinItem *>(batch->dev + batch->off_joins);
        j.n_items = batch->n_joins, j.max_rows = batch->join_rows;
        KV_TRY(lora::launch_attn_join(j, c.dtype, c.head_dim, false, st));
    }
    if (batch->n_tile_joins) {
        j.items = reinterpret_cast<const JoinItem *>(batch->dev + batch->off_tile_joins);
        j.n_items = batch->n_tile_joins, j.max_rows = way == lora::KV_TILES_TURNS ? lora::KV_TURNS_TILE : lora::KV_TILE;
        KV_TRY(lora::launch_attn_join(j, c.dtype, c.head_dim, true, st));
    }
    if (batch->n_shared_joins) {
        lora::SharedJoinArgs h{};
        h.out = out, h.out_stride = out_stride;
        h.items = reinterpret_cast<const SharedJoin *>(batch->dev + batch->off_shared_joins);
        h.sources = reinterpret_cast<const SharedSource *>(batch->dev + batch->off_sources);
        h.blocks = reinterpret_cast<const SharedBlock *>(batch->dev + batch->off_blocks);
        h.part_o = kv->part_o, h.part_ml = kv->part_ml;
        h.n_items = batch->n_shared_joins, h.n_kv = c.n_kv_heads, h.group = kv->group(), h.max_rows = batch->shared_rows;
        KV_TRY(lora::launch_shared_join(h, c.dtype, c.head_dim, st));
    }
    return LORA_OK;
}

}  // extern "C"
