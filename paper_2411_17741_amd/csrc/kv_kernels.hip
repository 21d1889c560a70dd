// The paged key-value cache's writes (gfx950): new keys and values into the pages with their positions turned, and
// pages copied to others.  Both only move bytes; the layout of the pages is in include/lora_kv.h.
#include <algorithm>

#include "kv_internal.h"
#include "lora_device.h"
#include "lora_internal.h"

namespace lora {

namespace {

template <typename E> constexpr int CHUNK = 16 / (int)sizeof(E);  // values of a 16-byte chunk

template <typename E> struct alignas(16) Vals {
    E v[CHUNK<E>];
};

// 16 bytes, past the caches with PAST: what is read once, and what is written here to be read when much else has been
typedef uint32_t Words __attribute__((ext_vector_type(4)));
template <bool PAST, typename E> __device__ __forceinline__ Vals<E> load_once(const E *p)
{
    if constexpr (PAST) return __builtin_bit_cast(Vals<E>, __builtin_nontemporal_load(reinterpret_cast<const Words *>(p)));
    else return *reinterpret_cast<const Vals<E> *>(p);
}
template <bool PAST, typename E> __device__ __forceinline__ void store_past(E *p, const Vals<E> &v)
{
    if constexpr (PAST) __builtin_nontemporal_store(__builtin_bit_cast(Words, v), reinterpret_cast<Words *>(p));
    else *reinterpret_cast<Vals<E> *>(p) = v;
}

}  // namespace

// Keys and queries: a thread takes two chunks of one token whose values turn together (HALVES: chunk p and the one rope_dim / 2 values on;
// NEIGHBOURS and unturned values: two chunks in a row), of HEADS heads: the position's cosines and sines are fetched once for
// them.  8 tokens go with a run of 8 threads: a token's key chunks lie page_tokens chunks apart in the page, the same chunk of
// the next token right beside, so that a prompt is read and written in runs of 128 bytes.
// Values: a thread takes u values of a head of the tokens that share their chunks, turns the u x u square round in its registers,
// and the wavefront hands the chunks round through LDS to store them 1 KB at a time; chunks that this group does not fill
// are written value by value.
//
// Only bytes move.  Large batches: 8 heads a thread, past the caches, 12900 tokens of 32 + 32 + 32 heads of 128 (650 MB) in 160 us, 4.1 TB/s (172 with 4 heads).  Small ones, which stay in the
// caches until the attention reads them: 2 heads a thread and no such hints, 920 tokens of 32 + 32 + 32 heads 19.9 -> 18.5 us, with their attention, two layers, 187 -> 182; 64 tokens 5.9 us of kernel time.
// From 16 MB of rows on the former is faster (6 x 300 tokens, 2 -> 8 heads a thread 26.0 -> 23.3, two layers with their attention 99.7 -> 85.4).  Of batches of single tokens every key chunk is a piece of 16 bytes of a line of its own, every value one of 2.
constexpr int APPEND_MANY_HEADS = 8, APPEND_FEW_HEADS = 2;
constexpr int64_t APPEND_MANY = 1 << 24;  // bytes of keys and queries from which a batch is a large one

template <typename E, int APPEND_HEADS>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a, uint32_t key_blocks)
{
    constexpr int U = CHUNK<E>;
    constexpr bool PAST = APPEND_HEADS == APPEND_MANY_HEADS;
    const int page_tokens = 1 << a.page_shift;
    const size_t head_values = (size_t)a.dim << a.page_shift;  // of one half of a page
    if (blockIdx.x < key_blocks) {
        const int n_pairs = a.dim / (2 * U);
        uint32_t i = blockIdx.x * 256u + threadIdx.x;
        const int t8 = i & 7;
        i >>= 3;
        const int p = i % n_pairs;
        i /= n_pairs;
        const int heads = (a.q ? a.n_heads : 0) + a.n_kv, head_groups = (heads + APPEND_HEADS - 1) / APPEND_HEADS;
        const int h0 = i % head_groups * APPEND_HEADS;
        const int t = (int)(i / head_groups) * 8 + t8;
        if (t >= a.n_tokens) return;
        const KvToken tok = a.tokens[t];
        const int turned = a.rope_dim / (2 * U);  // pairs of chunks that turn
        const bool turn = p < turned, halves = turn && !a.neighbours;
        const int c0 = halves ? p : 2 * p, c1 = halves ? p + turned : 2 * p + 1;
        // keys come first, then queries
        const auto source = [&](int h) {
            return h < a.n_kv ? static_cast<const E *>(a.k) + t * a.k_stride + h * a.dim : static_cast<const E *>(a.q) + t * a.q_stride + (h - a.n_kv) * a.dim;
        };
        Vals<E> x[APPEND_HEADS], y[APPEND_HEADS];
#pragma unroll
        for (int k = 0; k < APPEND_HEADS; ++k) {
            const E *src = source(min(h0 + k, heads - 1));
            x[k] = load_once<PAST>(src + c0 * U);
            y[k] = load_once<PAST>(src + c1 * U);
        }
        if (turn) {
            // HALVES: entries c0 U .. c0 U + U - 1 turn x with y; NEIGHBOURS: entries p U .. turn the pairs of x, then those of y
            float c[U], s[U];
            const float *cs = a.rope + (size_t)tok.pos * a.rope_dim + p * U, *sn = cs + a.rope_dim / 2;
#pragma unroll
            for (int e = 0; e < U; ++e) c[e] = cs[e], s[e] = sn[e];
            if (halves) {
#pragma unroll
                for (int k = 0; k < APPEND_HEADS; ++k)
#pragma unroll
                    for (int e = 0; e < U; ++e) {
                        const float u = (float)x[k].v[e], w = (float)y[k].v[e];
                        x[k].v[e] = (E)(u * c[e] - w * s[e]);
                        y[k].v[e] = (E)(w * c[e] + u * s[e]);
                    }
            } else {
                const auto pairs = [&](Vals<E> &z, int first) {
#pragma unroll
                    for (int e = 0; e < U; e += 2) {
                        const float u = (float)z.v[e], w = (float)z.v[e + 1];
                        z.v[e] = (E)(u * c[first + e / 2] - w * s[first + e / 2]);
                        z.v[e + 1] = (E)(w * c[first + e / 2] + u * s[first + e / 2]);
                    }
                };
#pragma unroll
                for (int k = 0; k < APPEND_HEADS; ++k) pairs(x[k], 0), pairs(y[k], U / 2);
            }
        }
#pragma unroll
        for (int k = 0; k < APPEND_HEADS; ++k) {
            const int h = h0 + k;
            if (h < a.n_kv) {
                E *page = reinterpret_cast<E *>(a.pages + tok.page * a.page_stride) + h * head_values + (size_t)(tok.pos & (page_tokens - 1)) * U;
                *reinterpret_cast<Vals<E> *>(page + ((size_t)c0 << a.page_shift) * U) = x[k];
                *reinterpret_cast<Vals<E> *>(page + ((size_t)c1 << a.page_shift) * U) = y[k];
            } else if (h < heads) {
                E *to = static_cast<E *>(a.q_out) + t * a.q_out_stride + (h - a.n_kv) * a.dim;
                store_past<PAST>(to + c0 * U, x[k]);
                store_past<PAST>(to + c1 * U, y[k]);
            }
        }
        return;
    }
    __shared__ Vals<E> turned[4][64 * U];
    const int n_chunks = a.dim / U, lane = threadIdx.x & 63;
    uint32_t i = (blockIdx.x - key_blocks) * 256u + threadIdx.x;
    const int c = i % n_chunks;
    i /= n_chunks;
    const int h = i % a.n_kv;
    const int g = i / a.n_kv;
    KvGroup grp{0, 0, 0, 0};
    if (g < a.n_groups) grp = a.groups[g];
    const E *src = static_cast<const E *>(a.v) + (int64_t)grp.tok * a.v_stride + h * a.dim + c * U;
    const int at = grp.pos & (page_tokens - 1);
    E *to = reinterpret_cast<E *>(a.pages + grp.page * a.page_stride) + (a.n_kv + h) * head_values + (size_t)(at / U) * a.dim * U;  // the chunks of value 0, 1, ... of the head
    Vals<E> *const mine = turned[threadIdx.x >> 6];
    if (grp.n == U) {
        Vals<E> in[U];
#pragma unroll
        for (int t = 0; t < U; ++t) in[t] = load_once<PAST>(src + t * a.v_stride);
#pragma unroll
        for (int d = 0; d < U; ++d) {
            Vals<E> o;
#pragma unroll
            for (int t = 0; t < U; ++t) o.v[t] = in[t].v[d];
            mine[lane * U + (d ^ (lane & (U - 1)))] = o;  // (a lane's chunks in an order of its own: the lanes' banks differ)
        }
    } else {
        for (int t = 0; t < grp.n; ++t) {
            const Vals<E> in = load_once<PAST>(src + t * a.v_stride);
#pragma unroll
            for (int d = 0; d < U; ++d) to[(c * U + d) * U + at % U + t] = in.v[d];
        }
    }
    __builtin_amdgcn_wave_barrier();
    // chunk n of the wavefront's 64 u is lane n / u's; the 64 / u lanes of a store belong to one group and head (dim is a multiple of 64)
    const uint64_t base = reinterpret_cast<uint64_t>(to);
#pragma unroll
    for (int k = 0; k < U; ++k) {
        const int from = k * (64 / U), owner = from + lane / U;
        const bool whole = __builtin_amdgcn_readlane(grp.n, from) == U;
        const uint64_t there = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(base >> 32), from) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)base, from);
        const int first = __builtin_amdgcn_readlane(c, from) * U;
        if (whole) store_past<PAST>(reinterpret_cast<E *>(there) + (first + lane) * U, mine[owner * U + ((lane & (U - 1)) ^ (owner & (U - 1)))]);
    }
}

hipError_t launch_append(const AppendArgs &a, int dtype, hipStream_t st)
{
    const int u = dtype == LORA_BF16 ? 8 : 4;
    const int64_t heads = (a.q ? a.n_heads : 0) + a.n_kv;
    const bool many = a.n_tokens * heads * a.dim * (dtype == LORA_BF16 ? 2 : 4) >= APPEND_MANY;
    const int64_t each = many ? APPEND_MANY_HEADS : APPEND_FEW_HEADS;
    const int64_t keys = ((int64_t)(a.n_tokens + 7) / 8 * ((heads + each - 1) / each) * (a.dim / (2 * u)) * 8 + 255) / 256;
    const int64_t vals = ((int64_t)a.n_groups * a.n_kv * (a.dim / u) + 255) / 256;
    if (keys * 256 > UINT32_MAX || vals * 256 > UINT32_MAX || keys + vals > INT32_MAX) return hipErrorInvalidValue;
    const dim3 grid((unsigned)(keys + vals));
    if (dtype == LORA_BF16) {
        if (many) hipLaunchKernelGGL((append_kernel<__bf16, APPEND_MANY_HEADS>), grid, dim3(256), 0, st, a, (uint32_t)keys);
        else hipLaunchKernelGGL((append_kernel<__bf16, APPEND_FEW_HEADS>), grid, dim3(256), 0, st, a, (uint32_t)keys);
    } else {
        if (many) hipLaunchKernelGGL((append_kernel<float, APPEND_MANY_HEADS>), grid, dim3(256), 0, st, a, (uint32_t)keys);
        else hipLaunchKernelGGL((append_kernel<float, APPEND_FEW_HEADS>), grid, dim3(256), 0, st, a, (uint32_t)keys);
    }
    return hipGetLastError();
}

// A page's bytes, all layers, in pieces of 16 KB: a block each, 4 chunks of 16 bytes in flight per thread.  4 pages of 34 MB that are copies
// of one: 34 us, written past the caches at 3.9 TB/s and read from them.
constexpr int MOVE_BYTES = 256 * 4 * 16;

// A batch's lists go up with its copies (row n of the grid): a launch less, 8 forks of a request of 487 tokens with 6 / 2 heads, 8 layers, 12.6 -> 10.2 us.
__global__ __launch_bounds__(256) void moves_kernel(KvMoves m, int n, char *pages, int64_t page_stride, KvLists lists)
{
    if ((int)blockIdx.y == n) {
        for (uint32_t i = blockIdx.x * 256u + threadIdx.x; i < lists.n; i += gridDim.x * 256u) static_cast<Words *>(lists.to)[i] = static_cast<const Words *>(lists.from)[i];
        return;
    }
    const int64_t at = (int64_t)blockIdx.x * MOVE_BYTES + threadIdx.x * 16;
    const char *from = pages + m.from[blockIdx.y] * page_stride;
    char *to = pages + m.to[blockIdx.y] * page_stride;
    Words v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (at + i * 4096 < page_stride) v[i] = *reinterpret_cast<const Words *>(from + at + i * 4096);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (at + i * 4096 < page_stride) __builtin_nontemporal_store(v[i], reinterpret_cast<Words *>(to + at + i * 4096));
}

hipError_t launch_moves(const KvMoves &m, int n, char *pages, int64_t page_stride, const KvLists &lists, hipStream_t st, hipEvent_t done)
{
    const int64_t blocks = std::max((page_stride + MOVE_BYTES - 1) / MOVE_BYTES, (int64_t)(lists.n + 255) / 256);
    if (blocks > INT32_MAX || n > KV_MAX_MOVES) return hipErrorInvalidValue;
    launch_k(nullptr, done, 0, moves_kernel, dim3((unsigned)blocks, (unsigned)(n + (lists.n != 0))), dim3(256), 0, st, m, n, pages, page_stride, lists);
    return hipGetLastError();
}

}  // namespace lora
