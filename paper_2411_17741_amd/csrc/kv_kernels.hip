// The paged key-value cache's writes (gfx950): new keys and values into the pages with their positions turned, and
// pages copied to others.  Both only move bytes; the layout of the pages is in include/lora_kv.h.
#include "kv_internal.h"
#include "lora_device.h"

namespace lora {

namespace {

template <typename E> constexpr int CHUNK = 16 / (int)sizeof(E);  // values of a 16-byte chunk

template <typename E> struct alignas(16) Vals {
    E v[CHUNK<E>];
};

}  // namespace

// Keys and queries: a thread takes two chunks of one head of one token whose values turn together (HALVES: chunk p and the one rope_dim / 2
// values on; NEIGHBOURS and unturned values: two chunks in a row).  8 tokens go with a run of 8 threads: a token's key chunks
// lie page_tokens chunks apart in the page, the same chunk of the next token right beside, so that a prompt is read and
// written in runs of 128 bytes.
// Values: a thread takes u values of a head of the tokens that share their chunks, turns the u x u square round in its registers
// and writes u chunks that lie in a row; chunks that are not filled by this group are written value by value.
template <typename E>
__global__ __launch_bounds__(256) void append_kernel(AppendArgs a, uint32_t key_blocks)
{
    constexpr int U = CHUNK<E>;
    const int page_tokens = 1 << a.page_shift;
    const size_t head_values = (size_t)a.dim << a.page_shift;  // of one half of a page
    if (blockIdx.x < key_blocks) {
        const int n_pairs = a.dim / (2 * U);
        uint32_t i = blockIdx.x * 256u + threadIdx.x;
        const int t8 = i & 7;
        i >>= 3;
        const int p = i % n_pairs;
        i /= n_pairs;
        const int heads = (a.q ? a.n_heads : 0) + a.n_kv;
        int h = i % heads;
        const int t = (int)(i / heads) * 8 + t8;
        if (t >= a.n_tokens) return;
        const bool is_key = h < a.n_kv;
        if (!is_key) h -= a.n_kv;
        const KvToken tok = a.tokens[t];
        const E *src = is_key ? static_cast<const E *>(a.k) + t * a.k_stride : static_cast<const E *>(a.q) + t * a.q_stride;
        src += h * a.dim;
        const int turned = a.rope_dim / (2 * U);  // pairs of chunks that turn
        const bool turn = p < turned, halves = turn && !a.neighbours;
        const int c0 = halves ? p : 2 * p, c1 = halves ? p + turned : 2 * p + 1;
        Vals<E> x = *reinterpret_cast<const Vals<E> *>(src + c0 * U), y = *reinterpret_cast<const Vals<E> *>(src + c1 * U);
        if (turn) {
            const float *cs = a.rope + (size_t)tok.pos * a.rope_dim, *sn = cs + a.rope_dim / 2;
            if (halves) {
#pragma unroll
                for (int e = 0; e < U; ++e) {
                    const float c = cs[c0 * U + e], s = sn[c0 * U + e], u = (float)x.v[e], w = (float)y.v[e];
                    x.v[e] = (E)(u * c - w * s);
                    y.v[e] = (E)(w * c + u * s);
                }
            } else {
#pragma unroll
                for (int e = 0; e < U; e += 2) {
                    const auto pair = [&](Vals<E> &z, int chunk) {
                        const int j = (chunk * U + e) / 2;
                        const float c = cs[j], s = sn[j], u = (float)z.v[e], w = (float)z.v[e + 1];
                        z.v[e] = (E)(u * c - w * s);
                        z.v[e + 1] = (E)(w * c + u * s);
                    };
                    pair(x, c0);
                    pair(y, c1);
                }
            }
        }
        if (is_key) {
            E *page = reinterpret_cast<E *>(a.pages + tok.page * a.page_stride) + h * head_values + (size_t)(tok.pos & (page_tokens - 1)) * U;
            *reinterpret_cast<Vals<E> *>(page + ((size_t)c0 << a.page_shift) * U) = x;
            *reinterpret_cast<Vals<E> *>(page + ((size_t)c1 << a.page_shift) * U) = y;
        } else {
            E *to = static_cast<E *>(a.q_out) + t * a.q_out_stride + h * a.dim;
            *reinterpret_cast<Vals<E> *>(to + c0 * U) = x;
            *reinterpret_cast<Vals<E> *>(to + c1 * U) = y;
        }
        return;
    }
    const int n_chunks = a.dim / U;
    uint32_t i = (blockIdx.x - key_blocks) * 256u + threadIdx.x;
    const int c = i % n_chunks;
    i /= n_chunks;
    const int h = i % a.n_kv;
    const int g = i / a.n_kv;
    if (g >= a.n_groups) return;
    const KvGroup grp = a.groups[g];
    const E *src = static_cast<const E *>(a.v) + (int64_t)grp.tok * a.v_stride + h * a.dim + c * U;
    const int at = grp.pos & (page_tokens - 1);
    E *to = reinterpret_cast<E *>(a.pages + grp.page * a.page_stride) + (a.n_kv + h) * head_values + ((size_t)(at / U) * a.dim + c * U) * U;
    if (grp.n == U) {
        Vals<E> in[U];
#pragma unroll
        for (int t = 0; t < U; ++t) in[t] = *reinterpret_cast<const Vals<E> *>(src + t * a.v_stride);
#pragma unroll
        for (int d = 0; d < U; ++d) {
            Vals<E> o;
#pragma unroll
            for (int t = 0; t < U; ++t) o.v[t] = in[t].v[d];
            *reinterpret_cast<Vals<E> *>(to + d * U) = o;
        }
    } else {
        for (int t = 0; t < grp.n; ++t) {
            const Vals<E> in = *reinterpret_cast<const Vals<E> *>(src + t * a.v_stride);
#pragma unroll
            for (int d = 0; d < U; ++d) to[d * U + at % U + t] = in.v[d];
        }
    }
}

hipError_t launch_append(const AppendArgs &a, int dtype, hipStream_t st)
{
    const int u = dtype == LORA_BF16 ? 8 : 4;
    const int64_t heads = (a.q ? a.n_heads : 0) + a.n_kv;
    const int64_t keys = ((int64_t)(a.n_tokens + 7) / 8 * heads * (a.dim / (2 * u)) * 8 + 255) / 256;
    const int64_t vals = ((int64_t)a.n_groups * a.n_kv * (a.dim / u) + 255) / 256;
    if (keys * 256 > UINT32_MAX || vals * 256 > UINT32_MAX || keys + vals > INT32_MAX) return hipErrorInvalidValue;
    const dim3 grid((unsigned)(keys + vals));
    if (dtype == LORA_BF16) hipLaunchKernelGGL((append_kernel<__bf16>), grid, dim3(256), 0, st, a, (uint32_t)keys);
    else hipLaunchKernelGGL((append_kernel<float>), grid, dim3(256), 0, st, a, (uint32_t)keys);
    return hipGetLastError();
}

// A page's bytes, all layers, in pieces of 16 KB: a block each, 4 chunks of 16 bytes in flight per thread.
constexpr int MOVE_BYTES = 256 * 4 * 16;

__global__ __launch_bounds__(256) void moves_kernel(KvMoves m, char *pages, int64_t page_stride)
{
    const int64_t at = (int64_t)blockIdx.x * MOVE_BYTES + threadIdx.x * 16;
    const char *from = pages + m.from[blockIdx.y] * page_stride;
    char *to = pages + m.to[blockIdx.y] * page_stride;
    uint4 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (at + i * 4096 < page_stride) v[i] = *reinterpret_cast<const uint4 *>(from + at + i * 4096);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (at + i * 4096 < page_stride) *reinterpret_cast<uint4 *>(to + at + i * 4096) = v[i];
}

hipError_t launch_moves(const KvMoves &m, int n, char *pages, int64_t page_stride, hipStream_t st)
{
    const int64_t blocks = (page_stride + MOVE_BYTES - 1) / MOVE_BYTES;
    if (blocks > INT32_MAX || n > KV_MAX_MOVES) return hipErrorInvalidValue;
    hipLaunchKernelGGL(moves_kernel, dim3((unsigned)blocks, (unsigned)n), dim3(256), 0, st, m, pages, page_stride);
    return hipGetLastError();
}

}  // namespace lora
