// The paged key-value cache's writes (gfx950): new keys and values into the pages with their positions turned, with norms of their
// heads and as 8-bit values where that is asked for, and pages copied to others; and what the pages hold read back.  Memory bounds all of it; the
// layout of the pages is in include/lora_kv.h.
#include <algorithm>
#include <type_traits>

#include "kv_e4m3.h"
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

// A block's share of the values; `mine`: 64 u chunks of LDS for the wavefront
template <typename E, bool PAST>
__device__ __forceinline__ void append_values(const AppendArgs &a, uint32_t block, Vals<E> *mine)
{
    constexpr int U = CHUNK<E>;
    const int page_tokens = 1 << a.page_shift;
    const size_t head_values = (size_t)a.dim << a.page_shift;  // of one half of a page
    const int n_chunks = a.dim / U, lane = threadIdx.x & 63;
    uint32_t i = block * 256u + threadIdx.x;
    const int c = i % n_chunks;
    i /= n_chunks;
    const int h = i % a.n_kv;
    const int g = i / a.n_kv;
    KvGroup grp{0, 0, 0, 0};
    if (g < a.n_groups) grp = a.groups[g];
    const E *src = static_cast<const E *>(a.v) + (int64_t)grp.tok * a.v_stride + h * a.dim + c * U;
    const int at = grp.pos & (page_tokens - 1);
    E *to = reinterpret_cast<E *>(a.pages + grp.page * a.page_stride) + (a.n_kv + h) * head_values + (size_t)(at / U) * a.dim * U;  // the chunks of value 0, 1, ... of the head
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
    append_values<E, PAST>(a, blockIdx.x - key_blocks, turned[threadIdx.x >> 6]);
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

// The same with norms of the heads, and into pages of 8-bit values.  A token's part of a head is dim / (2 u) threads' of one wavefront, which find the
// sum of its squares, or the largest of its values, between them by a few exchanges.
//
// 8 bits: a value that is beside a border between two of them goes the wrong way if what it is made of was rounded before, and is off by 2^-4 of itself then:
// keys are normed and turned in 64 bits (the products of a key without a norm and of 24-bit cosines and sines are exact there), and rounded to the nearest of 8 bits by way of fp32
// values that are rounded to odd -- towards zero, with the last bit set if anything was lost --, which leaves the second rounding what it has to know.
//
// Bound by memory in large batches: 4291 tokens of 32 + 8 + 8 heads of 128, normed, 108 MB, in 28.8 us, 3.7 TB/s (all squares in 64 bits and weights fetched head by head 36); 2544 of 64 + 8 + 8 into 8 bits, 92 MB, 26.5.  Small ones by trips to
// memory: one token of 40 + 40 + 40 heads 3.7 us, 297 of 32 + 8 + 8, normed, into 8 bits 7.9.
__device__ __forceinline__ float to_odd(double d)
{
    const float f = (float)d;
    const double lost = d - (double)f;
    uint32_t b = __float_as_uint(f);
    if ((lost < 0. || lost > 0.) && !(b & 1) && f != 0.f) b += (lost > 0.) == (f > 0.f) ? 1 : -1;
    return __uint_as_float(b);
}

// the largest |value| of those that are finite
__device__ __forceinline__ float larger(float top, float v)
{
    const float size = fabsf(v);
    return size < INFINITY && size > top ? size : top;
}

// The smallest e with top <= 448 * 2^e: 448 is 1.75 * 2^8, so a fraction over 1.75 takes one more
__device__ __forceinline__ int exponent_for(float top)
{
    return min(max((int)((__float_as_uint(top) + 0x1fffffu) >> 23) - 127 - 8, KV_EXP_MIN), KV_EXP_MAX);
}

// Four values of 448 at most to 8 bits (what is infinite or no number becomes no number)
__device__ __forceinline__ uint32_t four_e4m3(float a, float b, float c, float d)
{
    const int low = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, low, true);
}

// x and y of a thread, U values each, turned: the same roundings whatever is compiled beside it, and append_kernel's
__device__ __forceinline__ float fused(float a, float b, float c) { return __builtin_fmaf(a, b, c); }
__device__ __forceinline__ double fused(double a, double b, double c) { return __builtin_fma(a, b, c); }
template <typename T, int U>
__device__ __forceinline__ void turn_pairs(T (&x)[U], T (&y)[U], const float (&c)[U], const float (&s)[U], bool halves)
{
    if (halves) {
#pragma unroll
        for (int e = 0; e < U; ++e) {
            const T u = x[e], w = y[e];
            x[e] = fused(u, (T)c[e], -(w * s[e]));
            y[e] = fused(w, (T)c[e], u * s[e]);
        }
    } else {
        const auto pairs = [&](T(&z)[U], int first) {
#pragma unroll
            for (int e = 0; e < U; e += 2) {
                const T u = z[e], w = z[e + 1];
                z[e] = fused(u, (T)c[first + e / 2], -(w * s[first + e / 2]));
                z[e + 1] = fused(w, (T)c[first + e / 2], u * s[first + e / 2]);
            }
        };
        pairs(x, 0), pairs(y, U / 2);
    }
}

// The largest of two tokens' values each, over the lanes that have the other values of the head (`lanes` beside each other: 16, 32 or 64)
typedef unsigned short Sizes __attribute__((ext_vector_type(2)));
__device__ __forceinline__ Sizes largest(Sizes v, int lanes)
{
    const auto with = [&](auto ctrl) {
        v = __builtin_elementwise_max(v, __builtin_bit_cast(Sizes, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), decltype(ctrl)::value, 0xF, 0xF, true)));
    };
    with(std::integral_constant<int, 0xB1>{});   // the neighbour
    with(std::integral_constant<int, 0x4E>{});   // two lanes on
    with(std::integral_constant<int, 0x141>{});  // the other four of eight
    with(std::integral_constant<int, 0x140>{});  // the other eight of 16
    const auto far = [&](int off) { v = __builtin_elementwise_max(v, __builtin_bit_cast(Sizes, __shfl_xor(__builtin_bit_cast(int, v), off, 64))); };
    if (lanes > 16) far(16);
    if (lanes > 32) far(32);
    return v;
}

// A block's share of the values into pages of 8 bits: a thread takes 4 values of a head of up to 16 tokens that share their chunks (8 values: 185 registers instead of 100 and half the
// wavefronts).  bf16 values compare as whole numbers without their sign, two tokens at a time.
constexpr int VALUES_E4M3 = 4;
__device__ __forceinline__ void append_values_e4m3(const AppendArgs &a, uint32_t block)
{
    constexpr int U = VALUES_E4M3, N = 16;
    const int lanes = a.dim / U;  // that have a head's values
    uint32_t i = block * 256u + threadIdx.x;
    const int c = i % lanes;
    i /= lanes;
    const int h = i % a.n_kv;
    const int g = i / a.n_kv;
    KvGroup grp{0, 0, 0, 0};
    if (g < a.n_groups) grp = a.groups[g];
    const __bf16 *src = static_cast<const __bf16 *>(a.v) + (int64_t)grp.tok * a.v_stride + h * a.dim + c * U;
    const int at = grp.pos & ((1 << a.page_shift) - 1), first = at % N;
    char *const page = a.pages + grp.page * a.page_stride;
    const size_t head_values = (size_t)a.dim << a.page_shift;
    uint8_t *to = reinterpret_cast<uint8_t *>(page) + (a.n_kv + h) * head_values + (size_t)(at / N) * a.dim * N + c * U * N;
    uint8_t *exps = reinterpret_cast<uint8_t *>(page) + 2 * a.n_kv * head_values + ((size_t)(a.n_kv + h) << a.page_shift) + at;
    const auto size = [](uint32_t two) {  // of two values; of those that are infinite or no number 0
        Sizes v = __builtin_bit_cast(Sizes, two & 0x7fff7fffu);
        v[0] = v[0] < 0x7f80 ? v[0] : 0, v[1] = v[1] < 0x7f80 ? v[1] : 0;
        return v;
    };
    const auto top_of = [&](const uint2 &x) {
        const Sizes m = __builtin_elementwise_max(size(x.x), size(x.y));
        return m[0] > m[1] ? m[0] : m[1];
    };
    const auto exponent = [](unsigned short top) { return exponent_for(__uint_as_float((uint32_t)top << 16)); };
    const auto value = [](const uint2 &x, int d) { return d == 0 ? bf_lo(x.x) : d == 1 ? bf_hi(x.x) : d == 2 ? bf_lo(x.y) : bf_hi(x.y); };
    // Groups of more than a token or two: all tokens at once, by their places in the chunks.  What is not theirs in a chunk stays what it is (nobody else writes there now).
    if (__any(grp.n > 2)) {
        uint2 in[N];
        float unit[N];
        uint32_t e4[N / 4] = {};
#pragma unroll
        for (int t = 0; t < N; ++t) {
            in[t] = make_uint2(0, 0);
            if (t >= first && t < first + grp.n) in[t] = *reinterpret_cast<const uint2 *>(src + (t - first) * a.v_stride);
        }
#pragma unroll
        for (int t = 0; t < N; t += 2) {
            const Sizes top = largest(Sizes{top_of(in[t]), top_of(in[t + 1])}, lanes);
            const int e0 = exponent(top[0]), e1 = exponent(top[1]);
            unit[t] = unit_of(KV_EXP_BIAS - e0), unit[t + 1] = unit_of(KV_EXP_BIAS - e1);
            e4[t / 4] |= (uint32_t)(e0 + KV_EXP_BIAS | (e1 + KV_EXP_BIAS) << 8) << t % 4 * 8;
        }
        if (!grp.n) return;
        const bool whole = grp.n == N;
        uint4 chunk[U];
#pragma unroll
        for (int d = 0; d < U; ++d) {
            const auto four = [&](int t) {
                return four_e4m3(value(in[t], d) * unit[t], value(in[t + 1], d) * unit[t + 1], value(in[t + 2], d) * unit[t + 2], value(in[t + 3], d) * unit[t + 3]);
            };
            chunk[d] = make_uint4(four(0), four(4), four(8), four(12));
        }
        uint4 e = make_uint4(e4[0], e4[1], e4[2], e4[3]), *const e_to = reinterpret_cast<uint4 *>(exps - first);
        if (!whole) {
            // the bytes of dword w that are the group's
            const auto mine = [&](int w) {
                const int from = min(max(first - 4 * w, 0), 4), to = min(max(first + grp.n - 4 * w, 0), 4);
                const auto below = [](int n) { return n == 4 ? ~0u : (1u << n * 8) - 1u; };
                return below(to) & ~below(from);
            };
            const uint32_t m[4] = {mine(0), mine(1), mine(2), mine(3)};
            const auto merge = [&](uint4 &v, const uint4 &before) {
                v = make_uint4((v.x & m[0]) | (before.x & ~m[0]), (v.y & m[1]) | (before.y & ~m[1]), (v.z & m[2]) | (before.z & ~m[2]), (v.w & m[3]) | (before.w & ~m[3]));
            };
            uint4 old[U], old_e = make_uint4(0, 0, 0, 0);
#pragma unroll
            for (int d = 0; d < U; ++d) old[d] = *reinterpret_cast<const uint4 *>(to + d * N);
            if (c == 0) old_e = *e_to;
#pragma unroll
            for (int d = 0; d < U; ++d) merge(chunk[d], old[d]);
            merge(e, old_e);
        }
#pragma unroll
        for (int d = 0; d < U; ++d) *reinterpret_cast<uint4 *>(to + d * N) = chunk[d];
        if (c == 0) *e_to = e;
        return;
    }
#pragma unroll 1
    for (int t = 0; t < grp.n; ++t) {
        const uint2 x = *reinterpret_cast<const uint2 *>(src + t * a.v_stride);
        const int e = exponent(largest(Sizes{top_of(x), 0}, lanes)[0]);
        const float unit = unit_of(KV_EXP_BIAS - e);
        if (c == 0) exps[t] = (uint8_t)(e + KV_EXP_BIAS);
        const uint32_t v = four_e4m3(value(x, 0) * unit, value(x, 1) * unit, value(x, 2) * unit, value(x, 3) * unit);
#pragma unroll
        for (int d = 0; d < U; ++d) to[d * N + first + t] = (uint8_t)(v >> d * 8);
    }
}

// The sum over lanes `tokens` (4, 8 or 16) apart
__device__ __forceinline__ float over_pairs(float v, int tokens)
{
    const auto row = [&](auto ctrl) { v += __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), decltype(ctrl)::value, 0xF, 0xF, true)); };
    if (tokens < 16) row(std::integral_constant<int, 0x128>{});  // 16 lanes turned by 8
    if (tokens < 8) row(std::integral_constant<int, 0x124>{});
    const auto near = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = __uint_as_float(near[0]) + __uint_as_float(near[1]);
    const auto far = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(far[0]) + __uint_as_float(far[1]);
}

// Heads of a thread, all of whose values are on their way at once.  4291 tokens of 32 + 8 + 8 heads, normed: 2 heads 31.3 us, 4 29.4, 8 28.5; 2544 of 64 + 8 + 8 into 8 bits, whose keys take more registers, 31.9, 29.0, 32.1.
// Small batches (as the append above tells them apart) a head a thread.
constexpr int NORM_MANY_HEADS = 4, NORM_FEW_HEADS = 1;
template <typename E, bool E8, bool NORM, int HEADS>
__global__ __launch_bounds__(256) void append_heads_kernel(AppendHeadsArgs n, uint32_t key_blocks)
{
    constexpr int U = CHUNK<E>;
    constexpr bool PAST = HEADS > 1;
    const AppendArgs &a = n.a;
    if (blockIdx.x >= key_blocks) {
        if constexpr (E8) {
            append_values_e4m3(a, blockIdx.x - key_blocks);
        } else {
            __shared__ Vals<E> turned[4][64 * U];
            append_values<E, PAST>(a, blockIdx.x - key_blocks, turned[threadIdx.x >> 6]);
        }
        return;
    }
    const int page_tokens = 1 << a.page_shift;
    const size_t head_values = (size_t)a.dim << a.page_shift;  // of one half of a page
    const int n_pairs = a.dim / (2 * U), tokens = 64 / n_pairs, lane = threadIdx.x & 63;  // of a wavefront
    const int heads = (a.q ? a.n_heads : 0) + a.n_kv, head_groups = (heads + HEADS - 1) / HEADS;
    const uint32_t wave = __builtin_amdgcn_readfirstlane(blockIdx.x * 4u + (threadIdx.x >> 6));
    const int h0 = wave % head_groups * HEADS, first = (int)(wave / head_groups) * tokens;
    if (first >= a.n_tokens) return;
    // lanes behind the last token work on it with the others, and store nothing
    const int p = lane / tokens, t = min(first + lane % tokens, a.n_tokens - 1);
    const bool there = first + lane % tokens < a.n_tokens;
    const KvToken tok = a.tokens[t];
    const int turned = a.rope_dim / (2 * U);  // pairs of chunks that turn
    const bool turn = p < turned, halves = turn && !a.neighbours;
    const int c0 = halves ? p : 2 * p, c1 = halves ? p + turned : 2 * p + 1;
    // keys come first, then queries
    const auto source = [&](int h) {
        return h < a.n_kv ? static_cast<const E *>(a.k) + t * a.k_stride + h * a.dim : static_cast<const E *>(a.q) + t * a.q_stride + (h - a.n_kv) * a.dim;
    };
    const auto fetch = [&](Vals<E> &x, Vals<E> &y, int h) {
        const E *src = source(min(h, heads - 1));
        x = load_once<PAST>(src + c0 * U);
        y = load_once<PAST>(src + c1 * U);
    };
    Vals<E> x[HEADS], y[HEADS];
#pragma unroll
    for (int k = 0; k < HEADS; ++k) fetch(x[k], y[k], h0 + k);
    float c[U], s[U];
    if (turn) {
        const float *cs = a.rope + (size_t)tok.pos * a.rope_dim + p * U, *sn = cs + a.rope_dim / 2;
#pragma unroll
        for (int e = 0; e < U; ++e) c[e] = cs[e], s[e] = sn[e];
    }
    const float *held = nullptr;  // the weights that are in wx, wy
    float wx[U], wy[U];
    const auto work = [&](Vals<E> &x, Vals<E> &y, int h) {
        const bool key = h < a.n_kv;
        const float *w = nullptr;
        double factor = 1.;
        if constexpr (NORM) {
            w = key ? n.k_norm : n.q_norm;
            if (w) {
                w += (int64_t)(key ? h : h - a.n_kv) * (key ? n.k_norm_stride : n.q_norm_stride);
                if (w != held) {
                    held = w;
#pragma unroll
                    for (int e = 0; e < U; ++e) wx[e] = w[c0 * U + e], wy[e] = w[c1 * U + e];
                }
                const auto exactly = [&] {
                    double sum = 0.;
#pragma unroll
                    for (int e = 0; e < U; ++e) {
                        const double u = (double)(float)x.v[e], v = (double)(float)y.v[e];
                        sum += u * u;
                        sum += v * v;
                    }
                    for (int m = tokens; m < 64; m <<= 1) sum += __shfl_xor(sum, m, 64);
                    return 1. / sqrt(sum / a.dim + n.eps);
                };
                if (sizeof(E) == 4 || (E8 && key)) {
                    factor = exactly();
                } else if constexpr (sizeof(E) == 2) {
                    // the squares are exact in fp32, and so are sums of 16 of them to 2^-20; where they leave its range, 64 bits hold them
                    const uint4 xw = __builtin_bit_cast(uint4, x), yw = __builtin_bit_cast(uint4, y);
                    float sum = 0.f;
                    const auto add = [&](uint32_t two) { sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, two), __builtin_bit_cast(bf16x2, two), sum, false); };
                    add(xw.x), add(xw.y), add(xw.z), add(xw.w), add(yw.x), add(yw.y), add(yw.z), add(yw.w);
                    sum = over_pairs(sum, tokens);
                    const bool far = !(sum < 1e37f) || n.eps > 1e37;
                    factor = (double)__builtin_amdgcn_rsqf(sum / (float)a.dim + (float)n.eps);
                    if (__any(far)) {
                        const double f = exactly();
                        factor = far ? f : factor;
                    }
                }
            }
        }
        if (E8 && key) {
            double u[U], v[U];
#pragma unroll
            for (int e = 0; e < U; ++e) u[e] = (double)(float)x.v[e], v[e] = (double)(float)y.v[e];
            if (w) {
#pragma unroll
                for (int e = 0; e < U; ++e) u[e] *= factor * (double)wx[e], v[e] *= factor * (double)wy[e];
            }
            if (turn) turn_pairs(u, v, c, s, halves);
            float f[U], g[U], top = 0.f;
#pragma unroll
            for (int e = 0; e < U; ++e) {
                f[e] = to_odd(u[e]), g[e] = to_odd(v[e]);
                top = larger(larger(top, f[e]), g[e]);
            }
            for (int m = tokens; m < 64; m <<= 1) top = fmaxf(top, __shfl_xor(top, m, 64));
            const int e = exponent_for(top);
            const float unit = unit_of(KV_EXP_BIAS - e);
            if (there) {
                if constexpr (U == 8) {
                    uint8_t *const page = reinterpret_cast<uint8_t *>(a.pages + tok.page * a.page_stride);
                    uint8_t *const to = page + h * head_values + (size_t)(tok.pos & (page_tokens - 1)) * 16;
                    const auto put = [&](int chunk, const float(&z)[U]) {
                        *reinterpret_cast<uint2 *>(to + ((size_t)(chunk >> 1) << a.page_shift) * 16 + (chunk & 1) * 8) =
                            make_uint2(four_e4m3(z[0] * unit, z[1] * unit, z[2] * unit, z[3] * unit),
                                       four_e4m3(z[4] * unit, z[5] * unit, z[6] * unit, z[7] * unit));
                    };
                    put(c0, f), put(c1, g);
                    if (p == 0) page[2 * a.n_kv * head_values + ((size_t)h << a.page_shift) + (tok.pos & (page_tokens - 1))] = (uint8_t)(e + KV_EXP_BIAS);
                }
            }
            return;
        }
        if (w || turn) {
            float u[U], v[U];
#pragma unroll
            for (int e = 0; e < U; ++e) u[e] = (float)x.v[e], v[e] = (float)y.v[e];
            if (w) {
                const float by = (float)factor;
#pragma unroll
                for (int e = 0; e < U; ++e) u[e] = u[e] * by * wx[e], v[e] = v[e] * by * wy[e];  // (what is normed is of an ordinary size, a factor times a weight may be of none)
            }
            if (turn) turn_pairs(u, v, c, s, halves);
#pragma unroll
            for (int e = 0; e < U; ++e) x.v[e] = (E)u[e], y.v[e] = (E)v[e];
        }
        if (!there) return;
        if (key) {
            E *page = reinterpret_cast<E *>(a.pages + tok.page * a.page_stride) + h * head_values + (size_t)(tok.pos & (page_tokens - 1)) * U;
            *reinterpret_cast<Vals<E> *>(page + ((size_t)c0 << a.page_shift) * U) = x;
            *reinterpret_cast<Vals<E> *>(page + ((size_t)c1 << a.page_shift) * U) = y;
        } else {
            E *to = static_cast<E *>(a.q_out) + t * a.q_out_stride + (h - a.n_kv) * a.dim;
            store_past<PAST>(to + c0 * U, x);
            store_past<PAST>(to + c1 * U, y);
        }
    };
#pragma unroll
    for (int k = 0; k < HEADS; ++k)
        if (h0 + k < heads) work(x[k], y[k], h0 + k);
}

hipError_t launch_append_heads(const AppendHeadsArgs &n, int dtype, bool e4m3, hipStream_t st)
{
    const AppendArgs &a = n.a;
    const int u = dtype == LORA_BF16 ? 8 : 4;
    const int64_t heads = (a.q ? a.n_heads : 0) + a.n_kv, tokens = 64 / (a.dim / (2 * u));
    const bool many = a.n_tokens * heads * a.dim * (dtype == LORA_BF16 ? 2 : 4) >= APPEND_MANY, norm = n.q_norm || n.k_norm;
    const int64_t each = many ? NORM_MANY_HEADS : NORM_FEW_HEADS;
    const int64_t keys = ((a.n_tokens + tokens - 1) / tokens * ((heads + each - 1) / each) + 3) / 4;
    const int64_t vals = ((int64_t)a.n_groups * a.n_kv * (a.dim / (e4m3 ? VALUES_E4M3 : u)) + 255) / 256;
    if (keys * 256 > UINT32_MAX || vals * 256 > UINT32_MAX || keys + vals > INT32_MAX) return hipErrorInvalidValue;
    const dim3 grid((unsigned)(keys + vals));
    const auto launch = [&](auto e, auto e8, auto with) {
        typedef decltype(e) E;
        constexpr bool E8 = decltype(e8)::value, NORM = decltype(with)::value;
        if (many) hipLaunchKernelGGL((append_heads_kernel<E, E8, NORM, NORM_MANY_HEADS>), grid, dim3(256), 0, st, n, (uint32_t)keys);
        else hipLaunchKernelGGL((append_heads_kernel<E, E8, NORM, NORM_FEW_HEADS>), grid, dim3(256), 0, st, n, (uint32_t)keys);
    };
    if (dtype == LORA_F32) launch(float{}, std::false_type{}, std::true_type{});
    else if (!e4m3) launch(__bf16{}, std::false_type{}, std::true_type{});
    else if (norm) launch(__bf16{}, std::true_type{}, std::true_type{});
    else launch(__bf16{}, std::true_type{}, std::false_type{});
    return hipGetLastError();
}

// What pages hold, as rows: block row y takes a piece of a page.  Keys: a thread takes chunks of tokens 8 apart, READ_KEYS; 8 tokens go with a run of 8 threads, so
// that the page is read in runs of 128 bytes, and 8 threads beside each other in a row's.  Values: a thread takes 16 bytes of a row of all tokens that share their chunks.  A launch's
// first instructions come from memory, so there are few of them: 8 bits become bf16 two at a time, values of two tokens after they changed places by bytes.
// Past the caches: 4584 tokens of 32 heads of 128 in 8 bits, 113 MB in and out, in 27 us, 4.1 TB/s (value by value 50, with READ_KEYS 4 30, with 1 25.5); 33600 of 8 heads 45 us
// (48; 40).  Pages as they are, 4608 tokens of 32 heads of 128 in 2 bytes, 151 MB: 57 us (with READ_KEYS 2 58, 1 58); 16000 of 8 heads of 64 18.4 us (23; 24).  In 4 bytes 63 us (4: 62).
template <typename P>
constexpr int READ_KEYS = sizeof(P) == 2 ? 4 : 2;
template <typename E, typename P>
__global__ __launch_bounds__(256) void read_kernel(ReadArgs a)
{
    constexpr int U = CHUNK<P>, W = CHUNK<E>;  // values of 16 bytes of a page, of a row
    constexpr int KEYS = READ_KEYS<P>;
    constexpr bool AS_IS = sizeof(P) == sizeof(E);
    // tokens off .. off + n - 1 of a page are rows row ..
    const int at = blockIdx.y, off = a.off[at], n = a.row[at + 1] - a.row[at];
    const int64_t row = a.row[at];
    const char *const page = a.pages + a.page[at] * a.page_stride;
    const size_t head_values = (size_t)a.dim << a.page_shift;
    const P *const values = reinterpret_cast<const P *>(page);
    const uint8_t *const exps = reinterpret_cast<const uint8_t *>(page) + 2 * a.n_kv * head_values;  // (pages of 8 bits)
    uint32_t i = blockIdx.x * 256u + threadIdx.x;
    const uint32_t n_keys = ((uint32_t)(a.dim / U * a.n_kv) << a.page_shift) / KEYS;  // threads that have chunks of keys
    if (i < n_keys) {
        const int chunk_shift = 31 - __builtin_clz(a.dim / U), t8 = i & 7, c = (i >> 3) & (a.dim / U - 1);
        i >>= 3 + chunk_shift;
        const int h = i % a.n_kv, t0 = (int)(i / a.n_kv) * 8 * KEYS + t8;
        const P *const from = values + h * head_values + (((size_t)c << a.page_shift) + t0) * U;
        E *const to = static_cast<E *>(a.k) + (row + t0 - off) * a.k_stride + h * a.dim + c * U;
        const auto there = [&](int j) { return (unsigned)(t0 + 8 * j - off) < (unsigned)n; };
        Vals<P> in[KEYS];
        uint32_t exp[KEYS];
#pragma unroll
        for (int j = 0; j < KEYS; ++j)
            if (there(j)) {
                in[j] = load_once<true>(from + 8 * j * U);
                if constexpr (!AS_IS) exp[j] = exps[((size_t)h << a.page_shift) + t0 + 8 * j];
            }
#pragma unroll
        for (int j = 0; j < KEYS; ++j)
            if (there(j)) {
                E *const here = to + 8 * j * a.k_stride;
                if constexpr (AS_IS) {
                    store_past<true>(here, in[j]);
                } else {
                    const uint4 x = __builtin_bit_cast(uint4, in[j]);
                    store_past<true>(here, __builtin_bit_cast(Vals<E>, eight_bf16(x.x, x.y, unit_of(exp[j]))));
                    store_past<true>(here + W, __builtin_bit_cast(Vals<E>, eight_bf16(x.z, x.w, unit_of(exp[j]))));
                }
            }
        return;
    }
    i -= n_keys;
    const int c = i & (a.dim / W - 1);
    i /= a.dim / W;
    const int h = i % a.n_kv, t0 = i / a.n_kv * U;
    if (t0 + U <= off || t0 >= off + n) return;  // (of blocks beyond the page, too: t0 is no token of it)
    Vals<P> in[W];
#pragma unroll
    for (int e = 0; e < W; ++e) in[e] = load_once<true>(values + (a.n_kv + h) * head_values + ((size_t)(t0 / U) * a.dim + c * W + e) * U);
    E *const to = static_cast<E *>(a.v) + (row + t0 - off) * a.v_stride + h * a.dim + c * W;
    const auto put = [&](int k, const Vals<E> &v) {
        if ((unsigned)(t0 + k - off) < (unsigned)n) store_past<true>(to + k * a.v_stride, v);
    };
    if constexpr (AS_IS) {
#pragma unroll
        for (int k = 0; k < U; ++k) {
            Vals<E> out;
#pragma unroll
            for (int e = 0; e < W; ++e) out.v[e] = in[e].v[k];
            put(k, out);
        }
    } else {
        const uint4 exp = *reinterpret_cast<const uint4 *>(exps + ((size_t)(a.n_kv + h) << a.page_shift) + t0);
        const auto word = [](const uint4 &v, int w) { return w == 0 ? v.x : w == 1 ? v.y : w == 2 ? v.z : v.w; };
#pragma unroll
        for (int k = 0; k < U; k += 2) {
            uint32_t two[W / 2];  // values 2 e, 2 e + 1 of token k, and those of token k + 1
#pragma unroll
            for (int e = 0; e < W / 2; ++e)
                two[e] = __builtin_amdgcn_perm(word(__builtin_bit_cast(uint4, in[2 * e + 1]), k / 4), word(__builtin_bit_cast(uint4, in[2 * e]), k / 4), k % 4 ? 0x07030602 : 0x05010400);
            const float u0 = unit_of(word(exp, k / 4) >> k % 4 * 8 & 255), u1 = unit_of(word(exp, k / 4) >> (k % 4 * 8 + 8) & 255);
            uint32_t x[W / 2], y[W / 2];
#pragma unroll
            for (int e = 0; e < W / 2; ++e) {
                x[e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(two[e], u0, false));
                y[e] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(two[e], u1, true));
            }
            put(k, __builtin_bit_cast(Vals<E>, make_uint4(x[0], x[1], x[2], x[3])));
            put(k + 1, __builtin_bit_cast(Vals<E>, make_uint4(y[0], y[1], y[2], y[3])));
        }
    }
}

hipError_t launch_read(const ReadArgs &a, int dtype, bool e4m3, hipStream_t st)
{
    const int64_t u = e4m3 ? 16 : dtype == LORA_BF16 ? 8 : 4, w = dtype == LORA_BF16 ? 8 : 4;
    const int64_t threads = ((int64_t)(a.dim / u) * a.n_kv << a.page_shift) / (e4m3 ? READ_KEYS<E4m3> : dtype == LORA_BF16 ? READ_KEYS<__bf16> : READ_KEYS<float>) + (int64_t)(a.dim / w) * a.n_kv * ((1 << a.page_shift) / u);
    const int64_t blocks = (threads + 255) / 256;
    if (blocks > INT32_MAX || a.n_reads > KV_MAX_READS) return hipErrorInvalidValue;
    const dim3 grid((unsigned)blocks, (unsigned)a.n_reads);
    if (dtype == LORA_F32) hipLaunchKernelGGL((read_kernel<float, float>), grid, dim3(256), 0, st, a);
    else if (!e4m3) hipLaunchKernelGGL((read_kernel<__bf16, __bf16>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((read_kernel<__bf16, E4m3>), grid, dim3(256), 0, st, a);
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
