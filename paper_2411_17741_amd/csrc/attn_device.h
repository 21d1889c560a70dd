// Attention over the paged key-value cache (gfx950).
//
// For the rows of an item -- query vectors q_r of one key-value head -- and tokens [kv0, kv1) of its sequence, one pass
// over the tokens keeps, per row, the running maximum m of the scores (in units of log2: s = q.k * scale * log2 e), the
// sum l of exp2(s - m) and the vector o = sum exp2(s - m) v; when m grows, l and o are scaled by exp2(m_old - m_new).  The row's
// output is o / l.  Parts of a sequence are kept as m, l and o / l and join with M = max m_i as l = sum l_i exp2(m_i - M), out = sum (o_i / l_i) (l_i exp2(m_i - M) / l):
// means of values, which stay in range where the values do.  A part without a token that the row sees counts for nothing (l = 0); a row all of whose scores are -inf has no
// softmax, and its output is no number.  A token beyond the row's own position has weight 0 and its value is not multiplied at all.
#pragma once

#include <cfloat>
#include <type_traits>

#include "kv_e4m3.h"
#include "kv_internal.h"
#include "lora_device.h"

namespace lora {

namespace {

template <typename E> constexpr int CHUNK = 16 / (int)sizeof(E);  // values of a 16-byte chunk

template <typename E> struct alignas(16) Vals {
    E v[CHUNK<E>];
};

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v = fmaxf(v, __shfl_xor(v, off, 64));
    return v;
}

// Where the keys (half 0) or values (half 1) of one page and head lie
template <typename E, int D>
__device__ __forceinline__ const E *half_page(const AttnArgs &a, int page, int kv_head, int half)
{
    return reinterpret_cast<const E *>(a.pages + page * a.page_stride) + (((size_t)half * a.n_kv + kv_head) * D << a.page_shift);
}

// ... and the exponents of the page's tokens, where its values are of 8 bits
template <int D>
__device__ __forceinline__ const uint8_t *exponents(const AttnArgs &a, int page, int kv_head, int half)
{
    return reinterpret_cast<const uint8_t *>(a.pages + page * a.page_stride) + ((size_t)(2 * a.n_kv * D + half * a.n_kv + kv_head) << a.page_shift);
}

// The token in the packed batch of an item's rows t * group, t * group + 1, ...
__device__ __forceinline__ int token_of(const AttnArgs &a, const AttnItem &it, int t) { return it.ctx >= KV_SHARED ? a.row_tokens[it.tok0 + t] : it.tok0 + t; }

// One row by one wavefront, a token a lane for the scores and D / 64 values of the output a lane.  Lane i holds values i, i + 64, ...  The weights, and their sum l, are
// 2^28 times smaller than elsewhere: a sequence has no more tokens than that, so their sums with values of any size stay in range.  Sums over pages of 8 bits, whose values are small
// or large by whole tokens, are held in 64 bits: so small weights would leave the smallest values' products few bits.
constexpr float ROW_ROOM = 1 << 28;
static_assert(LORA_KV_MAX_TOKENS <= 1 << 28, "the room of one_row's sums");
// P: the pages' values
template <typename E, int D, typename P> struct RowState {
    float m, l;
    std::conditional_t<std::is_same_v<P, E>, float, double> o[D / 64];
};

template <typename E, int D, typename P = E>
__device__ void one_row(const AttnArgs &a, const AttnItem &it, int kv_head, int row, int kv0, int kv1, RowState<E, D, P> &st)
{
    constexpr int U = CHUNK<P>;
    const int lane = threadIdx.x & 63;
    const int t = row / a.group, head = kv_head * a.group + row % a.group;
    const E *q = static_cast<const E *>(a.q) + (int64_t)token_of(a, it, t) * a.q_stride + head * D;
    const int end = min(kv1, it.ctx + t + 1);
    const int in_page = (1 << a.page_shift) - 1;
    st.m = -FLT_MAX;
    st.l = 0.f;
#pragma unroll
    for (int j = 0; j < D / 64; ++j) st.o[j] = 0;
    for (int s0 = kv0; s0 < end; s0 += 64) {
        const int tok = min(s0 + lane, end - 1), page = a.page_list[it.page0 + (tok >> a.page_shift)];
        const P *k = half_page<P, D>(a, page, kv_head, 0) + (tok & in_page) * U;
        float s = 0.f;
        if constexpr (std::is_same_v<P, E>) {
            for (int c = 0; c < D / U; ++c) {
                const Vals<E> kc = *reinterpret_cast<const Vals<E> *>(k + ((size_t)c << a.page_shift) * U);
                const Vals<E> qc = *reinterpret_cast<const Vals<E> *>(q + c * U);
#pragma unroll
                for (int e = 0; e < U; ++e) s += (float)qc.v[e] * (float)kc.v[e];
            }
        } else {
            const float unit = unit_of(exponents<D>(a, page, kv_head, 0)[tok & in_page]);
            for (int c = 0; c < D / U; ++c) {
                const Vals<P> kc = *reinterpret_cast<const Vals<P> *>(k + ((size_t)c << a.page_shift) * U);
#pragma unroll
                for (int e = 0; e < U; ++e) s += (float)q[c * U + e] * (value_of(kc.v[e]) * unit);
            }
        }
        s = s0 + lane < end ? s * a.scale_log2 : -INFINITY;
        const float m = fmaxf(st.m, wave_max(s)), fade = __builtin_amdgcn_exp2f(st.m - m);
        const float p = s0 + lane < end ? __builtin_amdgcn_exp2f(s - m) * (1.f / ROW_ROOM) : 0.f;
        st.m = m;
        st.l = st.l * fade + wave_sum(p);
#pragma unroll
        for (int j = 0; j < D / 64; ++j) st.o[j] *= fade;
        for (int c = 0; c < 64 / U && s0 + c * U < end; ++c) {
            const int at = s0 + c * U;
            const int page = a.page_list[it.page0 + (at >> a.page_shift)];
            const P *v = half_page<P, D>(a, page, kv_head, 1) + (size_t)((at & in_page) / U) * D * U;
#pragma unroll
            for (int j = 0; j < D / 64; ++j) {
                const Vals<P> vc = *reinterpret_cast<const Vals<P> *>(v + (lane + 64 * j) * U);
#pragma unroll
                for (int e = 0; e < U; ++e) {
                    const float w = __shfl(p, c * U + e, 64);
                    if (at + e < end) {
                        if constexpr (std::is_same_v<P, E>) st.o[j] += w * (float)vc.v[e];
                        else st.o[j] += (double)w * (value_of(vc.v[e]) * unit_of(exponents<D>(a, page, kv_head, 1)[(at & in_page) + e]));
                    }
                }
            }
        }
    }
}

// acc += a . b over the chunks of a product's operands: a chunk is 8 bf16 values (one matrix instruction) or 4 fp32 values (four, the
// k-th of every lane's chunk in the k-th).  Which k a value is does not matter to the sum as long as a and b agree.
template <typename E> __device__ __forceinline__ void mma16(floatx4 &acc, const uint4 &a, const uint4 &b);
template <> __device__ __forceinline__ void mma16<__bf16>(floatx4 &acc, const uint4 &a, const uint4 &b)
{
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}
template <> __device__ __forceinline__ void mma16<float>(floatx4 &acc, const uint4 &a, const uint4 &b)
{
    const floatx4 x = __builtin_bit_cast(floatx4, a), y = __builtin_bit_cast(floatx4, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], acc, 0, 0, 0);
}
template <typename E> __device__ __forceinline__ void mma32(floatx16 &acc, const uint4 &a, const uint4 &b);
template <> __device__ __forceinline__ void mma32<__bf16>(floatx16 &acc, const uint4 &a, const uint4 &b)
{
    acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
}
template <> __device__ __forceinline__ void mma32<float>(floatx16 &acc, const uint4 &a, const uint4 &b)
{
    const floatx4 x = __builtin_bit_cast(floatx4, a), y = __builtin_bit_cast(floatx4, b);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[e], y[e], acc, 0, 0, 0);
}

// 16 bytes that nobody reads again soon: they leave what the caches hold alone
__device__ __forceinline__ uint4 load_once(const void *p)
{
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    const words w = __builtin_nontemporal_load(reinterpret_cast<const words *>(p));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// fmaxf of three values, of which none is a signalling NaN
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}

// acc = a . b
template <typename E> __device__ __forceinline__ void mma32_first(floatx16 &acc, const uint4 &a, const uint4 &b)
{
    floatx16 zero;
#pragma unroll
    for (int i = 0; i < 16; ++i) zero[i] = 0.f;
    acc = zero;
    mma32<E>(acc, a, b);
}

// the largest / the sum of the values of lanes 32 apart, and of lanes 16 and 32 apart
__device__ __forceinline__ float swap32(float v, float &other)
{
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    other = __uint_as_float(sw[1]);
    return __uint_as_float(sw[0]);
}
__device__ __forceinline__ float swap16(float v, float &other)
{
    const auto sw = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    other = __uint_as_float(sw[1]);
    return __uint_as_float(sw[0]);
}
__device__ __forceinline__ float max32(float v)
{
    float o;
    v = swap32(v, o);
    return fmaxf(v, o);
}
__device__ __forceinline__ float max16(float v)
{
    float o;
    v = swap16(v, o);
    return fmaxf(v, o);
}
__device__ __forceinline__ float sum32(float v)
{
    float o;
    v = swap32(v, o);
    return v + o;
}
__device__ __forceinline__ float sum16(float v)
{
    float o;
    v = swap16(v, o);
    return v + o;
}

// A chunk of weights, in the values' type: 4 fp32 weights as they are, 8 weights rounded to nearest bf16, the type of the product's operands.  Rows make up for what is lost with a second product;
// tiles, which are bound by their products and instructions, do not: it would be half as many products again.  Their outputs are off by 2.0e-3 of their norm where rounding the outputs
// alone makes 1.6e-3 (bf16, 8192 tokens).  But tiles of a prefix do whose rows are of segments that have few (KV_EXACT): sharing must not cost those any bits.  It costs time where the prefix
// is most of the work: 32 requests behind 100000 tokens with 64 / 8 heads of 128 129 -> 162 us, 256 of about 350 behind 2000 with 32 / 8 76.9 -> 78.4.
__device__ __forceinline__ uint4 weights(const float (&p)[8])
{
    bf16x8 v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (__bf16)p[e];
    return __builtin_bit_cast(uint4, v);
}
__device__ __forceinline__ uint4 weights(const float (&p)[4])
{
    return make_uint4(__float_as_uint(p[0]), __float_as_uint(p[1]), __float_as_uint(p[2]), __float_as_uint(p[3]));
}

// ... and what they lost when they were rounded
__device__ __forceinline__ uint4 weights(const float (&p)[8], uint4 &rest)
{
    const uint4 w = weights(p);
    const Vals<__bf16> rounded = __builtin_bit_cast(Vals<__bf16>, w);
    float x[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = p[e] - (float)rounded.v[e];
    rest = weights(x);
    return w;
}

// the first n values of a chunk, zeros for the others
template <typename E> __device__ __forceinline__ uint4 first_values(const uint4 &v, int n)
{
    Vals<E> x = __builtin_bit_cast(Vals<E>, v);
#pragma unroll
    for (int e = 0; e < CHUNK<E>; ++e)
        if (e >= n) x.v[e] = E{};
    return __builtin_bit_cast(uint4, x);
}

__device__ __forceinline__ uint4 from_lds(const unsigned char *p)
{
    typedef uint32_t words __attribute__((ext_vector_type(4)));
    const words w = *reinterpret_cast<const words *>(p);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename E> __device__ __forceinline__ void put_four(E *to, const floatx4 &v)
{
    struct alignas(4 * sizeof(E)) Four {
        E v[4];
    } four;
#pragma unroll
    for (int e = 0; e < 4; ++e) four.v[e] = (E)v[e];
    *reinterpret_cast<Four *>(to) = four;
}

// Entries of a sequence's page list, 64 at a time in the lanes of a register: the page of a step is named without a trip to memory.
struct PageList {
    const int32_t *list;
    int last, at, held;  // the last entry there is; lane i holds entry at + i
    __device__ __forceinline__ PageList(const int32_t *l, int last_entry, int first) : list(l), last(last_entry) { fetch(first); }
    __device__ __forceinline__ void fetch(int first)
    {
        at = first;
        held = list[min(at + (int)(threadIdx.x & 63), last)];
        asm volatile("" : "+v"(held));  // waited for here: not wherever an entry is used
    }
    __device__ __forceinline__ int operator[](int entry)  // the same in all lanes, no smaller than in earlier calls
    {
        entry = min(entry, last);
        if (entry - at >= 64) fetch(entry);
        return __builtin_amdgcn_readlane(held, entry - at);
    }
};

// The maximum that the weights are measured by follows the scores only when one is over it by more than this (in units of log2): weights
// up to 2^8 lose nothing in fp32 sums or in rounding, and the outputs are hardly ever scaled.
constexpr float SLACK = 8.f;

// Where value d of row r of 32 lies among a tile's partial results: as the wavefront that has them stores them, 4 values a lane
__device__ __forceinline__ int tile_part(int r, int d) { return ((d / 8) * 64 + (d / 4 % 2) * 32 + r) * 4 + d % 4; }

// A row that one_row() has done: to its place in the output, or with the partial results (`at`: the row's; tiles keep theirs in another order)
template <typename E, int D, bool TILE, typename P>
__device__ __forceinline__ void put_row(const AttnArgs &a, const AttnItem &it, int kv_head, int r, const RowState<E, D, P> &st)
{
    const int lane = threadIdx.x & 63;
    const float f = it.part >= 0 && st.l == 0.f ? 0.f : 1.f / st.l;
    if (it.part >= 0) {
        const int64_t at = it.part + (int64_t)kv_head * (TILE ? (it.n_rows + 31) & ~31 : it.n_rows) + r;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
            const int d = lane + 64 * j;
            if (TILE) a.part_o[(at - (r & 31)) * D + tile_part(r & 31, d)] = (float)(st.o[j] * f);  // (32 rows' results begin wherever the pieces before them end)
            else a.part_o[at * D + d] = (float)(st.o[j] * f);
        }
        if (lane == 0) a.part_ml[2 * at] = st.m, a.part_ml[2 * at + 1] = st.l * ROW_ROOM;
    } else {
        const int row = it.row0 + r;
        E *out = static_cast<E *>(a.out) + (int64_t)(it.tok0 + row / a.group) * a.out_stride + (kv_head * a.group + row % a.group) * D;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) out[lane + 64 * j] = (E)(float)(st.o[j] * f);
    }
}

}  // namespace

// Up to 16 rows (a token's query heads that share a key-value head, or the tokens of a short segment): the cache is read once and that
// is what the kernel's time goes into, so its wavefronts only have to keep enough requests in flight.  The four wavefronts of a
// block share the item's tokens out in four runs; each goes through its run in steps, keys and values straight from the pages into
// registers, a step ahead of the products that use them.
//
// The scores are formed transposed (S^T = K Q^T: keys the left operand, the rows' queries the right one), so that a lane holds
// the scores of ONE row: its running maximum and sum need two exchanges a step, and the weights are where the second product
// (O^T = V^T P^T) wants them, with no exchange at all: lane group g = lane / 16 holds tokens u g .. u g + u - 1 of the step, a chunk
// of values (u = 8 with bf16, where two products of 16 tokens make a step: row 4 g + i of product t is token 8 g + 4 t + i).
// Bound by memory: 512 tokens of about 1000 cached ones with 32 / 8 heads of 128, 2.6 GB, in 387 us, 6.75 TB/s (439 us with loads through the caches, which nothing here reads again); one token of
// 131071 with 64 / 8 heads, cut into 64 pieces, 79 us, 6.8 TB/s; fp32, 512 of about 1000 790 us, 6.6 TB/s.  With 16 rows an item's 16 x 16 products are mostly its own; the matrix units are busy 7 % of the time.
template <typename E, int D> constexpr bool ROWS_AHEAD = D <= 128;  // else two steps' registers are too many
constexpr int ROW_WAVES = 4, ROW_JOIN = 128;  // ROW_JOIN: columns that go through LDS at a time

template <int D> struct RowsLds {
    static constexpr int DP = D < ROW_JOIN ? D : ROW_JOIN;  // columns joined in one go; padded against bank conflicts
    alignas(16) float o[ROW_WAVES][KV_ROW_ITEM][DP + 4];
    float m[ROW_WAVES][KV_ROW_ITEM], l[ROW_WAVES][KV_ROW_ITEM];
    int redo[ROW_WAVES];
};

// The end of a wavefront's share of an item: rows r = lane % 16, of whose outputs lane group g = lane / 16 holds values 16 j + 4 g + i in o[j][i]
template <typename E, int D, bool ALONE, typename P>
__device__ __forceinline__ void finish_rows(const AttnArgs &a, const AttnItem &it, int kv_head, RowsLds<D> &lds, float m, float l, const floatx4 (&o)[D / 16])
{
    constexpr int VJ = D / 16, NW = ROW_WAVES, DP = RowsLds<D>::DP;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int row = it.row0 + min(r, it.n_rows - 1);
    l = sum16(sum32(l));
    // Outputs that are no numbers or infinite are worked out again: a value behind a row's own position had weight 0, but 0 times infinity is no number; an infinite value that
    // the row sees has met what its weight lost, which may be 0 or less; and weights that are up to 2^SLACK may have taken a sum out of range
    float none = 0.f;
#pragma unroll
    for (int j = 0; j < VJ; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) none += o[j][i] * 0.f;
    const bool redo = __any(none != 0.f);
    const auto again = [&](int from, int step) {
        for (int i = from; i < it.n_rows; i += step) {
            RowState<E, D, P> st;
            one_row<E, D, P>(a, it, kv_head, it.row0 + i, it.kv0, it.kv1, st);
            put_row<E, D, false>(a, it, kv_head, i, st);
        }
    };
    if constexpr (ALONE) {
        if (redo) return again(0, 1);
        if (r >= it.n_rows) return;
        if (it.part >= 0) {
            const int64_t at = it.part + (int64_t)kv_head * it.n_rows + r;
            const float each = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
            for (int j = 0; j < VJ; ++j) *reinterpret_cast<floatx4 *>(a.part_o + at * D + 16 * j + 4 * g) = o[j] * each;
            if (g == 0) *reinterpret_cast<float2 *>(a.part_ml + 2 * at) = make_float2(m, l);
            return;
        }
        const float f = 1.f / l;
        E *out = static_cast<E *>(a.out) + (int64_t)(it.tok0 + row / a.group) * a.out_stride + (kv_head * a.group + row % a.group) * D;
#pragma unroll
        for (int j = 0; j < VJ; ++j) put_four(out + 16 * j + 4 * g, o[j] * f);
        return;
    }
    if (g == 0) lds.m[wave][r] = m, lds.l[wave][r] = l;
    if (lane == 0) lds.redo[wave] = redo;
#pragma unroll
    for (int pass = 0; pass < D / DP; ++pass) {
        __syncthreads();
        if (pass == 0) {
            int any = 0;
#pragma unroll
            for (int w = 0; w < NW; ++w) any |= lds.redo[w];
            if (any) return again(wave, NW);
        }
#pragma unroll
        for (int j = 0; j < DP / 16; ++j) *reinterpret_cast<floatx4 *>(&lds.o[wave][r][16 * j + 4 * g]) = o[pass * (DP / 16) + j];
        __syncthreads();
        for (int i = threadIdx.x; i < it.n_rows * (DP / 4); i += 64 * NW) {
            const int rr = i / (DP / 4), d = i % (DP / 4) * 4;
            float top = lds.m[0][rr];
#pragma unroll
            for (int w = 1; w < NW; ++w) top = fmaxf(top, lds.m[w][rr]);
            float sum = 0.f, f[NW];
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                f[w] = __builtin_amdgcn_exp2f(lds.m[w][rr] - top);
                sum += lds.l[w][rr] * f[w];
            }
            const float each = it.part >= 0 && sum == 0.f ? 0.f : 1.f / sum;
            floatx4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < NW; ++w) v += *reinterpret_cast<const floatx4 *>(&lds.o[w][rr][d]) * (f[w] * each);
            if (it.part >= 0) {
                const int64_t at = it.part + (int64_t)kv_head * it.n_rows + rr;
                *reinterpret_cast<floatx4 *>(a.part_o + at * D + pass * DP + d) = v;
                if (pass == 0 && d == 0) a.part_ml[2 * at] = top, a.part_ml[2 * at + 1] = sum;
            } else {
                const int rw = it.row0 + rr;
                E *out = static_cast<E *>(a.out) + (int64_t)(it.tok0 + rw / a.group) * a.out_stride + (kv_head * a.group + rw % a.group) * D + pass * DP + d;
                put_four(out, v);
            }
        }
    }
}

template <typename E, int D, bool ALONE>
__device__ __forceinline__ void attn_rows(const AttnArgs &a, const AttnItem &it, int kv_head, RowsLds<D> &lds)
{
    constexpr int U = CHUNK<E>, NT = U / 4, STEP = 16 * NT, KC = D / U / 4, VJ = D / 16, NW = ROW_WAVES;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int in_page = (1 << a.page_shift) - 1;

    const int row = it.row0 + min(r, it.n_rows - 1);
    const int end = it.ctx + row / a.group + 1;  // tokens that this lane's row sees
    uint4 q[KC];
    {
        const E *p = static_cast<const E *>(a.q) + (int64_t)token_of(a, it, row / a.group) * a.q_stride + (kv_head * a.group + row % a.group) * D;
#pragma unroll
        for (int c = 0; c < KC; ++c) q[c] = *reinterpret_cast<const uint4 *>(p + (4 * c + g) * U);
    }

    const int steps = (it.kv1 - it.kv0 + STEP - 1) / STEP, per_wave = (steps + NW - 1) / NW;
    const int first = ALONE ? it.kv0 : it.kv0 + wave * per_wave * STEP, last = ALONE ? it.kv1 : min(it.kv1, first + per_wave * STEP);
    PageList pages(a.page_list + it.page0, (it.kv1 - 1) >> a.page_shift, min(first, it.kv1 - 1) >> a.page_shift);
    const auto page_at = [&](int pos) { return pages[pos >> a.page_shift]; };

    struct Step {
        uint4 k[NT][KC], v[VJ];
    };
    const int k_lane = U == 8 ? 8 * (r >> 2) + (r & 3) : r;
    const auto load = [&](Step &s, int pos, int page) {
        const E *kp = half_page<E, D>(a, page, kv_head, 0) + (pos & in_page) * U, *vp = half_page<E, D>(a, page, kv_head, 1) + (size_t)(pos & in_page) * D;
#pragma unroll
        for (int c = 0; c < KC; ++c)
#pragma unroll
            for (int t = 0; t < NT; ++t) s.k[t][c] = load_once(kp + (((4 * c + g) << a.page_shift) + k_lane + 4 * t) * U);
#pragma unroll
        for (int j = 0; j < VJ; ++j) s.v[j] = load_once(vp + (g * D + 16 * j + r) * U);
    };

    float m = -FLT_MAX, l = 0.f;
    floatx4 o[VJ];
#pragma unroll
    for (int j = 0; j < VJ; ++j) o[j] = floatx4{0.f, 0.f, 0.f, 0.f};

    const auto use = [&](Step &s, int pos) {
        float p[U];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < KC; ++c) mma16<E>(acc, s.k[t][c], q[c]);
#pragma unroll
            for (int i = 0; i < 4; ++i) p[4 * t + i] = pos + U * g + 4 * t + i < end ? acc[i] * a.scale_log2 : -INFINITY;
        }
        float top = p[0];
#pragma unroll
        for (int e = 1; e < U; ++e) top = fmaxf(top, p[e]);
        top = max16(max32(top));
        if (__any(top > m + SLACK)) {
            const float now = fmaxf(m, top), fade = __builtin_amdgcn_exp2f(m - now);
            m = now;
            l *= fade;
#pragma unroll
            for (int j = 0; j < VJ; ++j) o[j] *= fade;
        }
#pragma unroll
        for (int e = 0; e < U; ++e) {
            p[e] = __builtin_amdgcn_exp2f(p[e] - m);
            l += p[e];
        }
        const uint4 w = weights(p);
        uint4 w_rest = w;  // what the weights lost when they were rounded: there is time for a second product, and the outputs are as exact as with fp32 weights
        if constexpr (sizeof(E) == 2) {
            const Vals<E> rounded = __builtin_bit_cast(Vals<E>, w);
#pragma unroll
            for (int e = 0; e < U; ++e) p[e] -= (float)rounded.v[e];
            w_rest = weights(p);
        }
        if (pos + STEP > it.kv1) {  // behind the sequence's last token: whatever is there, it is no value
#pragma unroll
            for (int j = 0; j < VJ; ++j) s.v[j] = first_values<E>(s.v[j], it.kv1 - pos - U * g);
        }
#pragma unroll
        for (int j = 0; j < VJ; ++j) {
            mma16<E>(o[j], s.v[j], w);
            if constexpr (sizeof(E) == 2) mma16<E>(o[j], s.v[j], w_rest);
        }
    };

    if (first < last) {
        if constexpr (ROWS_AHEAD<E, D>) {
            Step s0, s1;
            load(s0, first, page_at(first));
            for (int pos = first;; pos += 2 * STEP) {
                if (pos + STEP < last) load(s1, pos + STEP, page_at(pos + STEP));
                use(s0, pos);
                if (pos + STEP >= last) break;
                if (pos + 2 * STEP < last) load(s0, pos + 2 * STEP, page_at(pos + 2 * STEP));
                use(s1, pos + STEP);
                if (pos + 2 * STEP >= last) break;
            }
        } else {
            Step s;
            for (int pos = first; pos < last; pos += STEP) {
                load(s, pos, page_at(pos));
                use(s, pos);
            }
        }
    }
    finish_rows<E, D, ALONE, E>(a, it, kv_head, lds, m, l, o);
}

// Up to 16 rows over pages of 8-bit values.  As above with steps of 64 tokens: a 16-byte chunk is 16 values, and so two operands.  The keys' chunks are turned into
// bf16 with their tokens' units at once, which is exact; a chunk of values is of 16 tokens, and the weights take their units.  Those may be 2^-126, and a weight that leaves the normal numbers loses
// bits: the maximum that weights are measured by lies ROWS_LEAD below the scores' (weights that leave them at the other end have their rows done again).  The tokens of a step may lie in two
// pages (of 32).  Bound by memory where there is much of it: 512 tokens of about 1000 cached ones with 32 / 8 heads of 128, 1.32 GB, in 206 us, 6.4 TB/s (matrix units busy 14 % of the time); one of 131071 with 64 / 8 46 to 47 us, 5.8.
constexpr float ROWS_LEAD = 24.f;
template <int D, bool ALONE>
__device__ __forceinline__ void attn_rows_e4m3(const AttnArgs &a, const AttnItem &it, int kv_head, RowsLds<D> &lds)
{
    constexpr int U = 16, NT = 4, STEP = 64, KC = D / 64, VJ = D / 16, NW = ROW_WAVES;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const bool two_pages = a.page_shift == 5;
    const int in_page = (1 << a.page_shift) - 1;

    const int row = it.row0 + min(r, it.n_rows - 1);
    const int end = it.ctx + row / a.group + 1;  // tokens that this lane's row sees
    uint4 q[2 * KC];
    {
        const __bf16 *p = static_cast<const __bf16 *>(a.q) + (int64_t)token_of(a, it, row / a.group) * a.q_stride + (kv_head * a.group + row % a.group) * D;
#pragma unroll
        for (int c = 0; c < 2 * KC; ++c) q[c] = *reinterpret_cast<const uint4 *>(p + (4 * (c / 2) + g) * U + c % 2 * 8);
    }

    const int steps = (it.kv1 - it.kv0 + STEP - 1) / STEP, per_wave = (steps + NW - 1) / NW;
    const int first = ALONE ? it.kv0 : it.kv0 + wave * per_wave * STEP, last = ALONE ? it.kv1 : min(it.kv1, first + per_wave * STEP);
    PageList pages(a.page_list + it.page0, (it.kv1 - 1) >> a.page_shift, min(first, it.kv1 - 1) >> a.page_shift);

    struct Step {
        uint4 k[NT][KC], v[VJ], k_units, v_units;
    };
    const size_t half = (size_t)a.n_kv * D << a.page_shift, units = 2 * half;  // bytes of a half of a page's layer; where its exponents begin
    const int k_lane = U * (r >> 2) + (r & 3);  // product t's row r is token k_lane + 4 t of the step
    const auto load = [&](Step &s, int pos) {
        const int page0 = pages[pos >> a.page_shift], page1 = two_pages ? pages[(pos + 32) >> a.page_shift] : page0, at = pos & in_page;
        const char *const k_page = a.pages + (r < 8 ? page0 : page1) * a.page_stride, *const v_page = a.pages + (g < 2 ? page0 : page1) * a.page_stride;
        const int k_at = (at + U * (r >> 2)) & in_page, v_at = (at + U * g) & in_page;
        const char *const kp = k_page + ((size_t)kv_head * D << a.page_shift) + (k_at + (r & 3)) * U, *const vp = v_page + half + ((size_t)kv_head * D << a.page_shift) + (size_t)v_at * D;
#pragma unroll
        for (int c = 0; c < KC; ++c)
#pragma unroll
            for (int t = 0; t < NT; ++t) s.k[t][c] = load_once(kp + (((size_t)(4 * c + g) << a.page_shift) + 4 * t) * U);
        s.k_units = *reinterpret_cast<const uint4 *>(k_page + units + ((size_t)kv_head << a.page_shift) + k_at);
        s.v_units = *reinterpret_cast<const uint4 *>(v_page + units + ((size_t)(a.n_kv + kv_head) << a.page_shift) + v_at);
#pragma unroll
        for (int j = 0; j < VJ; ++j) s.v[j] = load_once(vp + (16 * j + r) * U);
    };

    float m = -FLT_MAX, l = 0.f;
    floatx4 o[VJ];
#pragma unroll
    for (int j = 0; j < VJ; ++j) o[j] = floatx4{0.f, 0.f, 0.f, 0.f};

    const auto use = [&](Step &s, int pos) {
        const uint32_t ku[4] = {s.k_units.x, s.k_units.y, s.k_units.z, s.k_units.w}, vu[4] = {s.v_units.x, s.v_units.y, s.v_units.z, s.v_units.w};
        float p[U];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const float unit = unit_of(ku[t] >> 8 * (r & 3) & 255);
            floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < KC; ++c) {
                mma16<__bf16>(acc, eight_bf16(s.k[t][c].x, s.k[t][c].y, unit), q[2 * c]);
                mma16<__bf16>(acc, eight_bf16(s.k[t][c].z, s.k[t][c].w, unit), q[2 * c + 1]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) p[4 * t + i] = pos + U * g + 4 * t + i < end ? acc[i] * a.scale_log2 : -INFINITY;
        }
        float top = p[0];
#pragma unroll
        for (int e = 1; e < U; ++e) top = fmaxf(top, p[e]);
        top = max16(max32(top));
        top -= ROWS_LEAD;
        if (__any(top > m + SLACK)) {
            const float now = fmaxf(m, top), fade = __builtin_amdgcn_exp2f(m - now);
            m = now;
            l *= fade;
#pragma unroll
            for (int j = 0; j < VJ; ++j) o[j] *= fade;
        }
        const int there = it.kv1 - pos - U * g;  // of the lane's tokens: behind the sequence's last one, whatever is there is no value, and no exponent
#pragma unroll
        for (int e = 0; e < U; ++e) {
            p[e] = __builtin_amdgcn_exp2f(p[e] - m);
            l += p[e];
            p[e] *= unit_of(vu[e / 4] >> 8 * (e % 4) & 255);
        }
        if (pos + STEP > it.kv1) {
#pragma unroll
            for (int e = 0; e < U; ++e) p[e] = e < there ? p[e] : 0.f;
#pragma unroll
            for (int j = 0; j < VJ; ++j) s.v[j] = first_values<E4m3>(s.v[j], there);
        }
        // what the weights lose when they are rounded goes through a second product, as above
        uint4 w[2], rest[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = p[8 * k + e];
            w[k] = weights(x);
            const Vals<__bf16> rounded = __builtin_bit_cast(Vals<__bf16>, w[k]);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] -= (float)rounded.v[e];
            rest[k] = weights(x);
        }
#pragma unroll
        for (int j = 0; j < VJ; ++j) {
            const uint4 lo = eight_bf16(s.v[j].x, s.v[j].y, 1.f), hi = eight_bf16(s.v[j].z, s.v[j].w, 1.f);
            mma16<__bf16>(o[j], lo, w[0]);
            mma16<__bf16>(o[j], hi, w[1]);
            mma16<__bf16>(o[j], lo, rest[0]);
            mma16<__bf16>(o[j], hi, rest[1]);
        }
    };

    if (first < last) {
        if constexpr (ROWS_AHEAD<__bf16, D>) {
            Step s0, s1;
            load(s0, first);
            for (int pos = first;; pos += 2 * STEP) {
                if (pos + STEP < last) load(s1, pos + STEP);
                use(s0, pos);
                if (pos + STEP >= last) break;
                if (pos + 2 * STEP < last) load(s0, pos + 2 * STEP);
                use(s1, pos + STEP);
                if (pos + 2 * STEP >= last) break;
            }
        } else {
            Step s;
            for (int pos = first; pos < last; pos += STEP) {
                load(s, pos);
                use(s, pos);
            }
        }
    }
    finish_rows<__bf16, D, ALONE, E4m3>(a, it, kv_head, lds, m, l, o);
}

// Block b of the row items: the first n_rows of the list have a block for each key-value head; the others, n_short of them, are short and a wavefront does one
template <typename E, int D, typename P = E>
__device__ __forceinline__ void attn_rows_block(const AttnArgs &a, uint32_t b, RowsLds<D> &lds)
{
    const auto work = [&](const AttnItem &it, int kv_head, auto alone) {
        if constexpr (std::is_same_v<P, E4m3>) attn_rows_e4m3<D, decltype(alone)::value>(a, it, kv_head, lds);
        else attn_rows<E, D, decltype(alone)::value>(a, it, kv_head, lds);
    };
    const uint32_t blocks = (uint32_t)a.n_rows * a.n_kv;
    if (b < blocks) {
        const AttnItem it = a.rows[b / a.n_kv];
        work(it, b % a.n_kv, std::false_type{});
    } else {
        const uint32_t n = (b - blocks) * ROW_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (n >= (uint32_t)a.n_short * a.n_kv) return;
        const AttnItem it = a.rows[a.n_rows + n / a.n_kv];
        work(it, n % a.n_kv, std::true_type{});
    }
}

template <typename E, int D, typename P = E>
__global__ __launch_bounds__(64 * ROW_WAVES, 2) void attn_rows_kernel(AttnArgs a)
{
    __shared__ RowsLds<D> lds;
    attn_rows_block<E, D, P>(a, blockIdx.x, lds);
}

// Tiles of rows of one key-value head (its query heads token by token): wavefronts of 32 rows share the keys and values, which go through
// LDS stage by stage.  As in the kernel above scores are formed transposed, here in products of 32 tokens by 32 rows: lane half h holds,
// of 32 tokens, rows 8 j + 4 h + i of the product for its row, and the second product wants chunks of u tokens in a lane.  With bf16
// (u = 8) the keys of a product are therefore taken in the order that makes them so: product row 16 s + 8 b + 4 h + i is
// token 16 s + 8 h + 4 b + i (bits 2 and 3 of the number change places), which costs nothing as every lane names the chunk that
// it brings to LDS.
template <typename E> __device__ __forceinline__ int key_of_row(int row) { return sizeof(E) == 2 ? (row & ~12) | (row & 4) << 1 | (row & 8) >> 1 : row; }

// Requests of 4 wavefronts for stages of 64 tokens to LDS, keys as [D / u][64] chunks, values as [64 / u][D].  A wavefront's request brings 64
// chunks: keys of 64 tokens (32 in a page, 32 perhaps in another), values of u tokens (in one page).  The values are
// asked for after the keys: their pages are the ones that the keys were in.  Past the last stage requests may go on: they
// bring the last page's.
template <typename E, int D> struct Stages {
    static constexpr int TK = 64, U = CHUNK<E>, HALF = TK * D * (int)sizeof(E), PER = HALF / 4096;  // bytes of a stage's keys or values; a wavefront's requests for them
    PageList pages;
    const char *head, *k_lane;  // the head's keys in page 0, and the lane's first chunk of them
    uint32_t page_stride;
    int page_shift, loader, lane, values_at, page[2], at, t0;
    __device__ __forceinline__ Stages(const AttnArgs &a, const AttnItem &it, int kv_head, int which_loader, int first)
        : pages(a.page_list + it.page0, (it.kv1 - 1) >> a.page_shift, it.kv0 >> a.page_shift), page_stride((uint32_t)a.page_stride), page_shift(a.page_shift),
          loader(which_loader), lane(threadIdx.x & 63), values_at(((a.n_kv * D) << a.page_shift) * (int)sizeof(E)), at(0), t0(first)
    {
        head = a.pages + ((size_t)kv_head * D << a.page_shift) * sizeof(E);
        const int tok = (lane & 32) | key_of_row<E>(lane & 31);
        k_lane = head + ((loader << a.page_shift) + (a.page_shift == 5 ? tok & 31 : tok)) * 16;
        page[0] = page[1] = 0;
    }
    __device__ __forceinline__ void keys(unsigned char *to)  // of the next stage
    {
        page[0] = pages[t0 >> page_shift];
        page[1] = pages[(t0 + 32) >> page_shift];
        at = t0 & ((1 << page_shift) - 1);
        const char *const from = k_lane + (uint64_t)page_stride * (uint32_t)(lane < 32 ? page[0] : page[1]) + at * 16;
#pragma unroll
        for (int i = 0; i < PER; ++i) request16(reinterpret_cast<const __bf16 *>(from + ((4 * i) << page_shift) * 16), to + loader * 1024 + i * 4096);
        t0 += TK;
    }
    __device__ __forceinline__ void values(unsigned char *to)  // of the stage whose keys were asked for last
    {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int g = (4 * i + loader) * 64, tok = g / D * U;
            const int pg = tok < 32 ? page[0] : page[1], off = (tok < 32 || page_shift > 5 ? tok : tok - 32) + at;
            const char *const from = head + values_at + (uint64_t)page_stride * (uint32_t)pg + off * (D * (int)sizeof(E)) + (g % D + lane) * 16;
            request16(reinterpret_cast<const __bf16 *>(from), to + loader * 1024 + i * 4096);
        }
    }
};

// Such requests for stages of 32 tokens, STRIDE tokens apart.  They lie in one page, their values in one run: what differs between lanes is the same for all stages.
template <typename E, int D, int STRIDE> struct Steps {
    static constexpr int PER = 32 * D * (int)sizeof(E) / 4096;
    PageList pages;
    const char *head, *v_from;  // the head's keys in page 0; the values of the stage whose keys were asked for last
    uint32_t page_stride, k_lane, v_lane;
    int page_shift, loader, values_at, t0;
    __device__ __forceinline__ Steps(const AttnArgs &a, const AttnItem &it, int kv_head, int which_loader, int first)
        : pages(a.page_list + it.page0, (it.kv1 - 1) >> a.page_shift, it.kv0 >> a.page_shift), v_from(nullptr), page_stride((uint32_t)a.page_stride), page_shift(a.page_shift),
          loader(which_loader), values_at(((a.n_kv * D) << a.page_shift) * (int)sizeof(E)), t0(first)
    {
        const int lane = threadIdx.x & 63;
        head = a.pages + ((size_t)kv_head * D << a.page_shift) * sizeof(E);
        k_lane = (((2 * loader + lane / 32) << a.page_shift) + key_of_row<E>(lane & 31)) * 16;
        v_lane = (loader * 64 + lane) * 16;
    }
    __device__ __forceinline__ void keys(unsigned char *to)  // of the next stage
    {
        const int page = pages[t0 >> page_shift], at = t0 & ((1 << page_shift) - 1);
        const char *const base = head + (uint64_t)page_stride * (uint32_t)page;
        v_from = base + values_at + at * (D * (int)sizeof(E));
#pragma unroll
        for (int i = 0; i < PER; ++i) request16(reinterpret_cast<const __bf16 *>(base + (at + (8 * i << page_shift)) * 16 + k_lane), to + loader * 1024 + i * 4096);
        t0 += STRIDE;
    }
    __device__ __forceinline__ void values(unsigned char *to)  // of the stage whose keys were asked for last
    {
#pragma unroll
        for (int i = 0; i < PER; ++i) request16(reinterpret_cast<const __bf16 *>(v_from + i * 4096 + v_lane), to + loader * 1024 + i * 4096);
    }
};

// The same for pages of 8-bit values, for stages of TK tokens, STRIDE apart, by LOADERS wavefronts.  Their way to LDS leads through registers, where they become bf16 with their tokens' units:
// what comes to LDS was asked for a step before.  A thread has N chunks of keys, 16 values of a token each, and N chunks of values, 16 tokens of one value (heads of 64: half a chunk of
// both); the tokens of the latter are the same for all of a wavefront, their units scalars.  The work is done in pieces that fall beside the products of the step (8192 tokens with 32 / 8 heads of 128,
// tiles of 128 rows: all of it beside one product 608 us, in pieces 554; tiles of 256 in turns, by one group's wavefronts 531, by both groups' 528, and over bf16 pages 500 on that machine).
template <int D, int TK, int STRIDE, int LOADERS = 4> struct StagesE4m3 {
    static constexpr int ALL = D * TK / 16, THREADS = 64 * LOADERS, N = ALL < THREADS ? 1 : ALL / THREADS;
    static constexpr bool HALVES = ALL < THREADS;
    static constexpr int WORDS = HALVES ? 2 : 4, PIECES = N * (WORDS + WORDS / 2);  // of 4 values, 8 keys
    static_assert(HALVES ? ALL * 2 == THREADS && TK == 32 : ALL % THREADS == 0, "the threads' chunks");
    typedef std::conditional_t<HALVES, uint2, uint4> Part;
    PageList pages;
    const char *keys_at, *values_at;  // the head's in page 0, and the thread's first chunk of them
    const char *k_units_at, *v_units_at;
    uint32_t page_stride;
    int page_shift, w, row, t0, page[2];
    Part k[N], v[N], units[N];
    uint4 out;
    uint32_t k_unit;
    __device__ __forceinline__ StagesE4m3(const AttnArgs &a, const AttnItem &it, int kv_head, int loader, int first)
        : pages(a.page_list + it.page0, (it.kv1 - 1) >> a.page_shift, it.kv0 >> a.page_shift), page_stride((uint32_t)a.page_stride), page_shift(a.page_shift), w(loader), t0(first)
    {
        const int lane = threadIdx.x & 63, at = w * 64 + lane;
        row = lane % TK;
        int tok = (row & 32) | key_of_row<__bf16>(row & 31);
        if (a.page_shift == 5) tok &= 31;
        const size_t head = (size_t)kv_head * D << a.page_shift, half = (size_t)a.n_kv * D << a.page_shift;
        const int chunk = HALVES ? at / TK / 2 : at / TK, rest = HALVES ? at / TK % 2 * 8 : 0;
        keys_at = a.pages + head + (size_t)((chunk << a.page_shift) + tok) * 16 + rest;
        values_at = a.pages + half + head + at % D * 16 + (HALVES ? w % 2 * 8 : 0);
        k_units_at = a.pages + 2 * half + ((size_t)kv_head << a.page_shift) + tok;
        v_units_at = a.pages + 2 * half + ((size_t)(a.n_kv + kv_head) << a.page_shift) + (HALVES ? w % 2 * 8 : 0);
        page[0] = page[1] = 0;
        ask_keys();
        ask_values();
    }
    __device__ __forceinline__ int step_of(int i) const { return HALVES ? w / 2 : (i * THREADS + w * 64) / D; }  // of the wavefront's chunks of values: which 16 tokens of the stage
    __device__ __forceinline__ void ask_keys()  // of the next stage
    {
        page[0] = pages[t0 >> page_shift];
        if constexpr (TK == 64) page[1] = pages[(t0 + 32) >> page_shift];
        at = t0 & ((1 << page_shift) - 1);
        t0 += STRIDE;
        const uint64_t there = (uint64_t)page_stride * (uint32_t)(TK == 32 || row < 32 ? page[0] : page[1]) + at;
#pragma unroll
        for (int i = 0; i < N; ++i) k[i] = *reinterpret_cast<const Part *>(keys_at + there + at * 15 + ((i * (THREADS / TK)) << page_shift) * 16);
        k_unit = *reinterpret_cast<const uint8_t *>(k_units_at + there);
    }
    __device__ __forceinline__ void ask_values()  // of the stage whose keys were asked for last
    {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int s = step_of(i), in_page = (at + 16 * s) & ((1 << page_shift) - 1);
            const uint64_t there = (uint64_t)page_stride * (uint32_t)(TK == 32 || s < 2 ? page[0] : page[1]);
            v[i] = *reinterpret_cast<const Part *>(values_at + there + in_page * D);
            units[i] = *reinterpret_cast<const Part *>(v_units_at + there + in_page);
        }
    }
    static __device__ __forceinline__ uint32_t word(const uint2 &x, int n) { return n == 0 ? x.x : x.y; }
    static __device__ __forceinline__ uint32_t word(const uint4 &x, int n) { return n == 0 ? x.x : n == 1 ? x.y : n == 2 ? x.z : x.w; }
    // piece p of the work that brings to LDS the next stage's keys, and the values of the stage before it
    __device__ __forceinline__ void piece(int p, unsigned char *values_to, unsigned char *keys_to)
    {
        const int i = p / (WORDS + WORDS / 2), n = p % (WORDS + WORDS / 2), lane = threadIdx.x & 63;
        if (n < WORDS) {
            const uint32_t x = word(v[i], n), u = __builtin_amdgcn_readfirstlane(word(units[i], n));
            const bf16x2 y = {(__bf16)__builtin_amdgcn_cvt_scalef32_f32_fp8(x, unit_of(u & 255), 0), (__bf16)__builtin_amdgcn_cvt_scalef32_f32_fp8(x, unit_of(u >> 8 & 255), 1)};
            const bf16x2 z = {(__bf16)__builtin_amdgcn_cvt_scalef32_f32_fp8(x, unit_of(u >> 16 & 255), 2), (__bf16)__builtin_amdgcn_cvt_scalef32_f32_fp8(x, unit_of(u >> 24), 3)};
            if (n % 2 == 0) {
                out.x = __builtin_bit_cast(uint32_t, y), out.y = __builtin_bit_cast(uint32_t, z);
            } else {
                out.z = __builtin_bit_cast(uint32_t, y), out.w = __builtin_bit_cast(uint32_t, z);
                const int eight = HALVES ? w : 2 * step_of(i) + n / 2;  // which 8 tokens of the stage
                *reinterpret_cast<uint4 *>(values_to + (eight * D + (w * 64 + lane) % D) * 16) = out;
            }
        } else {
            const int q = n - WORDS, c = HALVES ? (w * 64 + lane) / TK : (i * THREADS + w * 64 + lane) / TK * 2 + q;
            *reinterpret_cast<uint4 *>(keys_to + (c * TK + row) * 16) = eight_bf16(word(k[i], 2 * q), word(k[i], 2 * q + 1), unit_of(k_unit));
        }
    }
    __device__ __forceinline__ void ask()
    {
        ask_values();
        ask_keys();
    }
    __device__ __forceinline__ void keys(unsigned char *to)  // of the next stage
    {
#pragma unroll
        for (int p = 0; p < PIECES; ++p)
            if (p % (WORDS + WORDS / 2) >= WORDS) piece(p, nullptr, to);
        ask_keys();
    }
    __device__ __forceinline__ void values(unsigned char *to)  // of the stage before the one whose keys were asked for last
    {
#pragma unroll
        for (int p = 0; p < PIECES; ++p)
            if (p % (WORDS + WORDS / 2) < WORDS) piece(p, to, nullptr);
        ask_values();
    }

private:
    int at = 0;  // where the stage whose keys were asked for last begins in its page
};

// 32 rows of a wavefront: lane r + 32 h has row r's queries (chunks 2 c + h), its maximum, half of its weights and outputs.  s: scores of
// the stage; w: its weights; o[j][4 k + i]: value 32 j + 8 k + 4 h + i.  EXACT: what the weights lost when they were rounded is kept too, for a second product
template <typename E, int D, int TK, bool EXACT = false> struct TileRows {
    static constexpr int U = CHUNK<E>, SUB = TK / 32, QC = D / (2 * U), DJ = D / 32, PK = 32 / (2 * U);
    static_assert(!EXACT || sizeof(E) == 2, "only bf16 weights lose anything");
    uint4 q[QC], w[SUB * PK], rest[EXACT ? SUB * PK : 1];
    floatx16 o[DJ], s[SUB];
    float m, l;
    int end, least;  // tokens that the lane's row sees, and the wavefront's first
    __device__ __forceinline__ TileRows(const AttnArgs &a, const AttnItem &it, int kv_head, int part)
    {
        const int lane = threadIdx.x & 63, h = lane >> 5, row = it.row0 + min(part * 32 + (lane & 31), it.n_rows - 1);
        const int t = row / a.group;
        end = it.ctx + t + 1;
        least = it.ctx + (it.row0 + min(part * 32, it.n_rows - 1)) / a.group + 1;
        const E *p = static_cast<const E *>(a.q) + (int64_t)token_of(a, it, t) * a.q_stride + (kv_head * a.group + row - t * a.group) * D;
#pragma unroll
        for (int c = 0; c < QC; ++c) q[c] = *reinterpret_cast<const uint4 *>(p + (2 * c + h) * U);
        m = -FLT_MAX;
        l = 0.f;
#pragma unroll
        for (int j = 0; j < DJ; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[j][i] = 0.f;
    }
    __device__ __forceinline__ void wait_for_queries()  // here, and nowhere below
    {
#pragma unroll
        for (int c = 0; c < QC; ++c) asm volatile("" : "+v"(q[c].x), "+v"(q[c].y), "+v"(q[c].z), "+v"(q[c].w));
    }
    __device__ __forceinline__ void take(int k, const float (&p)[U])  // chunk k of the stage's weights
    {
        if constexpr (EXACT) w[k] = weights(p, rest[k]);
        else w[k] = weights(p);
        asm volatile("" : "+v"(w[k].x), "+v"(w[k].y), "+v"(w[k].z), "+v"(w[k].w), "+v"(l));  // now, not where they are used
        if constexpr (EXACT) asm volatile("" : "+v"(rest[k].x), "+v"(rest[k].y), "+v"(rest[k].z), "+v"(rest[k].w));
    }
    __device__ __forceinline__ void add(int j, const uint4 &values, int k)  // o[j] += values . chunk k of the weights
    {
        mma32<E>(o[j], values, w[k]);
        if constexpr (EXACT) mma32<E>(o[j], values, rest[k]);
    }
    // the stage at t0: its scores become weights
    __device__ __forceinline__ void weigh(int t0, float scale_log2)
    {
        const int h = (threadIdx.x & 63) >> 5;
        if (t0 + TK > least) {
#pragma unroll
            for (int b = 0; b < SUB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (t0 + 32 * b + i / U * 2 * U + h * U + i % U >= end) s[b][i] = -INFINITY;
        }
        // (the compiler does not know of the instructions that max3 is: products' results may be read so many cycles after them)
#pragma unroll
        for (int b = 0; b < SUB; ++b) asm volatile("s_nop 15\n\ts_nop 7" : "+v"(s[b]));
        float top = -INFINITY;
#pragma unroll
        for (int b = 0; b < SUB; ++b)
#pragma unroll
            for (int i = 0; i < 16; i += 2) top = max3(top, s[b][i], s[b][i + 1]);
        top = max32(top) * scale_log2;
        if (__any(top > m + SLACK)) {
            const float now = fmaxf(m, top), fade = __builtin_amdgcn_exp2f(m - now);
            m = now;
            l *= fade;
#pragma unroll
            for (int j = 0; j < DJ; ++j) o[j] *= fade;
        }
#pragma unroll
        for (int k = 0; k < SUB * PK; ++k) {
            float p[U];
#pragma unroll
            for (int e = 0; e < U; ++e) {
                p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[k / PK][k % PK * U + e], scale_log2, -m));
                l += p[e];
            }
            take(k, p);
        }
    }
};

// The end of a wavefront's 32 rows
template <typename E, int D, typename P = E, int TK, bool EXACT>
__device__ __forceinline__ void finish_tile(const AttnArgs &a, const AttnItem &it, int kv_head, int part, const TileRows<E, D, TK, EXACT> &t)
{
    constexpr int DJ = D / 32;
    const int lane = threadIdx.x & 63, r = lane & 31, h = lane >> 5, my = part * 32 + r, row = it.row0 + min(my, it.n_rows - 1);
    const float l = sum32(t.l);
    // a value behind a row's own position had weight 0, but 0 times infinity is no number, and weights of up to 2^SLACK may have taken a sum out of range: such rows are done again
    float none = 0.f;
#pragma unroll
    for (int j = 0; j < DJ; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) none += t.o[j][i] * 0.f;
    if (__any(none != 0.f)) {
        for (int i = part * 32; i < min(it.n_rows, part * 32 + 32); ++i) {
            RowState<E, D, P> st;
            one_row<E, D, P>(a, it, kv_head, it.row0 + i, it.kv0, it.kv1, st);
            put_row<E, D, true>(a, it, kv_head, i, st);
        }
        return;
    }
    const float f = it.part >= 0 && l == 0.f ? 0.f : 1.f / l;
    if (it.part >= 0) {
        const int64_t at = it.part + (int64_t)kv_head * ((it.n_rows + 31) & ~31) + part * 32;
#pragma unroll
        for (int j = 0; j < DJ; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                *reinterpret_cast<floatx4 *>(a.part_o + at * D + ((4 * j + k) * 64 + lane) * 4) = floatx4{t.o[j][4 * k], t.o[j][4 * k + 1], t.o[j][4 * k + 2], t.o[j][4 * k + 3]} * f;
        if (h == 0) *reinterpret_cast<float2 *>(a.part_ml + 2 * (at + r)) = make_float2(t.m, l);
        return;
    }
    E *out = static_cast<E *>(a.out) + (int64_t)(it.tok0 + row / a.group) * a.out_stride + (kv_head * a.group + row % a.group) * D;
#pragma unroll
    for (int j = 0; j < DJ; ++j) {
        if constexpr (sizeof(E) == 2) {
#pragma unroll
            for (int k = 0; k < 4; k += 2) {  // the halves change 4 values each: 8 in a row for a lane
                typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
                bf16x4 x, y;
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = (__bf16)(t.o[j][4 * k + i] * f), y[i] = (__bf16)(t.o[j][4 * k + 4 + i] * f);
                const uint2 xu = __builtin_bit_cast(uint2, x), yu = __builtin_bit_cast(uint2, y);
                const auto a0 = __builtin_amdgcn_permlane32_swap(xu.x, yu.x, false, false), a1 = __builtin_amdgcn_permlane32_swap(xu.y, yu.y, false, false);
                if (my < it.n_rows) *reinterpret_cast<uint4 *>(out + 32 * j + 8 * k + 8 * h) = make_uint4(a0[0], a1[0], a0[1], a1[1]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (my < it.n_rows)
                    *reinterpret_cast<floatx4 *>(out + 32 * j + 8 * k + 4 * h) = floatx4{t.o[j][4 * k], t.o[j][4 * k + 1], t.o[j][4 * k + 2], t.o[j][4 * k + 3]} * f;
        }
    }
}

// Tiles of 128 rows, four wavefronts, stages of 32 tokens.  A wavefront has three stages in hand at a time, so that products and exponentials, which take about as long as each
// other, run side by side: in the step of stage t
//   O += P V of stage t - 1, beside the second half of its P and the maximum of the scores of stage t;   S = K Q of stage t + 1, beside the first half of P = exp2(S - m) of stage t.
// Keys and values are requested DEEP steps ahead, values of stage t together with keys of stage t + 1, which the step of stage t waits for.  The keys of a stage are read in one step,
// its values in that and the next: there are DEEP + 1 places for keys in LDS, DEEP + 2 for values.
// A step of a wavefront alone on its SIMD takes 0.50 us with heads of 128, 0.9 with 256, 0.45 with 64, where its products are 0.27, 0.53 and 0.13: the rest are its other instructions,
// one after the other, and the barrier.  5000 tokens with 32 / 8 heads of 256: 444 us, 0.92 PFLOP/s (585 with products and exponentials in turns); 8000 with 32 / 8 heads of 64: 305 us, 0.86.
// fp32, 4096 tokens: 32 / 8 heads of 128 1117 us, 123 TFLOP/s, of 64 539 us, 128; 16 / 4 of 256 1438 us, 96.
template <typename E, int D, typename P = E> struct TileShape {
    static constexpr int TK = 32, PLACE = TK * D * (int)sizeof(E);
    static constexpr int BLOCKS = PLACE <= 8192 ? 2 : 1;  // on a compute unit
    static constexpr int DEEP = PLACE <= 16384 && std::is_same_v<P, E> ? 3 : 1;  // (what goes through registers has been asked for a step before that)
    static constexpr int LDS = (2 * DEEP + 3) * PLACE;
};

template <typename E, int D, int GROUPS, typename P, bool EXACT>
__device__ __forceinline__ void attn_tile(const AttnArgs &a, const AttnItem &it, int kv_head, unsigned char *all_lds)
{
    typedef TileShape<E, D, P> Shape;
    constexpr bool AS_IS = std::is_same_v<P, E>;  // pages hold what the products take
    constexpr int TK = Shape::TK, PLACE = Shape::PLACE, DEEP = Shape::DEEP, K_END = (DEEP + 1) * PLACE, V_END = (DEEP + 2) * PLACE;
    constexpr int U = CHUNK<E>;
    typedef TileRows<E, D, TK, EXACT> Rows;
    constexpr int QC = Rows::QC, DJ = Rows::DJ, PK = Rows::PK, NV = PK * DJ, AHEAD = NV < 8 ? NV : 8, STRIDE = GROUPS * TK;
    typedef std::conditional_t<AS_IS, Steps<E, D, STRIDE>, StagesE4m3<D, 32, STRIDE>> Requests;
    // up to `steps` steps' requests are still on their way
    const auto wait = [](auto steps) {
        if constexpr (AS_IS) wait_requests<decltype(steps)::value * 2 * Steps<E, D, STRIDE>::PER>();
        else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    static_assert(NV % AHEAD == 0 && QC % AHEAD == 0, "the operands' ring");
    const int lane = threadIdx.x & 63, id = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = id & 3, group = id >> 2, r = lane & 31, h = lane >> 5;
    unsigned char *const lds = all_lds + group * Shape::LDS;
    const int begin = it.kv0 + group * TK;
    Requests stages(a, it, kv_head, wave, begin);
    Rows t(a, it, kv_head, wave);
    stages.keys(lds);
#pragma unroll
    for (int i = 0; i < DEEP; ++i) {  // past the last stage too
        stages.values(lds + K_END + i * PLACE);
        stages.keys(lds + (i + 1) * PLACE);
    }
    // stages that there are (of the first group), and of which the wavefront's rows see something
    const int n = (it.kv1 - it.kv0 + STRIDE - 1) / STRIDE, most = min(it.kv1, it.ctx + (it.row0 + min(wave * 32 + 31, it.n_rows - 1)) / a.group + 1);
    const int mine = wave * 32 < it.n_rows && most > begin ? (most - begin + STRIDE - 1) / STRIDE : 0;
    int put_k = 0, put_v = DEEP * PLACE, k = 0, v = V_END - PLACE, v_last = 0, t0 = begin;  // places of the next requests, of the step's keys and values, of the values of the stage before
    const auto after = [](int place, int end) { return place + PLACE == end ? 0 : place + PLACE; };
    const auto meet = [] {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    const auto next = [&] {  // a step begins: its operands have come, and nobody reads any more what its requests will overwrite
        wait(std::integral_constant<int, DEEP - 1>{});
        meet();
        v_last = v;
        v = after(v, V_END);
        k = after(k, K_END);
    };
    const auto request = [&] {
        __builtin_amdgcn_sched_barrier(0);
        stages.values(lds + K_END + put_v);
        stages.keys(lds + put_k);
        put_v = after(put_v, V_END);
        put_k = after(put_k, K_END);
    };
    const auto beside = [&](int i) {  // the same beside product i of a step
        if constexpr (AS_IS) {
            if (i == 1) request();
        } else {
            constexpr int FROM = (NV + QC) / 4, OVER = (NV + QC) * 3 / 8, PIECES = Requests::PIECES;
            if (i < FROM) return;
#pragma unroll
            for (int p = (i - FROM) * PIECES / OVER; p < (i + 1 - FROM) * PIECES / OVER && p < PIECES; ++p) stages.piece(p, lds + K_END + put_v, lds + put_k);
            if (i == FROM + OVER - 1) {
                stages.ask();
                put_v = after(put_v, V_END);
                put_k = after(put_k, K_END);
            }
        }
    };
    uint4 fk[AHEAD], fv[AHEAD];
    const unsigned char *const my_keys = lds + (h * TK + r) * 16, *const my_values = lds + K_END + (h * D + r) * 16;
    const auto key = [&](int i) { return from_lds(my_keys + k + 2 * i * TK * 16); };
    const auto value = [&](int i, int place) { return from_lds(my_values + place + (2 * (i / DJ) * D + 32 * (i % DJ)) * 16); };
    const float scale_log2 = a.scale_log2;
    const auto hide = [&](floatx16 &s) {  // the scores of tokens that rows don't see
        if (t0 + TK > t.least) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (t0 + i / U * 2 * U + h * U + i % U >= t.end) s[i] = -INFINITY;
        }
    };
    const auto follow = [&](float top) {  // the maximum of a stage's scores
        top = max32(top) * scale_log2;
        if (__any(top > t.m + SLACK)) {
            const float now = fmaxf(t.m, top), fade = __builtin_amdgcn_exp2f(t.m - now);
            t.m = now;
            t.l *= fade;
#pragma unroll
            for (int j = 0; j < DJ; ++j) t.o[j] *= fade;
        }
    };
    float p[U];
    const auto weigh = [&](const floatx16 &s, int from, int to) {  // scores from .. to - 1 of a lane's 16 become weights
#pragma unroll
        for (int i = from; i < to; ++i) {
            p[i % U] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], scale_log2, -t.m));
            t.l += p[i % U];
            if (i % U == U - 1) {
                t.take(i / U, p);
            }
        }
    };
    // the step of stage t0: its scores are in s, those of the stage before in `other`, where the next stage's come; operands come out of LDS well before they are used, in
    // this order, whatever the compiler thinks of it
    const auto step = [&](floatx16 &s, floatx16 &other, auto first) {
        constexpr bool FIRST = decltype(first)::value;
        next();
        hide(s);
        float top = -INFINITY;
        if constexpr (FIRST) {
            request();
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) fk[i] = key(i);
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[i]);
        } else {
#pragma unroll
            for (int e = 0; e < NV; ++e) {
                __builtin_amdgcn_sched_barrier(0);
                t.add(e % DJ, fv[e % AHEAD], e / DJ);
                if (e + AHEAD < NV) fv[e % AHEAD] = value(e + AHEAD, v_last);
                if (e < NV / 2) {
#pragma unroll
                    for (int i = e * 2 * AHEAD / NV; i < (e + 1) * 2 * AHEAD / NV; ++i) fk[i] = key(i);
                    weigh(other, 8 + e * 16 / NV, 8 + (e + 1) * 16 / NV);
                } else {  // (the compiler does not know of the instructions that max3 is: products lie between it and the scores')
#pragma unroll
                    for (int i = (e - NV / 2) * 16 / NV; i < (e + 1 - NV / 2) * 16 / NV; ++i) top = max3(top, s[2 * i], s[2 * i + 1]);
                }
                beside(e);
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        follow(top);
#pragma unroll
        for (int i = 0; i < QC; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            if (i == 0) mma32_first<E>(other, fk[i % AHEAD], t.q[i]);
            else mma32<E>(other, fk[i % AHEAD], t.q[i]);
            if (i + AHEAD < QC) fk[i % AHEAD] = key(i + AHEAD);
            if (i < QC / 2) {
#pragma unroll
                for (int j = i * 2 * AHEAD / QC; j < (i + 1) * 2 * AHEAD / QC; ++j) fv[j] = value(j, v);
            }
            weigh(s, i * 8 / QC, (i + 1) * 8 / QC);
            if constexpr (!FIRST) beside(NV + i);
        }
        __builtin_amdgcn_sched_barrier(0);
        t0 += STRIDE;
    };
    t.wait_for_queries();
    wait(std::integral_constant<int, DEEP>{});
    meet();
    if (mine) {
        floatx16 s0, s1;
#pragma unroll
        for (int i = 0; i < QC; ++i) {
            if (i == 0) mma32_first<E>(s0, key(i), t.q[i]);
            else mma32<E>(s0, key(i), t.q[i]);
        }
        const int last = mine - 1;
        if (last) {
            step(s0, s1, std::true_type{});
            int i = 1;
            for (; i + 1 < last; i += 2) {
                step(s1, s0, std::false_type{});
                step(s0, s1, std::false_type{});
            }
            if (i < last) {
                step(s1, s0, std::false_type{});
                weigh(s1, 8, 16);
            } else {
                weigh(s0, 8, 16);
                s0 = s1;
            }
        }
        // the last stage, whose tokens may end before it does: whatever is behind the last, it is no value
        next();
        request();
        if (last) {
#pragma unroll
            for (int e = 0; e < NV; ++e) t.add(e % DJ, e < AHEAD ? fv[e] : value(e, v_last), e / DJ);
        }
        hide(s0);
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s0[i]);
        follow(top);
        weigh(s0, 0, 16);
#pragma unroll
        for (int e = 0; e < NV; ++e) t.add(e % DJ, first_values<E>(value(e, v), it.kv1 - t0 - (2 * (e / DJ) + h) * U), e / DJ);
    }
    for (int i = mine; i < n; ++i) {
        next();
        request();
    }
    wait(std::integral_constant<int, 0>{});  // none is on its way to LDS when the block ends
    if constexpr (GROUPS == 2) {  // the second group's maxima, sums and outputs go to the first through LDS
        meet();
        floatx4 *const other = reinterpret_cast<floatx4 *>(all_lds) + wave * DJ * 4 * 64 + lane;
        float2 *const other_ml = reinterpret_cast<float2 *>(all_lds + 4 * 32 * D * 4) + wave * 64 + lane;
        if (group == 1) {
#pragma unroll
            for (int j = 0; j < DJ; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) other[(4 * j + i) * 64] = floatx4{t.o[j][4 * i], t.o[j][4 * i + 1], t.o[j][4 * i + 2], t.o[j][4 * i + 3]};
            *other_ml = make_float2(t.m, t.l);
        }
        __syncthreads();
        if (group == 1) return;
        const float2 ml = *other_ml;
        const float m = fmaxf(t.m, ml.x), f0 = __builtin_amdgcn_exp2f(t.m - m), f1 = __builtin_amdgcn_exp2f(ml.x - m);
        t.m = m;
        t.l = t.l * f0 + ml.y * f1;
#pragma unroll
        for (int j = 0; j < DJ; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const floatx4 x = other[(4 * j + i) * 64];
#pragma unroll
                for (int e = 0; e < 4; ++e) t.o[j][4 * i + e] = t.o[j][4 * i + e] * f0 + x[e] * f1;
            }
    }
    if (wave * 32 < it.n_rows) finish_tile<E, D, P>(a, it, kv_head, wave, t);
}

// Without the steps' overlap, whose registers would leave room for two blocks on a compute unit, for three: their wavefronts' products and exponentials fall beside each other's, and
// so do waits for first rows and last stores.  Two stages in LDS: one is requested while the other is worked on.
template <typename E, int D, int TK>
__device__ __forceinline__ void attn_tile_plain(const AttnArgs &a, const AttnItem &it, int kv_head, unsigned char *lds)
{
    constexpr int U = CHUNK<E>, HALF = TK * D * (int)sizeof(E);
    typedef TileRows<E, D, TK> Rows;
    constexpr int SUB = Rows::SUB, QC = Rows::QC, DJ = Rows::DJ, PK = Rows::PK, NK = SUB * QC, NV = SUB * PK * DJ, AHEAD = 8;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, h = lane >> 5;
    Steps<E, D, TK> stages(a, it, kv_head, wave, it.kv0);
    stages.keys(lds);
    stages.values(lds + HALF);
    Rows t(a, it, kv_head, wave);
    // stages that there are, and of which the wavefront's rows see something
    const int n = (it.kv1 - it.kv0 + TK - 1) / TK, most = it.ctx + (it.row0 + min(wave * 32 + 31, it.n_rows - 1)) / a.group + 1;
    const int mine = wave * 32 < it.n_rows && most > it.kv0 ? min(n, (most - it.kv0 + TK - 1) / TK) : 0;
    t.wait_for_queries();
    int buf = 0, t0 = it.kv0;
    const auto next = [&](int i) {  // waits for stage i and requests the one behind it
        wait_requests<0>();
        __syncthreads();  // (nobody reads the other buffer any more)
        if (i + 1 < n) {
            stages.keys(lds + (buf ^ 1) * 2 * HALF);
            stages.values(lds + (buf ^ 1) * 2 * HALF + HALF);
        }
    };
    uint4 f[AHEAD];
    const unsigned char *const my_keys = lds + (h * TK + r) * 16, *const my_values = lds + HALF + (h * D + r) * 16;
    const auto key = [&](int i) { return from_lds(my_keys + buf * 2 * HALF + (2 * (i / SUB) * TK + 32 * (i % SUB)) * 16); };
    const auto value = [&](int i) { return from_lds(my_values + buf * 2 * HALF + (2 * (i / DJ) * D + 32 * (i % DJ)) * 16); };
    // operands come out of LDS AHEAD products before they are used, in this order, whatever the compiler thinks of it
    const auto scores = [&] {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) f[i] = key(i);
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            __builtin_amdgcn_sched_barrier(0);
            if (i < SUB) mma32_first<E>(t.s[i % SUB], f[i % AHEAD], t.q[i / SUB]);
            else mma32<E>(t.s[i % SUB], f[i % AHEAD], t.q[i / SUB]);
            if (i + AHEAD < NK) f[i % AHEAD] = key(i + AHEAD);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    const int whole = min(mine, n - 1);
    for (int i = 0; i < whole; ++i) {
        next(i);
        scores();
#pragma unroll
        for (int e = 0; e < AHEAD; ++e) f[e] = value(e);
        __builtin_amdgcn_sched_barrier(0);
        t.weigh(t0, a.scale_log2);
#pragma unroll
        for (int e = 0; e < NV; ++e) {
            __builtin_amdgcn_sched_barrier(0);
            t.add(e % DJ, f[e % AHEAD], e / DJ);
            if (e + AHEAD < NV) f[e % AHEAD] = value(e + AHEAD);
        }
        __builtin_amdgcn_sched_barrier(0);
        t0 += TK;
        buf ^= 1;
    }
    for (int i = whole; i < n - 1; ++i) {
        next(i);
        buf ^= 1;
    }
    next(n - 1);
    if (mine == n) {
        scores();
        t.weigh(t0, a.scale_log2);
        // behind the last token: whatever is there, it is no value
#pragma unroll
        for (int i = 0; i < NV; ++i) t.add(i % DJ, first_values<E>(value(i), it.kv1 - t0 - (2 * (i / DJ) + h) * U), i / DJ);
    }
    if (wave * 32 < it.n_rows) finish_tile<E, D>(a, it, kv_head, wave, t);
}

// A tile as its item wants it.  EXACT: some of the batch's tiles are KV_EXACT; the kernels of batches without any are of their own
template <bool EXACT, typename F>
__device__ __forceinline__ void tile_of(const AttnItem &it, F work)
{
    if constexpr (EXACT) {
        if (it.ctx == KV_EXACT) return work(std::true_type{});
    }
    work(std::false_type{});
}

template <typename E, int D, typename P, bool EXACT>
__global__ __launch_bounds__(256, (TileShape<E, D>::BLOCKS)) void attn_tiles_kernel(AttnArgs a)
{
    extern __shared__ __align__(16) unsigned char lds[];
    const AttnItem it = a.tiles[blockIdx.x / a.n_kv];
    tile_of<EXACT>(it, [&](auto exact) { attn_tile<E, D, 1, P, decltype(exact)::value>(a, it, blockIdx.x % a.n_kv, lds); });
}

template <typename E, int D> constexpr int MANY_LDS = 4 * 32 * D * (int)sizeof(E);
template <typename E, int D>
__global__ __launch_bounds__(256, 3) void attn_many_kernel(AttnArgs a)
{
    extern __shared__ __align__(16) unsigned char lds[];
    const AttnItem it = a.tiles[blockIdx.x / a.n_kv];
    attn_tile_plain<E, D, 32>(a, it, blockIdx.x % a.n_kv, lds);
}

// Tiles, and the blocks of the row items behind them in one launch, while there are no more than BOTH_ROUNDS times as many as are on the machine at once: rows wait for memory beside tiles' products.
// Apart -> together, heads of 128: prompts of 2 to 234 tokens with 64 / 8 heads 16.1 -> 11.7 us; 30 tokens of about 300 beside 100 + 200 with 40 heads 42.2 -> 37.0; 8 of 3000 beside 1500 with
// 32 / 8 heads 64.9 -> 56.5; 100 of 1000 beside 300 82.2 -> 73.3; 4 of 30000 beside 500 102.5 -> 96.8.  The rule counts blocks alone, and loses where the rows' bytes are most of the
// time: 20 of 3000 beside 900 + 700 72.0 -> 74.2, 20 of 8000 135.1 -> 145.7; 30 of 2000 beside 700 with 40 heads 203 -> 219.  Of larger batches nothing is gained, or lost where rows have
// fewer blocks on a compute unit this way (heads of 256, 100 tokens of 500 beside 600: 109 -> 122).
constexpr int BOTH_ROUNDS = 4;
template <typename E, int D, typename P, bool EXACT>
__global__ __launch_bounds__(256, (TileShape<E, D>::BLOCKS)) void attn_both_kernel(AttnArgs a)
{
    extern __shared__ __align__(16) unsigned char lds[];
    static_assert(TileShape<E, D, P>::LDS >= (int)sizeof(RowsLds<D>), "the rows' LDS is the tiles'");
    const uint32_t tiles = (uint32_t)a.n_tiles * a.n_kv;
    if (blockIdx.x < tiles) {
        const AttnItem it = a.tiles[blockIdx.x / a.n_kv];
        tile_of<EXACT>(it, [&](auto exact) { attn_tile<E, D, 1, P, decltype(exact)::value>(a, it, blockIdx.x % a.n_kv, lds); });
    } else {
        attn_rows_block<E, D, P>(a, blockIdx.x - tiles, *reinterpret_cast<RowsLds<D> *>(lds));
    }
}

// No more blocks than compute units: eight wavefronts to a tile, two on a SIMD, in two groups that take its stages in turn and join their results at the end
template <typename E, int D, typename P = E>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void attn_pairs_kernel(AttnArgs a)
{
    extern __shared__ __align__(16) unsigned char lds[];
    const uint32_t tiles = (uint32_t)a.n_tiles * a.n_kv;
    if (blockIdx.x < tiles) {
        const AttnItem it = a.tiles[blockIdx.x / a.n_kv];
        attn_tile<E, D, 2, P, false>(a, it, blockIdx.x % a.n_kv, lds);
    } else if (threadIdx.x < 64 * ROW_WAVES) {
        attn_rows_block<E, D, P>(a, blockIdx.x - tiles, *reinterpret_cast<RowsLds<D> *>(lds));
    }
}

// The same for bf16 heads of 128 values and long prompts, where the scores' exponentials take the vector units as long as the products
// take the matrix units: tiles of 256 rows, 8 wavefronts in two groups, one of each on a SIMD, that take turns.  In a time slot one group has
// its products -- O += P V of the last stage, S = K Q of the next -- while the other has its weights -- P = exp2(S - m) --, and a barrier
// ends the slot; group 1 is a slot behind group 0 all along.
//   group 0: slot 2 i products of stage i (S of it, O of i - 1), slot 2 i + 1 weights of stage i;   group 1: the same a slot later
// Keys and values have three places each in LDS.  Group 0 requests the keys of stage j and the values of stage j - 1 beside its products in
// slot 2 j - 4 (their places were last read by group 1 in slot 2 j - 5); they have come when slot 2 j - 2 ends, a slot
// before the first that needs them, so that a wavefront takes its first operands out of LDS before the barrier that starts its
// products.
// 8192 tokens with 32 / 8 heads: 480 to 499 us over runs, 1.10 to 1.15 PFLOP/s; 16384 with 64 / 8 3650 us, 1.20.  Bound by power: the clock is at 1.75 GHz, the matrix units are busy 56 % of the cycles (tiles of 128 rows: 537 and
// 3985 us).
constexpr int turn_lds(int dim) { return 6 * 64 * dim * 2; }

template <int D, typename P, bool EXACT>
__device__ __forceinline__ void attn_tile_turns(const AttnArgs &a, const AttnItem &it, int kv_head, unsigned char *lds)  // lds: keys of three stages, values of three
{
    typedef __bf16 E;
    constexpr bool AS_IS = std::is_same_v<P, E>;  // pages hold what the products take
    typedef std::conditional_t<AS_IS, Stages<E, D>, StagesE4m3<D, 64, 64, 8>> Requests;
    constexpr int U = 8, TK = Stages<E, D>::TK, HALF = Stages<E, D>::HALF, PER = Stages<E, D>::PER, DJ = D / 32;
    constexpr int AHEAD = 8, NV = 4 * DJ, NK = D / 8;  // products of values, of keys
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, h = lane >> 5;
    const bool second = wave >= 4;
    const int n = (it.kv1 - it.kv0 + TK - 1) / TK;
    const auto after = [](int place) { return place == 2 * HALF ? 0 : place + HALF; };
    Requests stages(a, it, kv_head, AS_IS ? wave & 3 : wave, it.kv0);
    const bool loads = !AS_IS || !second;  // conversions are shared out over all wavefronts, each beside its own products
    int put = 0, put_v = 0;
    const auto request_keys = [&] {
        stages.keys(lds + put);
        put_v = put;
        put = after(put);
    };
    const auto request_values = [&] { stages.values(lds + 3 * HALF + put_v); };
    const auto turn_over = [] {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    const auto wait = [] {  // up to a stage's requests are still on their way (of group 0: the others have none)
        if constexpr (AS_IS) wait_requests<2 * PER>();
        else asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    };
    if (loads) {
        request_keys();
        request_values();
        request_keys();
    }
    TileRows<E, D, TK, EXACT> t(a, it, kv_head, wave);
    t.wait_for_queries();

    // The products of a slot, NV of the values in place `v` of LDS and then NK of the keys in place `k`: operands come out of LDS AHEAD
    // products before they are used, in this order, whatever the compiler thinks of it
    uint4 f[AHEAD];
    const unsigned char *const my_keys = lds + (h * TK + r) * 16, *const my_values = lds + 3 * HALF + (h * D + r) * 16;
    const auto operand = [&](int i, int v, int k) {
        return i < NV ? from_lds(my_values + v + (2 * (i / DJ) * D + 32 * (i % DJ)) * 16) : from_lds(my_keys + k + (2 * ((i - NV) / 2) * TK + 32 * ((i - NV) % 2)) * 16);
    };
    const auto fetch_first = [&](int v, int k, auto from) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) f[i] = operand(decltype(from)::value + i, v, k);
    };
    const auto products = [&](int v, int k, auto from) {
        constexpr int FROM = decltype(from)::value, TO = NV + NK;
#pragma unroll
        for (int i = FROM; i < TO; ++i) {
            const int n_f = (i - FROM) % AHEAD;
            __builtin_amdgcn_sched_barrier(0);
            if (i < NV) t.add(i % DJ, f[n_f], i / DJ);
            else if (i - NV < 2) mma32_first<E>(t.s[(i - NV) % 2], f[n_f], t.q[(i - NV) / 2]);
            else mma32<E>(t.s[(i - NV) % 2], f[n_f], t.q[(i - NV) / 2]);
            if (i + AHEAD < TO) f[n_f] = operand(i + AHEAD, v, k);
            // (beside the products)
            if constexpr (AS_IS) {
                if (i == FROM + 2) {
                    __builtin_amdgcn_sched_barrier(0);
                    if (!second) {
                        request_values();
                        request_keys();
                    }
                }
            } else {
                constexpr int PIECES = Requests::PIECES, OVER = TO - FROM - 3;
                const int n = i - FROM - 2;
                if (n >= 0 && n <= OVER) {
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int p = n * PIECES / OVER; p < (n + 1) * PIECES / OVER && p < PIECES; ++p) stages.piece(p, lds + 3 * HALF + put_v, lds + put);
                    if (n == OVER) {
                        stages.ask();
                        put_v = put;
                        put = after(put);
                    }
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    typedef std::integral_constant<int, 0> All;
    typedef std::integral_constant<int, NV> Keys;

    int v = 0, k = 0, t0 = it.kv0;  // places of the stage's values and the next one's keys
    wait();
    turn_over();  // the keys of the first stage have come
    if (second) turn_over();
    fetch_first(0, 0, Keys{});
    products(0, 0, Keys{});
    if (loads) wait();
    turn_over();
    for (int i = 0; i + 1 < n; ++i) {
        t.weigh(t0, a.scale_log2);
        t0 += TK;
        k = after(k);
        fetch_first(v, k, All{});
        turn_over();
        __builtin_amdgcn_s_setprio(1);
        products(v, k, All{});
        __builtin_amdgcn_s_setprio(0);
        v = after(v);
        if (loads) wait();
        turn_over();
    }
    t.weigh(t0, a.scale_log2);
    if (!second) turn_over();
    // behind the last token: whatever is there, it is no value
#pragma unroll
    for (int i = 0; i < NV; ++i) t.add(i % DJ, first_values<E>(operand(i, v, 0), it.kv1 - t0 - (2 * (i / DJ) + h) * U), i / DJ);
    wait_requests<0>();  // none is on its way to LDS when the block ends
    if (wave * 32 < it.n_rows) finish_tile<E, D, P>(a, it, kv_head, wave, t);
}

template <int D, typename P, bool EXACT>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void attn_turns_kernel(AttnArgs a)
{
    extern __shared__ __align__(16) unsigned char lds[];
    const AttnItem it = a.tiles[blockIdx.x / a.n_kv];
    tile_of<EXACT>(it, [&](auto exact) { attn_tile_turns<D, P, decltype(exact)::value>(a, it, blockIdx.x % a.n_kv, lds); });
}

// A block joins the parts of one row: each wavefront finds the joined maximum and weight from all parts', then groups of D / 4 threads add
// up every 1024 / D-th part, four values of the head a thread, and the groups' sums are added in their order.  Bound by trips to memory, one
// after the other: 64 parts of 64 rows 4.9 us; one token of 99000 with 8 / 1 heads, 194 parts, 25.0 -> 23.7 us with the values asked for first.
template <typename E, int D>
__global__ __launch_bounds__(256) void attn_join_kernel(JoinArgs a)
{
    constexpr int GROUPS = 1024 / D;
    __shared__ __align__(16) float sums[GROUPS][D];
    const JoinItem it = a.items[blockIdx.x / a.n_kv];
    const int r = blockIdx.y;
    if (r >= it.n_rows) return;
    const int kv_head = blockIdx.x % a.n_kv, lane = threadIdx.x & 63, g = threadIdx.x / (D / 4), d = threadIdx.x % (D / 4) * 4;
    const int64_t first = it.part + (int64_t)kv_head * it.n_rows + r;
    const auto part = [&](int i) { return *reinterpret_cast<const floatx4 *>(a.part_o + (first + (int64_t)i * it.stride) * D + d); };
    constexpr int AT_ONCE = 8;  // parts that a group of threads asks for before it knows their weights: a trip to memory less
    floatx4 v[AT_ONCE];
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) v[k] = g + k * GROUPS < it.n_parts ? part(g + k * GROUPS) : floatx4{0.f, 0.f, 0.f, 0.f};
    float m = -FLT_MAX, l = 0.f;
    for (int i = lane; i < it.n_parts; i += 64) m = fmaxf(m, a.part_ml[2 * (first + (int64_t)i * it.stride)]);
    m = wave_max(m);
    for (int i = lane; i < it.n_parts; i += 64) {
        const float2 ml = *reinterpret_cast<const float2 *>(a.part_ml + 2 * (first + (int64_t)i * it.stride));
        l += ml.y * __builtin_amdgcn_exp2f(ml.x - m);
    }
    l = wave_sum(l);
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    const float each = 1.f / l;
    const auto weight = [&](int i) {
        const float2 ml = *reinterpret_cast<const float2 *>(a.part_ml + 2 * (first + (int64_t)i * it.stride));
        return ml.y * __builtin_amdgcn_exp2f(ml.x - m) * each;
    };
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k)
        if (g + k * GROUPS < it.n_parts) o += v[k] * weight(g + k * GROUPS);
    for (int i = g + AT_ONCE * GROUPS; i < it.n_parts; i += GROUPS) o += part(i) * weight(i);
    *reinterpret_cast<floatx4 *>(&sums[g][d]) = o;
    __syncthreads();
    if (g == 0) {
        for (int i = 1; i < GROUPS; ++i) o += *reinterpret_cast<const floatx4 *>(&sums[i][d]);
        const int row = it.row0 + r;
        put_four(static_cast<E *>(a.out) + (int64_t)(it.tok0 + row / a.group) * a.out_stride + (kv_head * a.group + row % a.group) * D + d, o);
    }
}

// A block joins the parts of 32 rows of a tile: a thread has D / 32 times 4 values of one row.  Values are asked for before the weights
// are known: 213 + 752 tokens with 6 / 2 heads of 128 15.6 -> 14.6 us, 1000 with 8 / 1 heads of 256 27.2 -> 25.2.
template <typename E, int D>
__global__ __launch_bounds__(256) void attn_join_tiles_kernel(JoinArgs a)
{
    constexpr int N = D / 32;
    const JoinItem it = a.items[blockIdx.x / a.n_kv];
    const int group = blockIdx.y, lane = threadIdx.x & 63, r = lane & 31;
    if (group * 32 >= it.n_rows) return;
    const int kv_head = blockIdx.x % a.n_kv;
    const int64_t first = it.part + (int64_t)kv_head * ((it.n_rows + 31) & ~31) + group * 32;
    const float2 *ml = reinterpret_cast<const float2 *>(a.part_ml) + first + r;
    const float *from = a.part_o + first * D + threadIdx.x * 4;
    constexpr int AT_ONCE = 16 / N;  // parts whose values are asked for before their weights are known: a trip to memory less
    float m = -FLT_MAX, l = 0.f;
    floatx4 o[N];
#pragma unroll
    for (int k = 0; k < N; ++k) o[k] = floatx4{0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < it.n_parts; i += AT_ONCE) {
        float2 x[AT_ONCE];
        floatx4 v[AT_ONCE][N];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            const bool there = i + j < it.n_parts;
            const int64_t at = (int64_t)(i + j) * it.stride;
            x[j] = there ? ml[at] : make_float2(-FLT_MAX, 0.f);
#pragma unroll
            for (int k = 0; k < N; ++k) v[j][k] = there ? *reinterpret_cast<const floatx4 *>(from + at * D + k * 1024) : floatx4{0.f, 0.f, 0.f, 0.f};
        }
        float top = m;
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) top = fmaxf(top, x[j].x);
        const float before = l * __builtin_amdgcn_exp2f(m - top);
        m = top;
        l = before;
        float w[AT_ONCE];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            w[j] = x[j].y * __builtin_amdgcn_exp2f(x[j].x - m);  // (of a part that is not there: 0)
            l += w[j];
        }
        const float each = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int k = 0; k < N; ++k) o[k] *= before * each;
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j)
#pragma unroll
            for (int k = 0; k < N; ++k) o[k] += v[j][k] * (w[j] * each);
    }
    if (group * 32 + r >= it.n_rows) return;
    const int row = it.row0 + group * 32 + r;
    E *out = static_cast<E *>(a.out) + (int64_t)(it.tok0 + row / a.group) * a.out_stride + (kv_head * a.group + row % a.group) * D;
#pragma unroll
    for (int k = 0; k < N; ++k) put_four(out + (k * 4 + threadIdx.x / 64) * 8 + lane / 32 * 4, l == 0.f ? o[k] / l : o[k]);
}

// Joins the parts of rows of batches with shared prefixes: D / 4 lanes to a row, 64 / (D / 4) rows to a wavefront.  A row's lanes find its sources all at once, then each a part of theirs
// with its maximum and sum; then each has 4 values of part after part, eight loads on their way at a time.  Bound by trips to memory one after the other, as the joins above are: 8192 rows of two
// parts 6.0 us (a wavefront to a row 9.6), 2048 of 33, 35 MB, 12.
template <int D> constexpr int SHARED_JOIN_ROWS = 4 * 256 / D;  // of a block
template <typename E, int D>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedJoinArgs a)
{
    constexpr int PER = D / 4, AHEAD = 8;
    const SharedJoin it = a.items[blockIdx.x / a.n_kv];
    const int kv_head = blockIdx.x % a.n_kv, lane = threadIdx.x & 63, j = lane % PER, base = lane - j, at_row = blockIdx.y * SHARED_JOIN_ROWS<D> + threadIdx.x / PER;
    if ((int)(blockIdx.y * SHARED_JOIN_ROWS<D> + (threadIdx.x & ~63u) / PER) >= it.n_rows) return;  // (a wavefront's first row)
    const int r = it.first + min(at_row, it.n_rows - 1);  // of the rows that the sources are of; rows behind the last are that, and stored by none
    // lane k of a row: source k's first part of the row, of how many
    int first = 0, stride = 0, n = 0, tile_row = -1;  // tile_row: the row of 32 in a tile's layout, or -1
    if (j < it.n_sources) {
        const SharedSource src = a.sources[it.source0 + j];
        const int row = src.row0 + r, at = row / src.rows, rr = row - at * src.rows;
        const SharedBlock blk = a.blocks[src.block0 + at];
        first = blk.part + kv_head * (src.tile ? (blk.n_rows + 31) & ~31 : blk.n_rows) + rr;
        stride = blk.stride, n = blk.n_parts;
        if (src.tile) tile_row = rr & 31;
    }
    int total = 0, begin = 0;  // parts of all sources; of those before the lane's
    for (int k = 0; k < it.n_sources; ++k) {
        if (j == k) begin = total;
        total += __shfl(n, base + k, 64);
    }
    const int d = j * 4, tile_d = (d / 8 * 64 + d / 4 % 2 * 32) * 4;
    float m = -FLT_MAX, l = 0.f;
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = 0; __any(p0 < total); p0 += PER) {
        // the lane's part: its row of partial results, and where its values begin (less one and negative: in a tile's layout)
        int row = 0, at = 0;
        for (int k = 0; k < it.n_sources; ++k) {
            const int i = p0 + j - __shfl(begin, base + k, 64), t = __shfl(tile_row, base + k, 64), from = __shfl(first, base + k, 64) + i * __shfl(stride, base + k, 64);
            if (i >= 0) row = from, at = t < 0 ? from * D : ~((from - t) * D + t * 4);
        }
        const int n_now = min(total - p0, PER);
        const float2 ml = j < n_now ? *reinterpret_cast<const float2 *>(a.part_ml + 2 * (int64_t)row) : make_float2(-FLT_MAX, 0.f);
        float top = fmaxf(m, ml.x);
#pragma unroll
        for (int off = PER / 2; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor(top, off, 64));
        const float before = l * __builtin_amdgcn_exp2f(m - top), w = ml.y * __builtin_amdgcn_exp2f(ml.x - top);
        m = top;
        l = w;
#pragma unroll
        for (int off = PER / 2; off > 0; off >>= 1) l += __shfl_xor(l, off, 64);
        l += before;
        const float each = l == 0.f ? 0.f : 1.f / l;
        o *= before * each;
        for (int i0 = 0; __any(i0 < n_now); i0 += AHEAD) {
            floatx4 v[AHEAD];
            float f[AHEAD];
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const int from = base + ((i0 + i) & (PER - 1)), where = __shfl(at, from, 64);
                f[i] = __shfl(w, from, 64) * each;
                v[i] = floatx4{0.f, 0.f, 0.f, 0.f};
                if (i0 + i < n_now) v[i] = *reinterpret_cast<const floatx4 *>(a.part_o + (where < 0 ? ~where + tile_d : where + d));
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i)
                if (i0 + i < n_now) o += v[i] * f[i];
        }
    }
    const int to = it.row0 + r;
    if (at_row < it.n_rows)
        put_four(static_cast<E *>(a.out) + (int64_t)(it.tok0 + to / a.group) * a.out_stride + (kv_head * a.group + to % a.group) * D + d, l == 0.f ? o / l : o);
}

}  // namespace lora
