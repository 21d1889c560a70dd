// Attention over the paged key-value cache (gfx950).
//
// For the rows of an item -- query vectors q_r of one key-value head -- and tokens [kv0, kv1) of its sequence, one pass
// over the tokens keeps, per row, the running maximum m of the scores (in units of log2: s = q.k * scale * log2 e), the
// sum l of exp2(s - m) and the vector o = sum exp2(s - m) v; when m grows, l and o are scaled by exp2(m_old - m_new).  The row's
// output is o / l.  Parts of a sequence are kept as m, l and o / l and join with M = max m_i as l = sum l_i exp2(m_i - M), out = sum (o_i / l_i) (l_i exp2(m_i - M) / l):
// means of values, which stay in range where the values do.  A part without a token that the row sees counts for nothing (l = 0); a row all of whose scores are -inf has no
// softmax, and its output is no number.  A token beyond the row's own position has weight 0 and its value is not multiplied at all.
#include <cfloat>
#include <type_traits>

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

// One row by one wavefront, a token a lane for the scores and D / 64 values of the output a lane.  Lane i holds values i, i + 64, ...  The weights, and their sum l, are
// 2^28 times smaller than elsewhere: a sequence has no more tokens than that, so their sums with values of any size stay in range.
constexpr float ROW_ROOM = 1 << 28;
static_assert(LORA_KV_MAX_TOKENS <= 1 << 28, "the room of one_row's sums");
template <typename E, int D> struct RowState {
    float m, l, o[D / 64];
};

template <typename E, int D>
__device__ void one_row(const AttnArgs &a, const AttnItem &it, int kv_head, int row, int kv0, int kv1, RowState<E, D> &st)
{
    constexpr int U = CHUNK<E>;
    const int lane = threadIdx.x & 63;
    const int t = row / a.group, head = kv_head * a.group + row % a.group;
    const E *q = static_cast<const E *>(a.q) + (int64_t)(it.tok0 + t) * a.q_stride + head * D;
    const int end = min(kv1, it.ctx + t + 1);
    const int in_page = (1 << a.page_shift) - 1;
    st.m = -FLT_MAX;
    st.l = 0.f;
#pragma unroll
    for (int j = 0; j < D / 64; ++j) st.o[j] = 0.f;
    for (int s0 = kv0; s0 < end; s0 += 64) {
        const int tok = min(s0 + lane, end - 1);
        const E *k = half_page<E, D>(a, a.page_list[it.page0 + (tok >> a.page_shift)], kv_head, 0) + (tok & in_page) * U;
        float s = 0.f;
        for (int c = 0; c < D / U; ++c) {
            const Vals<E> kc = *reinterpret_cast<const Vals<E> *>(k + ((size_t)c << a.page_shift) * U);
            const Vals<E> qc = *reinterpret_cast<const Vals<E> *>(q + c * U);
#pragma unroll
            for (int e = 0; e < U; ++e) s += (float)qc.v[e] * (float)kc.v[e];
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
            const E *v = half_page<E, D>(a, a.page_list[it.page0 + (at >> a.page_shift)], kv_head, 1) + (size_t)((at & in_page) / U) * D * U;
#pragma unroll
            for (int j = 0; j < D / 64; ++j) {
                const Vals<E> vc = *reinterpret_cast<const Vals<E> *>(v + (lane + 64 * j) * U);
#pragma unroll
                for (int e = 0; e < U; ++e) {
                    const float w = __shfl(p, c * U + e, 64);
                    if (at + e < end) st.o[j] += w * (float)vc.v[e];
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
// alone makes 1.6e-3 (bf16, 8192 tokens).
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

// the first n values of a chunk, zeros for the others
template <typename E> __device__ __forceinline__ uint4 first_values(const uint4 &v, int n)
{
    Vals<E> x = __builtin_bit_cast(Vals<E>, v);
#pragma unroll
    for (int e = 0; e < CHUNK<E>; ++e)
        if (e >= n) x.v[e] = (E)0.f;
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
template <typename E, int D, bool TILE>
__device__ __forceinline__ void put_row(const AttnArgs &a, const AttnItem &it, int kv_head, int r, const RowState<E, D> &st)
{
    const int lane = threadIdx.x & 63;
    const float f = it.part >= 0 && st.l == 0.f ? 0.f : 1.f / st.l;
    if (it.part >= 0) {
        const int64_t at = it.part + (int64_t)kv_head * (TILE ? (it.n_rows + 31) & ~31 : it.n_rows) + r;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) {
            const int d = lane + 64 * j;
            if (TILE) a.part_o[(at - (r & 31)) * D + tile_part(r & 31, d)] = st.o[j] * f;  // (32 rows' results begin wherever the pieces before them end)
            else a.part_o[at * D + d] = st.o[j] * f;
        }
        if (lane == 0) a.part_ml[2 * at] = st.m, a.part_ml[2 * at + 1] = st.l * ROW_ROOM;
    } else {
        const int row = it.row0 + r;
        E *out = static_cast<E *>(a.out) + (int64_t)(it.tok0 + row / a.group) * a.out_stride + (kv_head * a.group + row % a.group) * D;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) out[lane + 64 * j] = (E)(st.o[j] * f);
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

template <typename E, int D, bool ALONE>
__device__ __forceinline__ void attn_rows(const AttnArgs &a, const AttnItem &it, int kv_head, RowsLds<D> &lds)
{
    constexpr int U = CHUNK<E>, NT = U / 4, STEP = 16 * NT, KC = D / U / 4, VJ = D / 16, NW = ROW_WAVES, DP = RowsLds<D>::DP;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int in_page = (1 << a.page_shift) - 1;

    const int row = it.row0 + min(r, it.n_rows - 1);
    const int end = it.ctx + row / a.group + 1;  // tokens that this lane's row sees
    uint4 q[KC];
    {
        const E *p = static_cast<const E *>(a.q) + (int64_t)(it.tok0 + row / a.group) * a.q_stride + (kv_head * a.group + row % a.group) * D;
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
            RowState<E, D> st;
            one_row<E, D>(a, it, kv_head, it.row0 + i, it.kv0, it.kv1, st);
            put_row<E, D, false>(a, it, kv_head, i, st);
        }
    };
    if constexpr (ALONE) {  // (items that one wavefront has to itself are whole)
        if (redo) return again(0, 1);
        if (r >= it.n_rows) return;
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

// Block b of the row items: the first n_rows of the list have a block for each key-value head; the others, n_short of them, are short and a wavefront does one
template <typename E, int D>
__device__ __forceinline__ void attn_rows_block(const AttnArgs &a, uint32_t b, RowsLds<D> &lds)
{
    const uint32_t blocks = (uint32_t)a.n_rows * a.n_kv;
    if (b < blocks) {
        const AttnItem it = a.rows[b / a.n_kv];
        attn_rows<E, D, false>(a, it, b % a.n_kv, lds);
    } else {
        const uint32_t n = (b - blocks) * ROW_WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        if (n >= (uint32_t)a.n_short * a.n_kv) return;
        const AttnItem it = a.rows[a.n_rows + n / a.n_kv];
        attn_rows<E, D, true>(a, it, n % a.n_kv, lds);
    }
}

template <typename E, int D>
__global__ __launch_bounds__(64 * ROW_WAVES, 2) void attn_rows_kernel(AttnArgs a)
{
    __shared__ RowsLds<D> lds;
    attn_rows_block<E, D>(a, blockIdx.x, lds);
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

// 32 rows of a wavefront: lane r + 32 h has row r's queries (chunks 2 c + h), its maximum, half of its weights and outputs.  s: scores of
// the stage; w: its weights; o[j][4 k + i]: value 32 j + 8 k + 4 h + i
template <typename E, int D, int TK> struct TileRows {
    static constexpr int U = CHUNK<E>, SUB = TK / 32, QC = D / (2 * U), DJ = D / 32, PK = 32 / (2 * U);
    uint4 q[QC], w[SUB * PK];
    floatx16 o[DJ], s[SUB];
    float m, l;
    int end, least;  // tokens that the lane's row sees, and the wavefront's first
    __device__ __forceinline__ TileRows(const AttnArgs &a, const AttnItem &it, int kv_head, int part)
    {
        const int lane = threadIdx.x & 63, h = lane >> 5, row = it.row0 + min(part * 32 + (lane & 31), it.n_rows - 1);
        const int t = row / a.group;
        end = it.ctx + t + 1;
        least = it.ctx + (it.row0 + min(part * 32, it.n_rows - 1)) / a.group + 1;
        const E *p = static_cast<const E *>(a.q) + (int64_t)(it.tok0 + t) * a.q_stride + (kv_head * a.group + row - t * a.group) * D;
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
            w[k] = weights(p);
            asm volatile("" : "+v"(w[k].x), "+v"(w[k].y), "+v"(w[k].z), "+v"(w[k].w), "+v"(l));  // now, not where they are used
        }
    }
};

// The end of a wavefront's 32 rows
template <typename E, int D, int TK>
__device__ __forceinline__ void finish_tile(const AttnArgs &a, const AttnItem &it, int kv_head, int part, const TileRows<E, D, TK> &t)
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
            RowState<E, D> st;
            one_row<E, D>(a, it, kv_head, it.row0 + i, it.kv0, it.kv1, st);
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
template <typename E, int D> struct TileShape {
    static constexpr int TK = 32, PLACE = TK * D * (int)sizeof(E);
    static constexpr int BLOCKS = PLACE <= 8192 ? 2 : 1;  // on a compute unit
    static constexpr int DEEP = PLACE <= 16384 ? 3 : 1;
    static constexpr int LDS = (2 * DEEP + 3) * PLACE;
};

template <typename E, int D, int GROUPS>
__device__ __forceinline__ void attn_tile(const AttnArgs &a, const AttnItem &it, int kv_head, unsigned char *all_lds)
{
    typedef TileShape<E, D> Shape;
    constexpr int TK = Shape::TK, PLACE = Shape::PLACE, DEEP = Shape::DEEP, K_END = (DEEP + 1) * PLACE, V_END = (DEEP + 2) * PLACE;
    constexpr int U = CHUNK<E>;
    typedef TileRows<E, D, TK> Rows;
    constexpr int QC = Rows::QC, DJ = Rows::DJ, PK = Rows::PK, NV = PK * DJ, AHEAD = NV < 8 ? NV : 8, STRIDE = GROUPS * TK;
    typedef Steps<E, D, STRIDE> Requests;
    constexpr int PER = Requests::PER;
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
        wait_requests<(DEEP - 1) * 2 * PER>();
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
                t.w[i / U] = weights(p);
                asm volatile("" : "+v"(t.w[i / U].x), "+v"(t.w[i / U].y), "+v"(t.w[i / U].z), "+v"(t.w[i / U].w), "+v"(t.l));  // now, not where they are used
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
                mma32<E>(t.o[e % DJ], fv[e % AHEAD], t.w[e / DJ]);
                if (e + AHEAD < NV) fv[e % AHEAD] = value(e + AHEAD, v_last);
                if (e < NV / 2) {
#pragma unroll
                    for (int i = e * 2 * AHEAD / NV; i < (e + 1) * 2 * AHEAD / NV; ++i) fk[i] = key(i);
                    weigh(other, 8 + e * 16 / NV, 8 + (e + 1) * 16 / NV);
                } else {  // (the compiler does not know of the instructions that max3 is: products lie between it and the scores')
#pragma unroll
                    for (int i = (e - NV / 2) * 16 / NV; i < (e + 1 - NV / 2) * 16 / NV; ++i) top = max3(top, s[2 * i], s[2 * i + 1]);
                }
                if (e == 1) request();  // (beside the products)
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
        }
        __builtin_amdgcn_sched_barrier(0);
        t0 += STRIDE;
    };
    t.wait_for_queries();
    wait_requests<DEEP * 2 * PER>();
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
            for (int e = 0; e < NV; ++e) mma32<E>(t.o[e % DJ], e < AHEAD ? fv[e] : value(e, v_last), t.w[e / DJ]);
        }
        hide(s0);
        float top = -INFINITY;
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s0[i]);
        follow(top);
        weigh(s0, 0, 16);
#pragma unroll
        for (int e = 0; e < NV; ++e) mma32<E>(t.o[e % DJ], first_values<E>(value(e, v), it.kv1 - t0 - (2 * (e / DJ) + h) * U), t.w[e / DJ]);
    }
    for (int i = mine; i < n; ++i) {
        next();
        request();
    }
    wait_requests<0>();  // none is on its way to LDS when the block ends
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
    if (wave * 32 < it.n_rows) finish_tile<E, D, TK>(a, it, kv_head, wave, t);
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
            mma32<E>(t.o[e % DJ], f[e % AHEAD], t.w[e / DJ]);
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
        for (int i = 0; i < NV; ++i) mma32<E>(t.o[i % DJ], first_values<E>(value(i), it.kv1 - t0 - (2 * (i / DJ) + h) * U), t.w[i / DJ]);
    }
    if (wave * 32 < it.n_rows) finish_tile<E, D, TK>(a, it, kv_head, wave, t);
}

template <typename E, int D>
__global__ __launch_bounds__(256, (TileShape<E, D>::BLOCKS)) void attn_tiles_kernel(AttnArgs a)
{
    extern __shared__ __align__(16) unsigned char lds[];
    const AttnItem it = a.tiles[blockIdx.x / a.n_kv];
    attn_tile<E, D, 1>(a, it, blockIdx.x % a.n_kv, lds);
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
template <typename E, int D>
__global__ __launch_bounds__(256, (TileShape<E, D>::BLOCKS)) void attn_both_kernel(AttnArgs a)
{
    extern __shared__ __align__(16) unsigned char lds[];
    static_assert(TileShape<E, D>::LDS >= (int)sizeof(RowsLds<D>), "the rows' LDS is the tiles'");
    const uint32_t tiles = (uint32_t)a.n_tiles * a.n_kv;
    if (blockIdx.x < tiles) {
        const AttnItem it = a.tiles[blockIdx.x / a.n_kv];
        attn_tile<E, D, 1>(a, it, blockIdx.x % a.n_kv, lds);
    } else {
        attn_rows_block<E, D>(a, blockIdx.x - tiles, *reinterpret_cast<RowsLds<D> *>(lds));
    }
}

// No more blocks than compute units: eight wavefronts to a tile, two on a SIMD, in two groups that take its stages in turn and join their results at the end
template <typename E, int D>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void attn_pairs_kernel(AttnArgs a)
{
    extern __shared__ __align__(16) unsigned char lds[];
    const uint32_t tiles = (uint32_t)a.n_tiles * a.n_kv;
    if (blockIdx.x < tiles) {
        const AttnItem it = a.tiles[blockIdx.x / a.n_kv];
        attn_tile<E, D, 2>(a, it, blockIdx.x % a.n_kv, lds);
    } else if (threadIdx.x < 64 * ROW_WAVES) {
        attn_rows_block<E, D>(a, blockIdx.x - tiles, *reinterpret_cast<RowsLds<D> *>(lds));
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

template <int D>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void attn_turns_kernel(AttnArgs a)
{
    typedef __bf16 E;
    constexpr int U = 8, TK = Stages<E, D>::TK, HALF = Stages<E, D>::HALF, PER = Stages<E, D>::PER, DJ = D / 32;
    constexpr int AHEAD = 8, NV = 4 * DJ, NK = D / 8;  // products of values, of keys
    extern __shared__ __align__(16) unsigned char lds[];  // keys of three stages, values of three
    const AttnItem it = a.tiles[blockIdx.x / a.n_kv];
    const int kv_head = blockIdx.x % a.n_kv;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, h = lane >> 5;
    const bool second = wave >= 4;
    const int n = (it.kv1 - it.kv0 + TK - 1) / TK;
    const auto after = [](int place) { return place == 2 * HALF ? 0 : place + HALF; };
    Stages<E, D> stages(a, it, kv_head, wave & 3, it.kv0);
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
    if (!second) {
        request_keys();
        request_values();
        request_keys();
    }
    TileRows<E, D, TK> t(a, it, kv_head, wave);
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
            if (i < NV) mma32<E>(t.o[i % DJ], f[n_f], t.w[i / DJ]);
            else if (i - NV < 2) mma32_first<E>(t.s[(i - NV) % 2], f[n_f], t.q[(i - NV) / 2]);
            else mma32<E>(t.s[(i - NV) % 2], f[n_f], t.q[(i - NV) / 2]);
            if (i + AHEAD < TO) f[n_f] = operand(i + AHEAD, v, k);
            if (i == FROM + 2) {  // (beside the products)
                __builtin_amdgcn_sched_barrier(0);
                if (!second) {
                    request_values();
                    request_keys();
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    typedef std::integral_constant<int, 0> All;
    typedef std::integral_constant<int, NV> Keys;

    int v = 0, k = 0, t0 = it.kv0;  // places of the stage's values and the next one's keys
    wait_requests<2 * PER>();       // (of group 0: the others have none)
    turn_over();                    // the keys of the first stage have come
    if (second) turn_over();
    fetch_first(0, 0, Keys{});
    products(0, 0, Keys{});
    if (!second) wait_requests<2 * PER>();
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
        if (!second) wait_requests<2 * PER>();
        turn_over();
    }
    t.weigh(t0, a.scale_log2);
    if (!second) turn_over();
    // behind the last token: whatever is there, it is no value
#pragma unroll
    for (int i = 0; i < NV; ++i) mma32<E>(t.o[i % DJ], first_values<E>(operand(i, v, 0), it.kv1 - t0 - (2 * (i / DJ) + h) * U), t.w[i / DJ]);
    wait_requests<0>();  // none is on its way to LDS when the block ends
    if (wave * 32 < it.n_rows) finish_tile<E, D, TK>(a, it, kv_head, wave, t);
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

namespace {

template <typename F>
hipError_t by_type(int dtype, int dim, F f)
{
    if (dtype == LORA_BF16) {
        if (dim == 64) f(__bf16{}, std::integral_constant<int, 64>{});
        else if (dim == 128) f(__bf16{}, std::integral_constant<int, 128>{});
        else f(__bf16{}, std::integral_constant<int, 256>{});
    } else {
        if (dim == 64) f(float{}, std::integral_constant<int, 64>{});
        else if (dim == 128) f(float{}, std::integral_constant<int, 128>{});
        else f(float{}, std::integral_constant<int, 256>{});
    }
    return hipGetLastError();
}

}  // namespace

hipError_t prepare_attn_kernels()
{
    hipError_t e = hipSuccess;
    const auto allow = [&](const void *kernel, int lds) {
        if (e == hipSuccess) e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    };
    for (int dim : {64, 128, 256})
        for (int dtype : {LORA_BF16, LORA_F32})
            (void)by_type(dtype, dim, [&](auto t, auto d) {
                typedef decltype(t) E;
                constexpr int D = decltype(d)::value;
                allow(reinterpret_cast<const void *>(&attn_tiles_kernel<E, D>), TileShape<E, D>::LDS);
                allow(reinterpret_cast<const void *>(&attn_both_kernel<E, D>), TileShape<E, D>::LDS);
                if constexpr (kv_many(sizeof(E) == 2 ? LORA_BF16 : LORA_F32, D)) allow(reinterpret_cast<const void *>(&attn_many_kernel<E, D>), MANY_LDS<E, D>);
                if constexpr (kv_pairs(sizeof(E) == 2 ? LORA_BF16 : LORA_F32, D)) {
                    static_assert(2 * TileShape<E, D>::LDS >= 4 * (32 * D * 4 + 512), "one group's results in LDS");
                    allow(reinterpret_cast<const void *>(&attn_pairs_kernel<E, D>), 2 * TileShape<E, D>::LDS);
                }
            });
    allow(reinterpret_cast<const void *>(&attn_turns_kernel<128>), turn_lds(128));
    return e;
}

hipError_t launch_attn(const AttnArgs &a, int dtype, int dim, KvTiles way, int n_cu, hipStream_t st)
{
    const int64_t n_tiles = (int64_t)a.n_tiles * a.n_kv, n_rows = (int64_t)a.n_rows * a.n_kv + ((int64_t)a.n_short * a.n_kv + ROW_WAVES - 1) / ROW_WAVES;
    if (n_tiles > INT32_MAX || n_rows > INT32_MAX) return hipErrorInvalidValue;
    const dim3 tiles((unsigned)n_tiles), rows((unsigned)n_rows);
    return by_type(dtype, dim, [&](auto e, auto d) {
        typedef decltype(e) E;
        constexpr int D = decltype(d)::value;
        if (n_tiles && n_rows && way == KV_TILES_PLAIN && n_tiles + n_rows <= BOTH_ROUNDS * TileShape<E, D>::BLOCKS * n_cu) {
            hipLaunchKernelGGL((attn_both_kernel<E, D>), dim3((unsigned)(n_tiles + n_rows)), dim3(256), (TileShape<E, D>::LDS), st, a);
            return;
        }
        if constexpr (kv_pairs(sizeof(E) == 2 ? LORA_BF16 : LORA_F32, D))
            if (way == KV_TILES_PAIRS) {
                hipLaunchKernelGGL((attn_pairs_kernel<E, D>), dim3((unsigned)(n_tiles + n_rows)), dim3(512), (2 * TileShape<E, D>::LDS), st, a);
                return;
            }
        bool done = n_tiles == 0;
        if constexpr (kv_turns(sizeof(E) == 2 ? LORA_BF16 : LORA_F32, D))
            if (!done && way == KV_TILES_TURNS) {
                hipLaunchKernelGGL((attn_turns_kernel<D>), tiles, dim3(512), turn_lds(D), st, a);
                done = true;
            }
        if constexpr (kv_many(sizeof(E) == 2 ? LORA_BF16 : LORA_F32, D))
            if (!done && way == KV_TILES_MANY) {
                hipLaunchKernelGGL((attn_many_kernel<E, D>), tiles, dim3(256), (MANY_LDS<E, D>), st, a);
                done = true;
            }
        if (!done) hipLaunchKernelGGL((attn_tiles_kernel<E, D>), tiles, dim3(256), (TileShape<E, D>::LDS), st, a);
        if (n_rows) hipLaunchKernelGGL((attn_rows_kernel<E, D>), rows, dim3(64 * ROW_WAVES), 0, st, a);
    });
}

hipError_t launch_attn_join(const JoinArgs &a, int dtype, int dim, bool tiles, hipStream_t st)
{
    if ((int64_t)a.n_items * a.n_kv > INT32_MAX) return hipErrorInvalidValue;
    return by_type(dtype, dim, [&](auto e, auto d) {
        typedef decltype(e) E;
        constexpr int D = decltype(d)::value;
        if (tiles) hipLaunchKernelGGL((attn_join_tiles_kernel<E, D>), dim3(a.n_items * a.n_kv, (a.max_rows + 31) / 32), dim3(256), 0, st, a);
        else hipLaunchKernelGGL((attn_join_kernel<E, D>), dim3(a.n_items * a.n_kv, a.max_rows), dim3(256), 0, st, a);
    });
}

}  // namespace lora
