// Attention over the paged key-value cache (gfx950).
//
// For the rows of an item -- query vectors q_r of one key-value head -- and tokens [kv0, kv1) of its sequence, one pass
// over the tokens keeps, per row, the running maximum m of the scores (in units of log2: s = q.k * scale * log2 e), the
// sum l of exp2(s - m) and the vector o = sum exp2(s - m) v; when m grows, l and o are scaled by exp2(m_old - m_new).  The row's
// output is o / l.  Parts of a sequence join with M = max m_i as l = sum l_i exp2(m_i - M), o = sum o_i exp2(m_i - M).  A
// token beyond the row's own position has weight 0 and its value is not multiplied at all.
#include <cfloat>

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

// One row by one wavefront, a token a lane for the scores and D / 64 values of the output a lane.  Lane i holds values i, i + 64, ...
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
        const float p = s0 + lane < end ? __builtin_amdgcn_exp2f(s - m) : 0.f;
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

// a chunk of weights: rounded to the values' type (8 weights to nearest bf16, the product's operand type; 4 fp32 weights as they are)
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

template <typename E, int D>
__device__ __forceinline__ void put_row(const AttnArgs &a, const AttnItem &it, int kv_head, int r, const RowState<E, D> &st)
{
    const int lane = threadIdx.x & 63;
    if (it.part >= 0) {
        const int64_t at = it.part + (int64_t)kv_head * it.n_rows + r;
#pragma unroll
        for (int j = 0; j < D / 64; ++j) a.part_o[at * D + lane + 64 * j] = st.o[j];
        if (lane == 0) a.part_ml[2 * at] = st.m, a.part_ml[2 * at + 1] = st.l;
    } else {
        const int row = it.row0 + r;
        E *out = static_cast<E *>(a.out) + (int64_t)(it.tok0 + row / a.group) * a.out_stride + (kv_head * a.group + row % a.group) * D;
        const float f = st.l == 0.f ? 0.f : 1.f / st.l;
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
template <typename E, int D> constexpr bool ROWS_AHEAD = D <= 128;  // else two steps' registers are too many
constexpr int ROW_WAVES = 4, ROW_JOIN = 128;  // ROW_JOIN: columns that go through LDS at a time

template <typename E, int D>
__global__ __launch_bounds__(64 * ROW_WAVES, 2) void attn_rows_kernel(AttnArgs a)
{
    constexpr int U = CHUNK<E>, NT = U / 4, STEP = 16 * NT, KC = D / U / 4, VJ = D / 16, NW = ROW_WAVES;
    constexpr int DP = D < ROW_JOIN ? D : ROW_JOIN, LD = DP + 4;  // columns joined in one go through LDS; padded against bank conflicts
    __shared__ __align__(16) float lds_o[NW][KV_ROW_ITEM][LD];
    __shared__ float lds_m[NW][KV_ROW_ITEM], lds_l[NW][KV_ROW_ITEM];
    __shared__ int lds_redo;
    const AttnItem it = a.items[blockIdx.x / a.n_kv];
    const int kv_head = blockIdx.x % a.n_kv;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, g = lane >> 4;
    const int in_page = (1 << a.page_shift) - 1;
    if (threadIdx.x == 0) lds_redo = 0;

    const int row = it.row0 + min(r, it.n_rows - 1);
    const int end = it.ctx + row / a.group + 1;  // tokens that this lane's row sees
    uint4 q[KC];
    {
        const E *p = static_cast<const E *>(a.q) + (int64_t)(it.tok0 + row / a.group) * a.q_stride + (kv_head * a.group + row % a.group) * D;
#pragma unroll
        for (int c = 0; c < KC; ++c) q[c] = *reinterpret_cast<const uint4 *>(p + (4 * c + g) * U);
    }

    const int steps = (it.kv1 - it.kv0 + STEP - 1) / STEP, per_wave = (steps + NW - 1) / NW;
    const int first = it.kv0 + wave * per_wave * STEP, last = min(it.kv1, first + per_wave * STEP);
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
            for (int t = 0; t < NT; ++t) s.k[t][c] = *reinterpret_cast<const uint4 *>(kp + (((4 * c + g) << a.page_shift) + k_lane + 4 * t) * U);
#pragma unroll
        for (int j = 0; j < VJ; ++j) s.v[j] = *reinterpret_cast<const uint4 *>(vp + (g * D + 16 * j + r) * U);
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
        if (pos + STEP > it.kv1) {  // behind the sequence's last token: whatever is there, it is no value
#pragma unroll
            for (int j = 0; j < VJ; ++j) s.v[j] = first_values<E>(s.v[j], it.kv1 - pos - U * g);
        }
#pragma unroll
        for (int j = 0; j < VJ; ++j) mma16<E>(o[j], s.v[j], w);
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
    // rows of several tokens: a value behind a row's own position had weight 0, but 0 times infinity is no number.  Such rows are done again
    // without touching it
    if ((it.row0 + it.n_rows - 1) / a.group != it.row0 / a.group) {
        float none = 0.f;
#pragma unroll
        for (int j = 0; j < VJ; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) none += o[j][i] * 0.f;
        __syncthreads();
        if (none != 0.f) lds_redo = 1;
        __syncthreads();
        if (lds_redo) {
            for (int i = wave; i < it.n_rows; i += NW) {
                RowState<E, D> st;
                one_row<E, D>(a, it, kv_head, it.row0 + i, it.kv0, it.kv1, st);
                put_row<E, D>(a, it, kv_head, i, st);
            }
            return;
        }
    }
    if (g == 0) lds_m[wave][r] = m, lds_l[wave][r] = l;
#pragma unroll
    for (int pass = 0; pass < D / DP; ++pass) {
        __syncthreads();
#pragma unroll
        for (int j = 0; j < DP / 16; ++j) *reinterpret_cast<floatx4 *>(&lds_o[wave][r][16 * j + 4 * g]) = o[pass * (DP / 16) + j];
        __syncthreads();
        for (int i = threadIdx.x; i < it.n_rows * (DP / 4); i += 64 * NW) {
            const int rr = i / (DP / 4), d = i % (DP / 4) * 4;
            float top = lds_m[0][rr];
#pragma unroll
            for (int w = 1; w < NW; ++w) top = fmaxf(top, lds_m[w][rr]);
            float sum = 0.f;
            floatx4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const float f = __builtin_amdgcn_exp2f(lds_m[w][rr] - top);
                sum += lds_l[w][rr] * f;
                v += *reinterpret_cast<const floatx4 *>(&lds_o[w][rr][d]) * f;
            }
            if (it.part >= 0) {
                const int64_t at = it.part + (int64_t)kv_head * it.n_rows + rr;
                *reinterpret_cast<floatx4 *>(a.part_o + at * D + pass * DP + d) = v;
                if (pass == 0 && d == 0) a.part_ml[2 * at] = top, a.part_ml[2 * at + 1] = sum;
            } else {
                const int rw = it.row0 + rr;
                const float f = sum == 0.f ? 0.f : 1.f / sum;
                E *out = static_cast<E *>(a.out) + (int64_t)(it.tok0 + rw / a.group) * a.out_stride + (kv_head * a.group + rw % a.group) * D + pass * DP + d;
                put_four(out, v * f);
            }
        }
    }
}

// Tiles of 128 rows of one key-value head (its query heads token by token): 4 wavefronts of 32 rows each share the keys and values, which
// go through LDS stage by stage (TK tokens), a stage ahead of the products.  As in the kernel above scores are formed
// transposed, here in products of 32 tokens by 32 rows: lane half h holds, of 32 tokens, rows 8 j + 4 h + i of the product for its row, and the
// second product wants chunks of u tokens in a lane.  With bf16 (u = 8) the keys of a product are therefore taken in the order that makes
// them so: product row 16 s + 8 b + 4 h + i is token 16 s + 8 h + 4 b + i (bits 2 and 3 of the number change places), which
// costs nothing as every lane names the chunk that it brings to LDS.
template <typename E> __device__ __forceinline__ int key_of_row(int row) { return sizeof(E) == 2 ? (row & ~12) | (row & 4) << 1 | (row & 8) >> 1 : row; }

template <typename E, int D> struct TileShape {
    static constexpr int TK = sizeof(E) == 2 && D <= 128 ? 64 : 32;  // tokens of a stage
    static constexpr int HALF = TK * D * (int)sizeof(E);             // bytes of its keys, and of its values
    static constexpr int LDS = 4 * HALF;                             // two stages
};

template <typename E, int D>
__global__ __launch_bounds__(256, (TileShape<E, D>::LDS <= 80 * 1024 && sizeof(E) * D <= 256) ? 2 : 1) void attn_tiles_kernel(AttnArgs a)
{
    using Shape = TileShape<E, D>;
    constexpr int U = CHUNK<E>, TK = Shape::TK, HALF = Shape::HALF, SUB = TK / 32, QC = D / (2 * U), DJ = D / 32, PK = 32 / (2 * U);
    extern __shared__ __align__(16) unsigned char lds[];
    const AttnItem it = a.items[blockIdx.x / a.n_kv];
    const int kv_head = blockIdx.x % a.n_kv;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 31, h = lane >> 5;
    const int in_page = (1 << a.page_shift) - 1;
    PageList pages(a.page_list + it.page0, (it.kv1 - 1) >> a.page_shift, it.kv0 >> a.page_shift);

    // which chunk a lane brings: of the i-th request of the stage's keys, chunk (i * 64 + lane) of [D / U][TK]; of its values, of [TK / U][D]
    const auto request = [&](int t0, int buf) {
        unsigned char *const to = lds + buf * 2 * HALF;
        int page[SUB];
#pragma unroll
        for (int i = 0; i < SUB; ++i) page[i] = pages[(t0 + 32 * i) >> a.page_shift];
#pragma unroll
        for (int i = 0; i < HALF / 4096; ++i) {
            const int n = (4 * i + wave) * 64 + lane, slot = n % TK, tok = (slot & ~31) + key_of_row<E>(slot & 31);
            const int pg = SUB == 1 ? page[0] : slot < 32 ? page[0] : page[SUB - 1];
            const E *from = half_page<E, D>(a, pg, kv_head, 0) + (((n / TK) << a.page_shift) + ((t0 + tok) & in_page)) * U;
            request16(reinterpret_cast<const __bf16 *>(from), to + (4 * i + wave) * 1024);
        }
#pragma unroll
        for (int i = 0; i < HALF / 4096; ++i) {
            const int n = (4 * i + wave) * 64 + lane, tok = n / D * U;
            const int pg = SUB == 1 ? page[0] : tok < 32 ? page[0] : page[SUB - 1];
            const E *from = half_page<E, D>(a, pg, kv_head, 1) + (size_t)((t0 + tok) & in_page) * D + n % D * U;
            request16(reinterpret_cast<const __bf16 *>(from), to + HALF + (4 * i + wave) * 1024);
        }
    };
    request(it.kv0, 0);

    const int my = wave * 32 + r, row = it.row0 + min(my, it.n_rows - 1);
    const int end = it.ctx + row / a.group + 1;  // tokens that this lane's row sees
    const int least = it.ctx + (it.row0 + min(wave * 32, it.n_rows - 1)) / a.group + 1, most = it.ctx + (it.row0 + min(wave * 32 + 31, it.n_rows - 1)) / a.group + 1;
    uint4 q[QC];
    {
        const E *p = static_cast<const E *>(a.q) + (int64_t)(it.tok0 + row / a.group) * a.q_stride + (kv_head * a.group + row % a.group) * D;
#pragma unroll
        for (int c = 0; c < QC; ++c) q[c] = *reinterpret_cast<const uint4 *>(p + (2 * c + h) * U);
    }

#pragma unroll
    for (int c = 0; c < QC; ++c) asm volatile("" : "+v"(q[c].x), "+v"(q[c].y), "+v"(q[c].z), "+v"(q[c].w));  // they have come: no wait for them below
    float m = -FLT_MAX, l = 0.f;
    floatx16 o[DJ];
#pragma unroll
    for (int j = 0; j < DJ; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[j][i] = 0.f;

    for (int t0 = it.kv0, buf = 0; t0 < it.kv1; t0 += TK, buf ^= 1) {
        wait_requests<0>();
        __syncthreads();  // this stage has come, and nobody reads the other buffer any more
        if (t0 + TK < it.kv1) request(t0 + TK, buf ^ 1);
        if (t0 >= most || wave * 32 >= it.n_rows) continue;  // none of the wavefront's rows sees any of it
        const unsigned char *const keys = lds + buf * 2 * HALF, *const vals = keys + HALF;
        floatx16 s[SUB];
#pragma unroll
        for (int b = 0; b < SUB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
        // the operands of the first products are all requested before the first is used
        constexpr int AHEAD = QC < 8 ? QC : 8;
#pragma unroll
        for (int c0 = 0; c0 < QC; c0 += AHEAD) {
            uint4 k[SUB][AHEAD];
#pragma unroll
            for (int c = 0; c < AHEAD; ++c)
#pragma unroll
                for (int b = 0; b < SUB; ++b) k[b][c] = from_lds(keys + ((2 * (c0 + c) + h) * TK + 32 * b + r) * 16);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int c = 0; c < AHEAD; ++c)
#pragma unroll
                for (int b = 0; b < SUB; ++b) mma32<E>(s[b], k[b][c], q[c0 + c]);
        }
        if (t0 + TK > least) {
#pragma unroll
            for (int b = 0; b < SUB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    if (t0 + 32 * b + i / U * 2 * U + h * U + i % U >= end) s[b][i] = -INFINITY;
        }
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < SUB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
        top = max32(top) * a.scale_log2;
        if (__any(top > m + SLACK)) {
            const float now = fmaxf(m, top), fade = __builtin_amdgcn_exp2f(m - now);
            m = now;
            l *= fade;
#pragma unroll
            for (int j = 0; j < DJ; ++j) o[j] *= fade;
        }
        uint4 w[SUB][PK];
#pragma unroll
        for (int b = 0; b < SUB; ++b)
#pragma unroll
            for (int k = 0; k < PK; ++k) {
                float p[U];
#pragma unroll
                for (int e = 0; e < U; ++e) {
                    p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][k * U + e], a.scale_log2, -m));
                    l += p[e];
                }
                w[b][k] = weights(p);
            }
        const bool tail = t0 + TK > it.kv1;
#pragma unroll
        for (int b = 0; b < SUB; ++b) {
            uint4 v[PK][DJ];
#pragma unroll
            for (int k = 0; k < PK; ++k)
#pragma unroll
                for (int j = 0; j < DJ; ++j) v[k][j] = from_lds(vals + ((32 / U * b + 2 * k + h) * D + 32 * j + r) * 16);
            if (tail) {  // behind the last token: whatever is there, it is no value
#pragma unroll
                for (int k = 0; k < PK; ++k)
#pragma unroll
                    for (int j = 0; j < DJ; ++j) v[k][j] = first_values<E>(v[k][j], it.kv1 - t0 - (32 / U * b + 2 * k + h) * U);
            }
#pragma unroll
            for (int k = 0; k < PK; ++k)
#pragma unroll
                for (int j = 0; j < DJ; ++j) mma32<E>(o[j], v[k][j], w[b][k]);
        }
    }
    if (wave * 32 >= it.n_rows) return;
    l = sum32(l);
    // a value behind a row's own position had weight 0, but 0 times infinity is no number: such rows are done again without touching it
    float none = 0.f;
#pragma unroll
    for (int j = 0; j < DJ; ++j)
#pragma unroll
        for (int i = 0; i < 16; ++i) none += o[j][i] * 0.f;
    if (__any(none != 0.f)) {
        for (int i = wave * 32; i < min(it.n_rows, wave * 32 + 32); ++i) {
            RowState<E, D> st;
            one_row<E, D>(a, it, kv_head, it.row0 + i, it.kv0, it.kv1, st);
            put_row<E, D>(a, it, kv_head, i, st);
        }
        return;
    }
    // o[j][4 k + i] is value 32 j + 8 k + 4 h + i of this lane's row
    if (it.part >= 0) {
        if (my >= it.n_rows) return;
        const int64_t at = it.part + (int64_t)kv_head * it.n_rows + my;
#pragma unroll
        for (int j = 0; j < DJ; ++j)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                *reinterpret_cast<floatx4 *>(a.part_o + at * D + 32 * j + 8 * k + 4 * h) = floatx4{o[j][4 * k], o[j][4 * k + 1], o[j][4 * k + 2], o[j][4 * k + 3]};
        if (h == 0) a.part_ml[2 * at] = m, a.part_ml[2 * at + 1] = l;
        return;
    }
    const float f = l == 0.f ? 0.f : 1.f / l;
    E *out = static_cast<E *>(a.out) + (int64_t)(it.tok0 + row / a.group) * a.out_stride + (kv_head * a.group + row % a.group) * D;
#pragma unroll
    for (int j = 0; j < DJ; ++j) {
        if constexpr (sizeof(E) == 2) {
#pragma unroll
            for (int k = 0; k < 4; k += 2) {  // the halves change 4 values each: 8 in a row for a lane
                typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
                bf16x4 x, y;
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = (__bf16)(o[j][4 * k + i] * f), y[i] = (__bf16)(o[j][4 * k + 4 + i] * f);
                const uint2 xu = __builtin_bit_cast(uint2, x), yu = __builtin_bit_cast(uint2, y);
                const auto a0 = __builtin_amdgcn_permlane32_swap(xu.x, yu.x, false, false), a1 = __builtin_amdgcn_permlane32_swap(xu.y, yu.y, false, false);
                if (my < it.n_rows) *reinterpret_cast<uint4 *>(out + 32 * j + 8 * k + 8 * h) = make_uint4(a0[0], a1[0], a0[1], a1[1]);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (my < it.n_rows)
                    *reinterpret_cast<floatx4 *>(out + 32 * j + 8 * k + 4 * h) = floatx4{o[j][4 * k], o[j][4 * k + 1], o[j][4 * k + 2], o[j][4 * k + 3]} * f;
        }
    }
}

// A block joins the parts of one row: each wavefront finds the joined maximum and weight from all parts', then groups of D / 4 threads add
// up every 1024 / D-th part, four values of the head a thread, and the groups' sums are added in their order.
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
    float m = -FLT_MAX, l = 0.f;
    for (int i = lane; i < it.n_parts; i += 64) m = fmaxf(m, a.part_ml[2 * (first + (int64_t)i * it.stride)]);
    m = wave_max(m);
    for (int i = lane; i < it.n_parts; i += 64) {
        const float2 ml = *reinterpret_cast<const float2 *>(a.part_ml + 2 * (first + (int64_t)i * it.stride));
        l += ml.y * __builtin_amdgcn_exp2f(ml.x - m);
    }
    l = wave_sum(l);
    floatx4 o = {0.f, 0.f, 0.f, 0.f};
    for (int i = g; i < it.n_parts; i += GROUPS) {
        const int64_t at = first + (int64_t)i * it.stride;
        o += *reinterpret_cast<const floatx4 *>(a.part_o + at * D + d) * __builtin_amdgcn_exp2f(a.part_ml[2 * at] - m);
    }
    *reinterpret_cast<floatx4 *>(&sums[g][d]) = o;
    __syncthreads();
    if (g == 0) {
        for (int i = 1; i < GROUPS; ++i) o += *reinterpret_cast<const floatx4 *>(&sums[i][d]);
        const int row = it.row0 + r;
        const float f = l == 0.f ? 0.f : 1.f / l;
        put_four(static_cast<E *>(a.out) + (int64_t)(it.tok0 + row / a.group) * a.out_stride + (kv_head * a.group + row % a.group) * D + d, o * f);
    }
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
    const auto lds = [&](auto t, auto d) {
        using Shape = TileShape<decltype(t), decltype(d)::value>;
        if (e == hipSuccess)
            e = hipFuncSetAttribute(reinterpret_cast<const void *>(&attn_tiles_kernel<decltype(t), decltype(d)::value>), hipFuncAttributeMaxDynamicSharedMemorySize, Shape::LDS);
    };
    for (int dim : {64, 128, 256})
        for (int dtype : {LORA_BF16, LORA_F32}) (void)by_type(dtype, dim, lds);
    return e;
}

hipError_t launch_attn_rows(const AttnArgs &a, int dtype, int dim, hipStream_t st)
{
    if ((int64_t)a.n_items * a.n_kv > INT32_MAX) return hipErrorInvalidValue;
    return by_type(dtype, dim, [&](auto e, auto d) {
        hipLaunchKernelGGL((attn_rows_kernel<decltype(e), decltype(d)::value>), dim3(a.n_items * a.n_kv), dim3(64 * ROW_WAVES), 0, st, a);
    });
}

hipError_t launch_attn_tiles(const AttnArgs &a, int dtype, int dim, hipStream_t st)
{
    if ((int64_t)a.n_items * a.n_kv > INT32_MAX) return hipErrorInvalidValue;
    return by_type(dtype, dim, [&](auto e, auto d) {
        using Shape = TileShape<decltype(e), decltype(d)::value>;
        hipLaunchKernelGGL((attn_tiles_kernel<decltype(e), decltype(d)::value>), dim3(a.n_items * a.n_kv), dim3(256), Shape::LDS, st, a);
    });
}

hipError_t launch_attn_join(const JoinArgs &a, int dtype, int dim, hipStream_t st)
{
    if ((int64_t)a.n_items * a.n_kv > INT32_MAX) return hipErrorInvalidValue;
    return by_type(dtype, dim, [&](auto e, auto d) {
        hipLaunchKernelGGL((attn_join_kernel<decltype(e), decltype(d)::value>), dim3(a.n_items * a.n_kv, a.max_rows), dim3(256), 0, st, a);
    });
}

}  // namespace lora
