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

}  // namespace

template <typename E, int D>
__global__ __launch_bounds__(256) void attn_plain_kernel(AttnArgs a)
{
    const AttnItem it = a.items[blockIdx.x / a.n_kv];
    const int kv_head = blockIdx.x % a.n_kv, lane = threadIdx.x & 63;
    for (int r = threadIdx.x >> 6; r < it.n_rows; r += 4) {
        RowState<E, D> st;
        one_row<E, D>(a, it, kv_head, it.row0 + r, it.kv0, it.kv1, st);
        if (it.part >= 0) {
            const int64_t at = it.part + (int64_t)kv_head * it.n_rows + r;
            for (int j = 0; j < D / 64; ++j) a.part_o[at * D + lane + 64 * j] = st.o[j];
            if (lane == 0) a.part_ml[2 * at] = st.m, a.part_ml[2 * at + 1] = st.l;
        } else {
            const int row = it.row0 + r;
            E *out = static_cast<E *>(a.out) + (int64_t)(it.tok0 + row / a.group) * a.out_stride + (kv_head * a.group + row % a.group) * D;
            const float f = st.l == 0.f ? 0.f : 1.f / st.l;
            for (int j = 0; j < D / 64; ++j) out[lane + 64 * j] = (E)(st.o[j] * f);
        }
    }
}

// A block joins the parts of one row: thread d one value of the head
template <typename E, int D>
__global__ __launch_bounds__(D) void attn_join_kernel(JoinArgs a)
{
    const JoinItem it = a.items[blockIdx.x / a.n_kv];
    const int kv_head = blockIdx.x % a.n_kv, d = threadIdx.x;
    for (int r = blockIdx.y; r < it.n_rows; r += gridDim.y) {
        const int64_t first = it.part + (int64_t)kv_head * it.n_rows + r;
        float m = -FLT_MAX;
        for (int i = 0; i < it.n_parts; ++i) m = fmaxf(m, a.part_ml[2 * (first + (int64_t)i * it.stride)]);
        float l = 0.f, o = 0.f;
        for (int i = 0; i < it.n_parts; ++i) {
            const int64_t at = first + (int64_t)i * it.stride;
            const float f = __builtin_amdgcn_exp2f(a.part_ml[2 * at] - m);
            l += a.part_ml[2 * at + 1] * f;
            o += a.part_o[at * D + d] * f;
        }
        const int row = it.row0 + r;
        E *out = static_cast<E *>(a.out) + (int64_t)(it.tok0 + row / a.group) * a.out_stride + (kv_head * a.group + row % a.group) * D;
        out[d] = (E)(l == 0.f ? 0.f : o / l);
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

hipError_t launch_attn_rows(const AttnArgs &a, int dtype, int dim, hipStream_t st)
{
    if ((int64_t)a.n_items * a.n_kv > INT32_MAX) return hipErrorInvalidValue;
    return by_type(dtype, dim, [&](auto e, auto d) {
        hipLaunchKernelGGL((attn_plain_kernel<decltype(e), decltype(d)::value>), dim3(a.n_items * a.n_kv), dim3(256), 0, st, a);
    });
}

hipError_t launch_attn_tiles(const AttnArgs &a, int dtype, int dim, hipStream_t st) { return launch_attn_rows(a, dtype, dim, st); }

hipError_t launch_attn_join(const JoinArgs &a, int dtype, int dim, hipStream_t st)
{
    if ((int64_t)a.n_items * a.n_kv > INT32_MAX) return hipErrorInvalidValue;
    return by_type(dtype, dim, [&](auto e, auto d) {
        constexpr int D = decltype(d)::value;
        hipLaunchKernelGGL((attn_join_kernel<decltype(e), D>), dim3(a.n_items * a.n_kv, KV_ROW_ITEM), dim3(D), 0, st, a);
    });
}

}  // namespace lora
