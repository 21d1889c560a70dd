// Attention over pages of 8-bit values (gfx950).
#include "attn_device.h"

namespace lora {

// A wavefront to a row
template <int D, bool TILE>
__global__ __launch_bounds__(256) void attn_each_kernel(AttnArgs a, const AttnItem *items)
{
    const AttnItem it = items[blockIdx.x / a.n_kv];
    for (int r = threadIdx.x >> 6; r < it.n_rows; r += 4) {
        RowState<__bf16, D> st;
        one_row<__bf16, D, E4m3>(a, it, blockIdx.x % a.n_kv, it.row0 + r, it.kv0, it.kv1, st);
        put_row<__bf16, D, TILE>(a, it, blockIdx.x % a.n_kv, r, st);
    }
}

hipError_t launch_attn_e4m3(const AttnArgs &a, int dim, KvTiles, int, hipStream_t st)
{
    const int64_t n_tiles = (int64_t)a.n_tiles * a.n_kv, n_rows = (int64_t)a.n_rows * a.n_kv + ((int64_t)a.n_short * a.n_kv + ROW_WAVES - 1) / ROW_WAVES;
    if (n_tiles > INT32_MAX || n_rows > INT32_MAX) return hipErrorInvalidValue;
    const auto launch = [&](auto d) {
        constexpr int D = decltype(d)::value;
        if (n_tiles) hipLaunchKernelGGL((attn_each_kernel<D, true>), dim3((unsigned)n_tiles), dim3(256), 0, st, a, a.tiles);
        if (n_rows) hipLaunchKernelGGL((attn_rows_kernel<__bf16, D, E4m3>), dim3((unsigned)n_rows), dim3(64 * ROW_WAVES), 0, st, a);
    };
    if (dim == 64) launch(std::integral_constant<int, 64>{});
    else if (dim == 128) launch(std::integral_constant<int, 128>{});
    else launch(std::integral_constant<int, 256>{});
    return hipGetLastError();
}

}  // namespace lora
