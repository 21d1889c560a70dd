// Attention over the paged key-value cache (gfx950): the kernels of attn_device.h for pages of 8-bit values, and their launchers.
#include "attn_device.h"

namespace lora {

namespace {

template <typename F>
hipError_t by_dim(int dim, F f)
{
    if (dim == 64) f(std::integral_constant<int, 64>{});
    else if (dim == 128) f(std::integral_constant<int, 128>{});
    else f(std::integral_constant<int, 256>{});
    return hipGetLastError();
}

}  // namespace

hipError_t prepare_attn_e4m3_kernels()
{
    hipError_t e = hipSuccess;
    const auto allow = [&](const void *kernel, int lds) {
        if (e == hipSuccess) e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    };
    for (int dim : {64, 128, 256})
        (void)by_dim(dim, [&](auto d) {
            constexpr int D = decltype(d)::value, LDS = TileShape<__bf16, D, E4m3>::LDS;
            const auto allow_tiles = [&](auto exact) {
                allow(reinterpret_cast<const void *>(&attn_tiles_kernel<__bf16, D, E4m3, decltype(exact)::value>), LDS);
                allow(reinterpret_cast<const void *>(&attn_both_kernel<__bf16, D, E4m3, decltype(exact)::value>), LDS);
            };
            allow_tiles(std::false_type{});
            allow_tiles(std::true_type{});
            if constexpr (kv_pairs(LORA_BF16, D)) {
                static_assert(2 * LDS >= 4 * (32 * D * 4 + 512), "one group's results in LDS");
                allow(reinterpret_cast<const void *>(&attn_pairs_kernel<__bf16, D, E4m3>), 2 * LDS);
            }
        });
    allow(reinterpret_cast<const void *>(&attn_turns_kernel<128, E4m3, false>), turn_lds(128));
    allow(reinterpret_cast<const void *>(&attn_turns_kernel<128, E4m3, true>), turn_lds(128));
    return e;
}

hipError_t launch_attn_e4m3(const AttnArgs &a, int dim, KvTiles way, int n_cu, hipStream_t st)
{
    const int64_t n_tiles = (int64_t)a.n_tiles * a.n_kv, n_rows = (int64_t)a.n_rows * a.n_kv + ((int64_t)a.n_short * a.n_kv + ROW_WAVES - 1) / ROW_WAVES;
    if (n_tiles > INT32_MAX || n_rows > INT32_MAX) return hipErrorInvalidValue;
    const dim3 tiles((unsigned)n_tiles), rows((unsigned)n_rows);
    return by_dim(dim, [&](auto d) {
        constexpr int D = decltype(d)::value, LDS = TileShape<__bf16, D, E4m3>::LDS;
        const auto launch = [&](auto exact) {
            constexpr bool EXACT = decltype(exact)::value;
            if (n_tiles && n_rows && way == KV_TILES_PLAIN && (n_tiles + n_rows <= BOTH_ROUNDS * TileShape<__bf16, D>::BLOCKS * n_cu || (a.prefixes && TileShape<__bf16, D>::BLOCKS > 1 && n_tiles + n_rows <= INT32_MAX))) {
                hipLaunchKernelGGL((attn_both_kernel<__bf16, D, E4m3, EXACT>), dim3((unsigned)(n_tiles + n_rows)), dim3(256), LDS, st, a);
                return;
            }
            if constexpr (kv_pairs(LORA_BF16, D))
                if (way == KV_TILES_PAIRS) {  // (no batch with prefixes)
                    hipLaunchKernelGGL((attn_pairs_kernel<__bf16, D, E4m3>), dim3((unsigned)(n_tiles + n_rows)), dim3(512), 2 * LDS, st, a);
                    return;
                }
            bool done = n_tiles == 0;
            if constexpr (kv_turns(LORA_BF16, D))
                if (!done && way == KV_TILES_TURNS) {
                    hipLaunchKernelGGL((attn_turns_kernel<D, E4m3, EXACT>), tiles, dim3(512), turn_lds(D), st, a);
                    done = true;
                }
            if (!done) hipLaunchKernelGGL((attn_tiles_kernel<__bf16, D, E4m3, EXACT>), tiles, dim3(256), LDS, st, a);
            if (n_rows) hipLaunchKernelGGL((attn_rows_kernel<__bf16, D, E4m3>), rows, dim3(64 * ROW_WAVES), 0, st, a);
        };
        if (a.exact) launch(std::true_type{});
        else launch(std::false_type{});
    });
}

}  // namespace lora
