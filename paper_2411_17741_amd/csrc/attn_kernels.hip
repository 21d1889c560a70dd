// Attention over the paged key-value cache (gfx950): the kernels of attn_device.h for pages of bf16 and fp32 values, and their launchers.
#include "attn_device.h"

namespace lora {

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
                const auto allow_tiles = [&](auto exact) {
                    allow(reinterpret_cast<const void *>(&attn_tiles_kernel<E, D, E, decltype(exact)::value>), TileShape<E, D>::LDS);
                    allow(reinterpret_cast<const void *>(&attn_both_kernel<E, D, E, decltype(exact)::value>), TileShape<E, D>::LDS);
                };
                allow_tiles(std::false_type{});
                if constexpr (sizeof(E) == 2) allow_tiles(std::true_type{});
                if constexpr (kv_many(sizeof(E) == 2 ? LORA_BF16 : LORA_F32, D)) allow(reinterpret_cast<const void *>(&attn_many_kernel<E, D>), MANY_LDS<E, D>);
                if constexpr (kv_pairs(sizeof(E) == 2 ? LORA_BF16 : LORA_F32, D)) {
                    static_assert(2 * TileShape<E, D>::LDS >= 4 * (32 * D * 4 + 512), "one group's results in LDS");
                    allow(reinterpret_cast<const void *>(&attn_pairs_kernel<E, D>), 2 * TileShape<E, D>::LDS);
                }
            });
    allow(reinterpret_cast<const void *>(&attn_turns_kernel<128, __bf16, false>), turn_lds(128));
    allow(reinterpret_cast<const void *>(&attn_turns_kernel<128, __bf16, true>), turn_lds(128));
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
        const auto launch = [&](auto exact) {
            constexpr bool EXACT = decltype(exact)::value;
            if (n_tiles && n_rows && way == KV_TILES_PLAIN && (n_tiles + n_rows <= BOTH_ROUNDS * TileShape<E, D>::BLOCKS * n_cu || (a.prefixes && TileShape<E, D>::BLOCKS > 1 && n_tiles + n_rows <= INT32_MAX))) {
                hipLaunchKernelGGL((attn_both_kernel<E, D, E, EXACT>), dim3((unsigned)(n_tiles + n_rows)), dim3(256), (TileShape<E, D>::LDS), st, a);
                return;
            }
            if constexpr (kv_pairs(sizeof(E) == 2 ? LORA_BF16 : LORA_F32, D))
                if (way == KV_TILES_PAIRS) {  // (no batch with prefixes)
                    hipLaunchKernelGGL((attn_pairs_kernel<E, D>), dim3((unsigned)(n_tiles + n_rows)), dim3(512), (2 * TileShape<E, D>::LDS), st, a);
                    return;
                }
            bool done = n_tiles == 0;
            if constexpr (kv_turns(sizeof(E) == 2 ? LORA_BF16 : LORA_F32, D))
                if (!done && way == KV_TILES_TURNS) {
                    hipLaunchKernelGGL((attn_turns_kernel<D, E, EXACT>), tiles, dim3(512), turn_lds(D), st, a);
                    done = true;
                }
            if constexpr (kv_many(sizeof(E) == 2 ? LORA_BF16 : LORA_F32, D))
                if (!done && way == KV_TILES_MANY) {  // (no batch with KV_EXACT tiles)
                    hipLaunchKernelGGL((attn_many_kernel<E, D>), tiles, dim3(256), (MANY_LDS<E, D>), st, a);
                    done = true;
                }
            if (!done) hipLaunchKernelGGL((attn_tiles_kernel<E, D, E, EXACT>), tiles, dim3(256), (TileShape<E, D>::LDS), st, a);
            if (n_rows) hipLaunchKernelGGL((attn_rows_kernel<E, D>), rows, dim3(64 * ROW_WAVES), 0, st, a);
        };
        if constexpr (sizeof(E) == 2)
            if (a.exact) return launch(std::true_type{});
        launch(std::false_type{});
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

hipError_t launch_shared_join(const SharedJoinArgs &a, int dtype, int dim, hipStream_t st)
{
    if ((int64_t)a.n_items * a.n_kv > INT32_MAX) return hipErrorInvalidValue;
    return by_type(dtype, dim, [&](auto e, auto d) {
        typedef decltype(e) E;
        constexpr int D = decltype(d)::value;
        hipLaunchKernelGGL((shared_join_kernel<E, D>), dim3(a.n_items * a.n_kv, (a.max_rows + SHARED_JOIN_ROWS<D> - 1) / SHARED_JOIN_ROWS<D>), dim3(256), 0, st, a);
    });
}

}  // namespace lora
