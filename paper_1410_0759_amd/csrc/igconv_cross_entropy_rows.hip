// Instantiations of the tile kernels with the end that adds rows: gradients of cross entropy by its features and by its filter.
#include "igconv_cross_entropy_tiles.hpp"

namespace igc {

template <class Cfg>
static TileKernel entry(bool f32_out) {
    return {Cfg::BM, Cfg::BN, Cfg::THREADS,
            f32_out ? reinterpret_cast<const void *>(&linear_tiles_kernel<Cfg, WithRows<float>, AddendArgs>)
                    : reinterpret_cast<const void *>(&linear_tiles_kernel<Cfg, WithRows<bf16_t>, AddendArgs>),
            Cfg::WAVES_M};
}

// (the shapes of tile_kernel_rows_columns and tile_kernel_columns)
TileKernel with_rows_tile_kernel(CrossKind kind, int shape, bool f32_out) {
    if (kind == kFilterWithRows) {
        if (shape == 0) return entry<TileConfig<256, 256, 2, 4, true, true>>(f32_out);
        if (shape == 1) return entry<TileConfig<128, 128, 2, 4, true, true>>(f32_out);
        return {};
    }
    if (shape == 0) return entry<TileConfig<256, 256, 2, 4, false, true>>(f32_out);
    if (shape == 1) return entry<TileConfig<128, 128, 2, 4, false, true>>(f32_out);
    if (shape == 2) return entry<TileConfig<64, 128, 1, 4, false, true>>(f32_out);
    if (shape == 3) return entry<TileConfig<64, 128, 1, 4, false, true, 2, true>>(f32_out);
    return {};
}

}  // namespace igc
