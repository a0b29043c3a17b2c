// Instantiations of the tile kernels with the ends for cross entropy: bfloat16.
#include "igconv_cross_entropy_tiles.hpp"

namespace igc {

template <class Cfg>
static TileKernel entry(CrossKind kind) {
    return {Cfg::BM, Cfg::BN, Cfg::THREADS,
            kind == kRowStatistics ? reinterpret_cast<const void *>(&linear_tiles_kernel<Cfg, RowStatistics, CrossArgs>)
                                   : reinterpret_cast<const void *>(&linear_tiles_kernel<Cfg, Slopes<bf16_t>, CrossArgs>),
            Cfg::WAVES_M};
}

TileKernel cross_tile_kernel(CrossKind kind, int shape) {
    if (shape == 0) return entry<TileConfig<256, 256, 2, 4, false, false>>(kind);
    if (shape == 1) return entry<TileConfig<128, 128, 2, 4, false, false>>(kind);
    if (shape == 2) return entry<TileConfig<64, 128, 1, 4, false, false>>(kind);
    if (shape == 3) return entry<TileConfig<64, 128, 1, 4, false, false, 2, true>>(kind);
    return {};
}

}  // namespace igc
