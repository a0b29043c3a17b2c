// Instantiations of linear_tiles_kernel: backward filter, both operands read along their features.
#include "igconv_linear_tiles.hpp"

namespace igc {

template <class Cfg>
static TileKernel entry(bool f32_out) {
    return {Cfg::BM, Cfg::BN, Cfg::THREADS,
            f32_out ? reinterpret_cast<const void *>(&linear_tiles_kernel<Cfg, float>) : reinterpret_cast<const void *>(&linear_tiles_kernel<Cfg, bf16_t>)};
}

TileKernel tile_kernel_columns(int shape, bool f32_out) {
    if (shape == 0) return entry<TileConfig<256, 256, 2, 4, true, true>>(f32_out);
    if (shape == 1) return entry<TileConfig<128, 128, 2, 4, true, true>>(f32_out);
    return {};   // (a gradient of few features out is short anyway)
}

}  // namespace igc
