// Instantiations of linear_tiles_kernel: backward data, the filter read along its features in.
#include "igconv_linear_tiles.hpp"

namespace igc {

template <class Cfg>
static TileKernel entry(bool f32_out) {
    return {Cfg::BM, Cfg::BN, Cfg::THREADS,
            f32_out ? reinterpret_cast<const void *>(&linear_tiles_kernel<Cfg, float>) : reinterpret_cast<const void *>(&linear_tiles_kernel<Cfg, bf16_t>)};
}

TileKernel tile_kernel_rows_columns(int shape, bool f32_out) {
    if (shape == 0) return entry<TileConfig<256, 256, 2, 4, false, true>>(f32_out);
    if (shape == 1) return entry<TileConfig<128, 128, 2, 4, false, true>>(f32_out);
    if (shape == 2) return entry<TileConfig<64, 128, 1, 4, false, true>>(f32_out);   // few tokens
    if (shape == 3) return entry<TileConfig<64, 128, 1, 4, false, true, 2, true>>(f32_out);   // the same, operands through registers
    return {};
}

}  // namespace igc
