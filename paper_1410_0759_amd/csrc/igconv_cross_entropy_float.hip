// Instantiations of the tile kernels with the ends for cross entropy: float.
#include "igconv_cross_entropy_tiles.hpp"

namespace igc {

TileKernel cross_float_kernel(CrossKind kind) {
    typedef FloatConfig<128, 128, 2, 4> Cfg;
    return {Cfg::BM, Cfg::BN, Cfg::THREADS,
            kind == kRowStatistics ? reinterpret_cast<const void *>(&linear_float_kernel<Cfg, RowStatistics, CrossArgs>)
                                   : reinterpret_cast<const void *>(&linear_float_kernel<Cfg, Slopes<float>, CrossArgs>),
            Cfg::WAVES_M};
}

template <int BM>
static TileKernel direct(CrossKind kind) {
    typedef TileConfig<BM, 128, 1, 4, false, false, 4> Cfg;
    return {Cfg::BM, Cfg::BN, Cfg::THREADS,
            kind == kRowStatistics ? reinterpret_cast<const void *>(&linear_tiles_kernel<Cfg, RowStatistics, CrossArgs>)
                                   : reinterpret_cast<const void *>(&linear_tiles_kernel<Cfg, Slopes<float>, CrossArgs>),
            Cfg::WAVES_M};
}
TileKernel cross_direct_float_kernel(CrossKind kind, int shape) { return shape == 0 ? direct<64>(kind) : direct<32>(kind); }

}  // namespace igc
