// Instantiations of linear_float_kernel, and of linear_tiles_kernel for float.
#include "igconv_linear_float.hpp"

namespace igc {

TileKernel float_kernel() {
    typedef FloatConfig<128, 128, 2, 4> Cfg;
    return {Cfg::BM, Cfg::BN, Cfg::THREADS, reinterpret_cast<const void *>(&linear_float_kernel<Cfg>)};
}

template <int BM, bool SA, bool SB>
static TileKernel direct() {
    typedef TileConfig<BM, 128, 1, 4, SA, SB, 4> Cfg;
    return {Cfg::BM, Cfg::BN, Cfg::THREADS, reinterpret_cast<const void *>(&linear_tiles_kernel<Cfg, float>)};
}
TileKernel direct_float_kernel(bool sa, bool sb, int shape) {
    if (sa) return shape == 0 ? direct<64, true, true>() : TileKernel{};
    if (sb) return shape == 0 ? direct<64, false, true>() : direct<32, false, true>();
    return shape == 0 ? direct<64, false, false>() : direct<32, false, false>();
}

}  // namespace igc
