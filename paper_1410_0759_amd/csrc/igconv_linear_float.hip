// Instantiations of linear_float_kernel, and of linear_tiles_kernel for float.
#include "igconv_linear_float.hpp"

namespace igc {

TileKernel float_kernel() {
    typedef FloatConfig<128, 128, 2, 4> Cfg;
    return {Cfg::BM, Cfg::BN, Cfg::THREADS, reinterpret_cast<const void *>(&linear_float_kernel<Cfg>)};
}

template <bool SB>
static TileKernel few() {
    typedef TileConfig<32, 128, 1, 4, false, SB, 4> Cfg;
    return {Cfg::BM, Cfg::BN, Cfg::THREADS, reinterpret_cast<const void *>(&linear_tiles_kernel<Cfg, float>)};
}
TileKernel few_float_kernel(bool sb) { return sb ? few<true>() : few<false>(); }

}  // namespace igc
