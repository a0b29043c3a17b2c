// Instantiation of linear_float_kernel.
#include "igconv_linear_float.hpp"

namespace igc {

TileKernel float_kernel() {
    typedef FloatConfig<128, 128, 2, 4> Cfg;
    return {Cfg::BM, Cfg::BN, Cfg::THREADS, reinterpret_cast<const void *>(&linear_float_kernel<Cfg>)};
}

}  // namespace igc
