// Instantiations of linear4_tiles_kernel.
#include "igconv_linear4_tiles.hpp"

namespace igc {

template <int GROUP>
static TileKernel of_group(int shape, bool parts, bool f32_out) {
    if (parts) {
        typedef Tile4Config<kPartsTokens, 256, 2, 4, 3, GROUP, 4> Cfg;
        typedef Tile4Config<kPartsTokens, 128, 2, 4, 3, GROUP, 4> Narrow;
        if (shape == 3) return {Narrow::BM, Narrow::BN, Narrow::THREADS, reinterpret_cast<const void *>(&linear4_tiles_kernel<Narrow, float>), Narrow::WAVES_M};
        return shape == 0 ? TileKernel{Cfg::BM, Cfg::BN, Cfg::THREADS, reinterpret_cast<const void *>(&linear4_tiles_kernel<Cfg, float>), Cfg::WAVES_M} : TileKernel{};
    }
    typedef Tile4Config<128, 256, 2, 4, 1, GROUP, 6> Wide;
    typedef Tile4Config<128, 128, 2, 4, 1, GROUP, 6> Small;
    typedef Tile4Config<256, 256, 2, 4, 1, GROUP, 3> Widest;
    typedef Tile4Config<64, 128, 1, 4, 1, GROUP, 6> Low;
    if (shape == 3)
        return {Low::BM, Low::BN, Low::THREADS,
                f32_out ? reinterpret_cast<const void *>(&linear4_tiles_kernel<Low, float>) : reinterpret_cast<const void *>(&linear4_tiles_kernel<Low, bf16_t>), Low::WAVES_M};
    if (shape == 2) {
        if constexpr (GROUP == 32) return {};      // (spills registers: 4096 x 4096 -> 8192 324 us for 332)
        else return {Widest::BM, Widest::BN, Widest::THREADS,
                     f32_out ? reinterpret_cast<const void *>(&linear4_wide_kernel<Widest, float>) : reinterpret_cast<const void *>(&linear4_wide_kernel<Widest, bf16_t>), Widest::WAVES_M};
    }
    if (shape == 0)
        return {Wide::BM, Wide::BN, Wide::THREADS,
                f32_out ? reinterpret_cast<const void *>(&linear4_tiles_kernel<Wide, float>) : reinterpret_cast<const void *>(&linear4_tiles_kernel<Wide, bf16_t>), Wide::WAVES_M};
    return {Small::BM, Small::BN, Small::THREADS,
            f32_out ? reinterpret_cast<const void *>(&linear4_tiles_kernel<Small, float>) : reinterpret_cast<const void *>(&linear4_tiles_kernel<Small, bf16_t>), Small::WAVES_M};
}

TileKernel tile4_kernel(int shape, int group, bool parts, bool f32_out) {
    if (group == 32) return of_group<32>(shape, parts, f32_out);
    return group == 64 ? of_group<64>(shape, parts, f32_out) : of_group<128>(shape, parts, f32_out);
}

}  // namespace igc
