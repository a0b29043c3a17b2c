// Products with filters in four bits: launch constants and what the kernels share.  Internal.
#ifndef IGCONV_LINEAR4_H_
#define IGCONV_LINEAR4_H_

#include "igconv_linear_tiles.hpp"

namespace igc {

constexpr int kCodeBlock = 128, kCodeBlockBytes = 64;      // features and bytes of a block of codes

struct Linear4Args : TileArgs {      // a: x; M tokens, N rows of W, K features
    const uint8_t *codes;
    const uint16_t *scales;
    int group4;      // features to a scale
    long long scaleRow;   // elements from one group's scales to the next
};

// Tiles for more than a few tokens (igconv_linear4_tiles.hpp), shape 3 64 x 128 for the fewer of them: x bfloat16 in rows that the tiles take, or (parts) three bfloat16 parts of float x, laid out for them.
// Scales on 4-byte boundaries, scaleRow even.
constexpr int kTile4Shapes = 4, kPartsTokens = 64;      // tokens of a tile of the parts
TileKernel tile4_kernel(int shape, int group, bool parts, bool f32_out);

using bf16x2 = __bf16 __attribute__((ext_vector_type(2)));

__host__ __device__ inline long long code_row(int C) { return (long long)((C + kCodeBlock - 1) / kCodeBlock) * kCodeBlockBytes; }

// eight codes as bfloat16 numbers
__device__ __forceinline__ bf16x8 widen8(uint32_t codes) {
    const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, 1.f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, 1.f, 1);
    const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, 1.f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, 1.f, 3);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// the scales of four rows of W from row n on (zeros behind the last), as they are stored
__device__ __forceinline__ u32x2 load_scales(const uint16_t *from, int n, int N) {
    if (n + 4 <= N) return __builtin_bit_cast(u32x2, *reinterpret_cast<const Adjacent<uint16_t, 4> *>(from + n));
    uint32_t v[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (n + e < N) v[e] = from[n + e];
    return u32x2{v[0] | v[1] << 16, v[2] | v[3] << 16};
}
__device__ __forceinline__ f32x4 widen_scales(u32x2 v) {
    return f32x4{bf16_bits_to_float(v[0]), __builtin_bit_cast(float, v[0] & 0xFFFF0000u), bf16_bits_to_float(v[1]), __builtin_bit_cast(float, v[1] & 0xFFFF0000u)};
}

}  // namespace igc
#endif
