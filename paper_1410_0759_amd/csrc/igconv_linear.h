// Products of token matrices with their epilogue: launch constants, and the arithmetic after the product.  Internal.
#ifndef IGCONV_LINEAR_H_
#define IGCONV_LINEAR_H_

#include "igconv_rows.h"

namespace igc {

// D[m][n] = sum_k A(m,k) B(n,k); element (m,k) of A lies at a + m * am + k * ak, one of the two strides being 1, likewise B.
//   forward          A = x (rows: tokens, k: features in),        B = w (rows: features out)
//   backward data    A = dy (rows: tokens, k: features out),      B = w read along its other index (rows: features in)
//   backward filter  A = dy (rows: features out, k: tokens),      B = x (rows: features in)
struct LinearArgs {
    const void *a, *b;
    long long am, ak, bn, bk;
    bool strided_a, strided_b;   // the reduction index runs along the rows in memory (am, bn are 1)
    bool padded_a, padded_b;     // the operand's rows in memory may be read up to the next eighth element, where (along the reduction index) zeros lie
    int M, N, K;
    // after the product: t = alpha D + bias[n]; z[m][n] = t where z is kept; t = f(t) (forward) or t f'(zin[m][n]) (backward
    // data); y[m][n] = t + beta r[m][n]
    float alpha, beta;
    const float *bias;
    int act;
    const void *zin;
    void *z;
    const void *r;
    void *y;
    long long zs, rs, ys;   // elements between rows (z is laid out as y is)
};

constexpr int kTileStep = 64, kFloatStep = 32;   // reduction indices per step (float: in parts)

struct TileArgs : LinearArgs {
    int tilesM, tilesN, group;     // tiles are taken `group` rows of tiles at a time
    int tilesPerXcd;
    int splits, stepsPerSplit;     // the reduction in ranges of steps
    float *parts;                  // [split][M][partsRow] (partsRow: N rounded up to 8), where splits > 1
    long long partsRow;
    float *columnParts;            // [split][tile column][M]: sums of the first operand's rows, or null
    int blocksA, blocksB;          // (float) blocks of 16 rows of the operands
};

// Tile shapes of linear_tiles_kernel (igconv_linear_tiles.hpp).  sa, sb: the operand's reduction index runs along its rows.
struct TileKernel {
    int bm, bn, threads;
    const void *kernel;   // null: not offered
    int wavesM;           // wavefronts along the tile's rows (ends that leave something for each)
};
constexpr int kTileShapes = 4, kStagedShape = 3 /* operands that the others have copied first */, kDirectShapes = 2;
TileKernel direct_float_kernel(bool sa, bool sb, int shape);   // float operands as they are: few tokens, small products
TileKernel float_kernel();                                           // any pass, operands in parts (igconv_linear_float.hpp)
TileKernel tile_kernel_rows(int shape, bool f32_out);          // forward: both operands' reduction indices adjacent
TileKernel tile_kernel_rows_columns(int shape, bool f32_out);  // backward data: B strided
TileKernel tile_kernel_columns(int shape, bool f32_out);       // backward filter: both strided

// One product with its epilogue on the handle's stream, by the fastest way that fits into the workspace (igconv_linear.hip), and what the fastest takes.
igcStatus product(igcHandle_t handle, igcDataType in, igcDataType out, const LinearArgs &a, void *workSpace, size_t bytes);
size_t product_room(igcHandle_t handle, igcDataType in, igcDataType out, const LinearArgs &a);

// ---- activations -----------------------------------------------------------------------------------------------------
// FINE: to float's last digits, for float results.  Otherwise for results that are rounded to bfloat16 (half a step: up to 2^-8 of
// the value): the normal distribution function then comes from the polynomial in 1 / (1 + p|v|) of Abramowitz and Stegun
// (Handbook of Mathematical Functions, 7.1.26: absolute error 1.5e-7), one exponential and one reciprocal instead of the
// library function's two ranges: a tile's epilogue has no matrix instructions to hide behind (8192 x 4096 -> 16384 with z kept: without an
// activation 797 us, with GELU 844).
__device__ __forceinline__ float fast_exp(float v) { return __builtin_amdgcn_exp2f(v * 1.44269504088896f); }
__device__ __forceinline__ float fast_rcp(float v) { return __builtin_amdgcn_rcpf(v); }

// Phi(v) = (1 + erf(v / sqrt 2)) / 2, and exp(-v v / 2) with it
template <bool FINE>
__device__ __forceinline__ float normal_cdf(float v, float *bell) {
    if constexpr (FINE) {
        *bell = expf(-0.5f * v * v);
        return 0.5f * erfcf(-v * 0.70710678118654752f);
    } else {
        const float w = v * 0.84932180028801905f;   // exp(-v v / 2) = 2^(-w w)
        const float e = __builtin_amdgcn_exp2f(-w * w);
        const float t = fast_rcp(1.f + 0.23164189f * __builtin_fabsf(v));
        const float tail = e * (t * (0.127414796f + t * (-0.142248368f + t * (0.7107068705f + t * (-0.7265760135f + t * 0.5307027145f)))));
        *bell = e;
        return v < 0.f ? tail : 1.f - tail;
    }
}

template <bool FINE>
__device__ __forceinline__ float logistic(float v) {
    if constexpr (FINE) return 1.f / (1.f + expf(-v));
    else return fast_rcp(1.f + fast_exp(-v));
}

// For products with a factor that has long vanished out there: the limit, not 0 times infinity.  (NaN: the factor is one.)
__device__ __forceinline__ float not_below(float v) { return fmaxf(v, -200.f); }
__device__ __forceinline__ float between(float v) { return fminf(fmaxf(v, -200.f), 200.f); }

template <bool FINE>
__device__ __forceinline__ float activation(int act, float v) {
    float bell;
    switch (act) {
    case IGC_ACTIVATION_SIGMOID: return logistic<FINE>(v);
    case IGC_ACTIVATION_RELU: return v > 0.f ? v : (v != v ? v : 0.f);
    case IGC_ACTIVATION_TANH:
        if constexpr (FINE) return tanhf(v);
        else   // (close to 0 the difference would lose v's digits: two terms of the series)
            return __builtin_fabsf(v) < 0.03f ? v * (1.f - v * v * (1.f / 3.f)) : 1.f - 2.f * fast_rcp(1.f + fast_exp(2.f * v));
    case IGC_ACTIVATION_GELU: return not_below(v) * normal_cdf<FINE>(v, &bell);
    case IGC_ACTIVATION_SILU: return not_below(v) * logistic<FINE>(v);
    default: return v;
    }
}

template <bool FINE>
__device__ __forceinline__ float activation_slope(int act, float v) {
    float bell;
    switch (act) {
    case IGC_ACTIVATION_SIGMOID: {
        // e / (1 + e)^2 with e = exp(-|v|): s (1 - s) would lose the digits of 1 - s
        const float e = FINE ? expf(-__builtin_fabsf(v)) : fast_exp(-__builtin_fabsf(v)), d = FINE ? 1.f / (1.f + e) : fast_rcp(1.f + e);
        return e * d * d;
    }
    case IGC_ACTIVATION_RELU: return v > 0.f ? 1.f : 0.f;
    case IGC_ACTIVATION_TANH: {
        const float e = FINE ? expf(-2.f * __builtin_fabsf(v)) : fast_exp(-2.f * __builtin_fabsf(v)), d = FINE ? 1.f / (1.f + e) : fast_rcp(1.f + e);
        return 4.f * e * d * d;
    }
    case IGC_ACTIVATION_GELU: {
        const float cdf = normal_cdf<FINE>(v, &bell);
        return cdf + between(v) * (bell * 0.39894228040143268f);
    }
    case IGC_ACTIVATION_SILU: {
        const float s = logistic<FINE>(v);
        return s + between(v) * (s * (1.f - s));
    }
    default: return 1.f;
    }
}

// f(the activation as a constant): one branch for several elements
template <int V> struct Constant { static constexpr int value = V; };
template <class F>
__device__ __forceinline__ void by_activation(int act, F f) {
    switch (act) {
    case IGC_ACTIVATION_SIGMOID: f(Constant<IGC_ACTIVATION_SIGMOID>()); break;
    case IGC_ACTIVATION_RELU: f(Constant<IGC_ACTIVATION_RELU>()); break;
    case IGC_ACTIVATION_TANH: f(Constant<IGC_ACTIVATION_TANH>()); break;
    case IGC_ACTIVATION_GELU: f(Constant<IGC_ACTIVATION_GELU>()); break;
    case IGC_ACTIVATION_SILU: f(Constant<IGC_ACTIVATION_SILU>()); break;
    default: break;
    }
}

// one result, element by element (the kernels that hold several neighbours of a row store them together)
template <class TO>
__device__ __forceinline__ void finish_element(const LinearArgs &a, int m, int n, float d) {
    constexpr bool FINE = sizeof(TO) == 4;
    float v = a.alpha * d;
    if (a.bias) v += a.bias[n];
    if (a.z) static_cast<TO *>(a.z)[m * a.zs + n] = Stored<TO>::narrow(v);
    if (a.zin) v *= activation_slope<FINE>(a.act, Stored<TO>::widen(static_cast<const TO *>(a.zin)[m * a.zs + n]));
    else v = activation<FINE>(a.act, v);
    if (a.beta != 0.f) v += a.beta * Stored<TO>::widen(static_cast<const TO *>(a.r)[m * a.rs + n]);
    static_cast<TO *>(a.y)[m * a.ys + n] = Stored<TO>::narrow(v);
}

}  // namespace igc
#endif
