// Tensors of the feed-forward functions (layer norm, matrix products) as matrices: every position (n,h,w) is a row, its
// feature maps are the columns.  Host code, and the conversions between stored types and the float or double that is
// computed with.  Internal.
#ifndef IGCONV_ROWS_H_
#define IGCONV_ROWS_H_

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "igconv_desc.h"

namespace igc {

struct Matrix {
    long long rows = 0, stride = 0;   // stride: elements from one row to the next
    int cols = 0;
};

// The descriptor's tensor as rows of adjacent feature maps; false where its feature maps do not lie next to each other or
// its positions are not evenly spaced in the order n, h, w, or where there are more than 2^30 rows or 2^26 columns (the
// kernels' indexes are 32 bits and step past the end before they stop; so are workgroups times threads).
constexpr long long kMostRows = 1ll << 30, kMostColumns = 1ll << 26;
inline bool matrix_of(const igcTensorStruct &t, Matrix *m) {
    if ((t.dim[1] > 1 && t.stride[1] != 1) || t.dim[1] > kMostColumns) return false;
    const int order[3] = {3, 2, 0};   // from the innermost position outwards
    long long rows = 1, step = 0;
    for (int d : order) {
        if (t.dim[d] == 1) continue;
        if (rows == 1) step = t.stride[d];
        else if (t.stride[d] != rows * step) return false;
        rows *= t.dim[d];
        if (rows > kMostRows) return false;
    }
    m->rows = rows;
    m->stride = rows == 1 ? t.dim[1] : step;
    m->cols = t.dim[1];
    return true;
}

inline bool same_positions(const igcTensorStruct &a, const igcTensorStruct &b) {
    return a.dim[0] == b.dim[0] && a.dim[2] == b.dim[2] && a.dim[3] == b.dim[3];
}

struct bf16_t {
    uint16_t bits;
};

// round to nearest, ties to even (what the conversion instruction does; NaN stays NaN)
__device__ __forceinline__ uint16_t to_bf16_bits(float v) { return __builtin_bit_cast(uint16_t, (__bf16)v); }
__device__ __forceinline__ float bf16_bits_to_float(uint32_t bits) { return __builtin_bit_cast(float, bits << 16); }

template <int C> struct DppControl {
    static constexpr int value = C;
};

// two of them side by side, the first in the low half: one conversion instruction
__device__ __forceinline__ uint32_t to_bf16_pair(float lo, float hi) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

// sum over each 16, 32 or all 64 lanes, the same in all of them: neighbours, pairs, quads and eights inside a row of 16 lanes, then the rows
template <int LANES>
__device__ __forceinline__ float lanes_sum(float v) {
    auto with = [&](auto control) {
        return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(control)::value, 0xF, 0xF, true));
    };
    v = with(DppControl<0xB1>());    // quad_perm 1 0 3 2
    v = with(DppControl<0x4E>());    // quad_perm 2 3 0 1
    v = with(DppControl<0x141>());   // mirrored within eight lanes
    v = with(DppControl<0x140>());   // mirrored within sixteen
    if constexpr (LANES == 16) return v;
    if constexpr (LANES == 32) return v + __shfl_xor(v, 16);
    const int i = __builtin_bit_cast(int, v);
    return (__builtin_bit_cast(float, __builtin_amdgcn_readlane(i, 0)) + __builtin_bit_cast(float, __builtin_amdgcn_readlane(i, 16))) +
           (__builtin_bit_cast(float, __builtin_amdgcn_readlane(i, 32)) + __builtin_bit_cast(float, __builtin_amdgcn_readlane(i, 48)));
}
template <int LANES>
__device__ __forceinline__ double lanes_sum(double v) {
#pragma unroll
    for (int d = LANES / 2; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

template <class T> struct Stored;   // wide_t: what is computed with
template <> struct Stored<float> {
    typedef float wide_t;
    static constexpr igcDataType kType = IGC_DATA_FLOAT;
    static __device__ __forceinline__ float widen(float v) { return v; }
    static __device__ __forceinline__ float narrow(float v) { return v; }
};
template <> struct Stored<bf16_t> {
    typedef float wide_t;
    static constexpr igcDataType kType = IGC_DATA_BFLOAT16;
    static __device__ __forceinline__ float widen(bf16_t v) { return bf16_bits_to_float(v.bits); }
    static __device__ __forceinline__ bf16_t narrow(float v) { return bf16_t{to_bf16_bits(v)}; }
};
template <> struct Stored<double> {
    typedef double wide_t;
    static constexpr igcDataType kType = IGC_DATA_DOUBLE;
    static __device__ __forceinline__ double widen(double v) { return v; }
    static __device__ __forceinline__ double narrow(double v) { return v; }
};

// (the launch call's own return value, not the thread's last-error state, which other users of the runtime may have set)
template <class Args>
igcStatus launch_kernel(const void *kernel, const Args &args, dim3 grid, int threads, void *stream) {
    Args copy = args;
    void *argv[] = {&copy};
    return hipLaunchKernel(kernel, grid, dim3(threads), argv, 0, static_cast<hipStream_t>(stream)) == hipSuccess ? IGC_STATUS_SUCCESS
                                                                                                                     : IGC_STATUS_EXECUTION_FAILED;
}

}  // namespace igc
#endif
