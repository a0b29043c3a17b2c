// What a tile of logits leaves in place of the logits: statistics of its rows, or its part of the loss's gradient.  Internal.
#ifndef IGCONV_CROSS_ENTROPY_H_
#define IGCONV_CROSS_ENTROPY_H_

#include "igconv_linear.h"

namespace igc {

struct RowPart {
    float most, sum;      // largest logit of some of a row's columns, sum of their exp(z - most)
};

struct RowStatistics {};               // ends of a tile, in place of the type of stored results
template <class TZ> struct Slopes {};  // dz stored as TZ

// The product's columns are the vocabulary from entry `first` on.
struct CrossEnd {
    const int *targets;
    int first, V;
    // RowStatistics
    RowPart *parts;             // [tile column][M]
    float *picked;              // [M]: the targets' logits
    // Slopes: dz goes to LinearArgs::y, with zeros from the last column up to the next eighth
    float alpha;
    const float *logSum, *dloss;
    float *sums;                // column sums of dz over each wavefront's rows, [sumBlocks][sumStride], or null
    bool twoParts;              // dz in two bfloat16 parts, the second as M more rows below
    float *rests;               // [M]: what rounding to bfloat16 left of dz at the targets, or null
    long long sumStride;
};
struct CrossArgs : TileArgs {
    CrossEnd end;
};

// A product of dz with rows added before its results are rounded: to row m, where i = rowOf[m] - first is one of 0 to count - 1, factor[m] (null: 1) times row i of `from`.
template <class TO> struct WithRows {};
struct RowAddend {
    const int *rowOf;
    const float *factor;
    const uint16_t *from;
    long long stride;
    int first, count;
};
struct AddendArgs : TileArgs {
    RowAddend add;
};

enum CrossKind { kRowStatistics, kSlopes, kDataWithRows, kFilterWithRows };
// The kernels with these ends: bfloat16 tiles (as tile_kernel_rows), float operands as they are, float in parts.
TileKernel cross_tile_kernel(CrossKind kind, int shape);
TileKernel with_rows_tile_kernel(CrossKind kind, int shape, bool f32_out);
TileKernel cross_direct_float_kernel(CrossKind kind, int shape);
TileKernel cross_float_kernel(CrossKind kind);

// Such a product by the kernels with these ends: us by the figures of the choice (below 0: none of them takes it), columns of a tile, blocks of rows with column sums.
struct CrossPlan {
    double us = -1.0;
    size_t room = 0;
    bool copiesB = false;      // the second operand is copied first
    int tileColumns = 0, sumBlocks = 0;
};
CrossPlan plan_cross_product(igcHandle_t handle, CrossKind kind, igcDataType in, const LinearArgs &a, size_t room);
igcStatus cross_product(igcHandle_t handle, CrossKind kind, igcDataType in, const LinearArgs &a, const CrossEnd &end, void *workSpace, size_t bytes,
                        CrossPlan *taken);
// A product of bfloat16 operands with rows added, of any layout, and its room.
igcStatus product_with_rows(igcHandle_t handle, CrossKind kind, igcDataType out, const LinearArgs &a, const RowAddend &add, void *workSpace, size_t bytes);
size_t product_with_rows_room(igcHandle_t handle, CrossKind kind, igcDataType out, const LinearArgs &a);
// The same for at most kFewTokens tokens of bfloat16 features, of any layout (igconv_cross_entropy_few.hip).  Slopes: dz in two parts; x is copied to z (rows zs apart, from 16-byte
// boundaries), twice below each other.  One block of column sums.
constexpr int kFewTokens = 16;
int cross_few_columns(igcHandle_t handle, int N);      // of an entry of the statistics
igcStatus cross_few(igcHandle_t handle, CrossKind kind, const LinearArgs &a, const CrossEnd &end);
// what an ordinary product takes, in us by the same figures, with so much room
double product_us(igcHandle_t handle, igcDataType in, igcDataType out, const LinearArgs &a, size_t room);

// what v rounded to bfloat16 leaves (an infinity: nothing)
__device__ __forceinline__ float rest_of(float v) {
    const float high = bf16_bits_to_float(to_bf16_bits(v));
    return high - high == 0.f ? v - high : 0.f;
}
__device__ __forceinline__ float exp_of(float v) { return __builtin_amdgcn_exp2f(v * 1.44269504088896f); }

}  // namespace igc
#endif
