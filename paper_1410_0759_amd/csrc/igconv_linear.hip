// Matrix products over tokens with what follows them in a feed-forward block:
//
//   forward          z = alpha x w^T + bias,  y = f(z) + beta r
//   backward data    dx = alpha (dy w) f'(z) + beta r
//   backward filter  dw = alpha dy^T x + beta dw,  dbias = alpha (column sums of dy) + beta dbias
//
// Accumulated in fp32 by the matrix instructions, in a fixed order.  Four kernels, the choice by what their steps were measured to take
// (`plan_tiles`): bfloat16 tiles of 256 x 256, 128 x 128 or 64 x 128, straight from memory or, where rows lie off 4-byte boundaries or end inside
// 16 bytes of the reduction, from copies or through registers (igconv_linear_tiles.hpp); float as it is where the filter's reading or the launch is what takes the time (the same file);
// float in bfloat16 parts (igconv_linear_float.hpp); and the one below for anything.  Few tiles: the reduction is cut into ranges, whose
// sums a second kernel adds in their order with the epilogue.
//
// Large products are bound by the matrix instructions under the card's power (zeros for numbers: 580 us for 770 in one run; 8192 x 4096 -> 16384 with
// GELU runs at 1.90 GHz, the matrix units busy for 64 % of that): 8192^3 forward 736 us, 1493 TFLOP/s,
// backward data 756, backward filter 796.  Their epilogue has no matrix instructions beside it: 8192 x 4096 -> 16384 775 us, with z kept 797, with
// GELU 844 to 867; the gradient back through GELU 789 -> 912 to 922, for 268 MB of z (55 us at a copy's rate, asked for by all compute units at once) and f'.
// Neither a quarter fewer vector instructions in f and f' nor z loaded before the last products made a difference: not kept.  Few
// tokens are bound by the filter's bytes: 8 x 4096 -> 16384 bfloat16 23 us for the tiles, 4.5 for the sum of four ranges, 31.7 the call with the filter in no
// cache; float 42 and 4.9 warm, 71 the call, 8 x 4001 -> 16384 45, 4.8 and 61.
#include "igconv_cross_entropy.h"
#include "igconv_linear_float.hpp"

namespace igc {
namespace {

constexpr long long kMostGroups = 1ll << 22;   // of a launch, to be safe with 512 threads each: their product is a 32-bit number

// ---- any strides, any alignment, no workspace -------------------------------------------------------------------------
// A workgroup computes 64 x 64 results, its four wavefronts 32 x 32 each, in steps of 32 of the reduction that go element by
// element through LDS, k innermost; the lanes of a load run along whichever index is adjacent in memory.
constexpr int kAnyTile = 64, kAnyStep = 32;

using f32x16 = float __attribute__((ext_vector_type(16)));

template <class T> struct AnyTile;
template <> struct AnyTile<float> {
    static constexpr int ROW = kAnyStep + 1;   // odd: the lanes of a fragment read lie in different banks
    typedef float lds_t;
    static __device__ __forceinline__ float raw(float v) { return v; }
    static __device__ __forceinline__ void multiply(const float *a, const float *b, int half, f32x16 &acc) {
#pragma unroll
        for (int k = 0; k < kAnyStep; k += 2) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(b[k + half], a[k + half], acc, 0, 0, 0);
    }
};
template <> struct AnyTile<bf16_t> {
    static constexpr int ROW = kAnyStep + 8;   // 16-byte fragments
    typedef uint16_t lds_t;
    static __device__ __forceinline__ uint16_t raw(bf16_t v) { return v.bits; }
    static __device__ __forceinline__ void multiply(const uint16_t *a, const uint16_t *b, int half, f32x16 &acc) {
#pragma unroll
        for (int k = 0; k < kAnyStep; k += 16)
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8 *>(b + k + 8 * half),
                                                          *reinterpret_cast<const bf16x8 *>(a + k + 8 * half), acc, 0, 0, 0);
    }
};

template <class T>
__device__ __forceinline__ void load_any(const void *from, long long sr, long long sk, int row0, int rows, int k0, int K,
                                         typename AnyTile<T>::lds_t *to) {
    const T *p = static_cast<const T *>(from);
    const int t = (int)threadIdx.x;
    if (sk == 1) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = t / 32 + 8 * i, k = t % 32;
            T v{};
            if (row0 + r < rows && k0 + k < K) v = p[(row0 + r) * sr + k0 + k];
            to[r * AnyTile<T>::ROW + k] = AnyTile<T>::raw(v);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int r = t % 64, k = t / 64 + 4 * i;
            T v{};
            if (row0 + r < rows && k0 + k < K) v = p[(k0 + k) * sk + (row0 + r) * sr];
            to[r * AnyTile<T>::ROW + k] = AnyTile<T>::raw(v);
        }
    }
}

struct AnyAddendArgs : LinearArgs {
    RowAddend add;
};
// a result of the product, with what is added before the epilogue
__device__ __forceinline__ float with_addend(const LinearArgs &, int, int, float d) { return d; }
__device__ __forceinline__ float with_addend(const AnyAddendArgs &p, int m, int n, float d) {
    const uint32_t at = (uint32_t)p.add.rowOf[m] - (uint32_t)p.add.first;
    if (at >= (uint32_t)p.add.count) return d;
    return d + (p.add.factor ? p.add.factor[m] : 1.f) * bf16_bits_to_float(p.add.from[at * p.add.stride + n]);
}

template <class T, class TO, class Args = LinearArgs>
__global__ __launch_bounds__(256) void linear_any_kernel(const Args p) {
    typedef AnyTile<T> Tile;
    __shared__ __attribute__((aligned(16))) typename Tile::lds_t la[kAnyTile * Tile::ROW], lb[kAnyTile * Tile::ROW];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, half = lane >> 5;
    const int tilesM = (p.M + kAnyTile - 1) / kAnyTile;
    const int wm = (wave >> 1) * 32, wn = (wave & 1) * 32;
    const long long tiles = (long long)tilesM * ((p.N + kAnyTile - 1) / kAnyTile);
    for (long long tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int m0 = (int)(tile % tilesM) * kAnyTile, n0 = (int)(tile / tilesM) * kAnyTile;
        f32x16 acc;
#pragma unroll
        for (int v = 0; v < 16; ++v) acc[v] = 0.f;
        for (int k0 = 0; k0 < p.K; k0 += kAnyStep) {
            load_any<T>(p.a, p.am, p.ak, m0, p.M, k0, p.K, la);
            load_any<T>(p.b, p.bn, p.bk, n0, p.N, k0, p.K, lb);
            __syncthreads();
            Tile::multiply(la + (wm + l32) * Tile::ROW, lb + (wn + l32) * Tile::ROW, half, acc);
            __syncthreads();
        }
        // (the second operand's index runs along the lanes, the first's along the registers: 8 (v / 4) + 4 half + v % 4)
        const int m = m0 + wm + l32;
#pragma unroll
        for (int v = 0; v < 16; ++v) {
            const int n = n0 + wn + 8 * (v >> 2) + 4 * half + (v & 3);
            if (m < p.M && n < p.N) finish_element<TO>(p, m, n, with_addend(p, m, n, acc[v]));
        }
    }
}

// ---- column sums (the bias gradient) -----------------------------------------------------------------------------------
struct ColumnArgs {
    const void *dy;
    long long dys;
    int M, K;
    float alpha, beta;
    float *out;
};

// lanes along 64 columns, the four wavefronts on every fourth row
template <class T>
__global__ __launch_bounds__(256) void column_sum_kernel(const ColumnArgs a) {
    __shared__ float sums[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, k = (int)blockIdx.x * 64 + lane;
    float sum = 0.f;
    if (k < a.K)
        for (int i = wave; i < a.M; i += 4) sum += Stored<T>::widen(static_cast<const T *>(a.dy)[i * a.dys + k]);
    sums[wave][lane] = sum;
    __syncthreads();
    if (wave == 0 && k < a.K) {
        float v = a.alpha * ((sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]));
        if (a.beta != 0.f) v += a.beta * a.out[k];
        a.out[k] = v;
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------
bool misaligned(const void *p, igcDataType t) { return (uintptr_t)p % (size_t)elem_size(t) != 0; }

bool known_activation(int act) {
    return act == IGC_ACTIVATION_IDENTITY || act == IGC_ACTIVATION_SIGMOID || act == IGC_ACTIVATION_RELU || act == IGC_ACTIVATION_TANH ||
           act == IGC_ACTIVATION_GELU || act == IGC_ACTIVATION_SILU;
}

// (x, w, y), (dy, w, dx) and (x, dy, dw) of one kind: bfloat16 operands with bfloat16 or float results, or float throughout
bool linear_types(igcDataType in1, igcDataType in2, igcDataType out) {
    return (in1 == IGC_DATA_BFLOAT16 && in2 == IGC_DATA_BFLOAT16 && (out == IGC_DATA_BFLOAT16 || out == IGC_DATA_FLOAT)) ||
           (in1 == IGC_DATA_FLOAT && in2 == IGC_DATA_FLOAT && out == IGC_DATA_FLOAT);
}

template <class F>
igcStatus by_types(igcDataType in, igcDataType out, F f) {
    if (in == IGC_DATA_FLOAT) return f(float(), float());
    return out == IGC_DATA_FLOAT ? f(bf16_t(), float()) : f(bf16_t(), bf16_t());
}

// `in`, `w` and `out`: x, w, y (forward) or dy, w, dx (backward data: w's index of features in is the one that stays)
igcStatus check_linear(igcTensorDescriptor_t in, igcFilterDescriptor_t w, igcTensorDescriptor_t out, bool backward, Matrix *mi, Matrix *mo) {
    if (!in || !w || !out) return IGC_STATUS_BAD_PARAM;
    if (!in->set || !w->set || !out->set) return IGC_STATUS_NOT_INITIALIZED;
    if (w->r != 1 || w->s != 1 || in->dim[1] != (backward ? w->k : w->c) || out->dim[1] != (backward ? w->c : w->k)) return IGC_STATUS_BAD_PARAM;
    if (!same_positions(*in, *out) || !non_aliasing(out->dim, out->stride)) return IGC_STATUS_BAD_PARAM;
    if (!linear_types(in->dtype, w->dtype, out->dtype) || !matrix_of(*in, mi) || !matrix_of(*out, mo)) return IGC_STATUS_NOT_SUPPORTED;
    return IGC_STATUS_SUCCESS;
}

igcStatus check_linear_filter(igcTensorDescriptor_t x, igcTensorDescriptor_t dy, igcFilterDescriptor_t dw, Matrix *mx, Matrix *mdy) {
    if (!x || !dy || !dw) return IGC_STATUS_BAD_PARAM;
    if (!x->set || !dy->set || !dw->set) return IGC_STATUS_NOT_INITIALIZED;
    if (dw->r != 1 || dw->s != 1 || x->dim[1] != dw->c || dy->dim[1] != dw->k || !same_positions(*x, *dy)) return IGC_STATUS_BAD_PARAM;
    if (!linear_types(x->dtype, dy->dtype, dw->dtype) || !matrix_of(*x, mx) || !matrix_of(*dy, mdy)) return IGC_STATUS_NOT_SUPPORTED;
    return IGC_STATUS_SUCCESS;
}

// a matrix of the epilogue (z or r): of the results' sizes and type
igcStatus check_beside(igcTensorDescriptor_t out, igcTensorDescriptor_t d, const void *p, Matrix *m) {
    if (!d || !p) return IGC_STATUS_BAD_PARAM;
    if (!d->set) return IGC_STATUS_NOT_INITIALIZED;
    if (!same_positions(*out, *d) || out->dim[1] != d->dim[1] || misaligned(p, d->dtype)) return IGC_STATUS_BAD_PARAM;
    if (d->dtype != out->dtype || !matrix_of(*d, m)) return IGC_STATUS_NOT_SUPPORTED;
    return IGC_STATUS_SUCCESS;
}

// ---- the sum of the ranges' parts, with the epilogue; the bias gradient ----------------------------------------------------
struct FinishArgs : TileArgs {
    long long partsGroups;         // workgroups of the first kind (0: one range, nothing to add)
    // the sums of the first operand's rows over ranges and columns of tiles: sums[i][M], i < sumsCount
    int sumsCount;
    float sumsAlpha, sumsBeta;
    float *sums;
};

// A thread per eight neighbours of a row; the workgroups behind them a thread per row's sum.  (One launch for both: 3333 x 1001 x 1503 backward filter
// 34.3 us for 36.1 with two.)
template <class TO>
__global__ __launch_bounds__(256) void linear_finish_kernel(const FinishArgs p) {
    if (blockIdx.x >= p.partsGroups) {
        const long long m = (blockIdx.x - p.partsGroups) * 256 + threadIdx.x;
        if (m >= p.M) return;
        float sum = 0.f;
#pragma unroll 8
        for (int i = 0; i < p.sumsCount; ++i) sum += p.columnParts[(long long)i * p.M + m];
        float v = p.sumsAlpha * sum;
        if (p.sumsBeta != 0.f) v += p.sumsBeta * p.sums[m];
        p.sums[m] = v;
        return;
    }
    const long long groups = p.partsRow / 8, id = (long long)blockIdx.x * 256 + threadIdx.x;
    const int n = (int)(id % groups) * 8;
    if (id / groups >= p.M) return;
    const int m = (int)(id / groups);
    Eight d = load8<float>(p.parts, (long long)m * p.partsRow + n);
#pragma unroll 4
    for (int s = 1; s < p.splits; ++s) {
        const Eight q = load8<float>(p.parts, ((long long)s * p.M + m) * p.partsRow + n);
#pragma unroll
        for (int e = 0; e < 8; ++e) d.v[e] += q.v[e];
    }
    Eight bias;
#pragma unroll
    for (int e = 0; e < 8; ++e) bias.v[e] = p.bias && n + e < p.N ? p.bias[n + e] : 0.f;
    if (n + 8 <= p.N) {
        finish8<TO>(p, m, n, d, bias);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (n + e < p.N) finish_element<TO>(p, m, n + e, d.v[e]);
    }
}

// ---- operands that are not laid out for the tiles --------------------------------------------------------------------------
struct PackOperand {
    const void *from;
    uint16_t *to;
    long long rows, stride, toRow;     // of the matrix in memory, elements
    int cols, groups;                  // (rows on 16-byte boundaries) groups of eight columns
    int strided, blocks;               // (parts) whether the reduction index runs along the rows; blocks of 16 of the other index
    long long workgroups;
};
struct PackArgs {
    PackOperand o[2];
};
template <class T>
struct __attribute__((packed, aligned(sizeof(T)))) EightStored {
    T v[8];
};

// a matrix copied into rows on 16-byte boundaries, zeros up to the next eighth column
__global__ __launch_bounds__(256) void linear_pack_kernel(const PackArgs args) {
    const bool second = (long long)blockIdx.x >= args.o[0].workgroups;
    const PackOperand &p = args.o[second ? 1 : 0];
    const long long id = ((long long)blockIdx.x - (second ? args.o[0].workgroups : 0)) * 256 + threadIdx.x;
    const long long row = id / p.groups;
    const int c = (int)(id % p.groups) * 8, left = p.cols - c;
    if (row >= p.rows) return;
    const uint16_t *from = static_cast<const uint16_t *>(p.from) + row * p.stride + c;
    EightStored<uint16_t> raw;
    if (left >= 8) {
        raw = *reinterpret_cast<const EightStored<uint16_t> *>(from);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            raw.v[e] = 0;
            if (e < left) raw.v[e] = from[e];
        }
    }
    u32x4 q;
#pragma unroll
    for (int e = 0; e < 4; ++e) q[e] = raw.v[2 * e] | (uint32_t)raw.v[2 * e + 1] << 16;
    *reinterpret_cast<u32x4 *>(p.to + row * p.toRow + c) = q;
}

// Eight neighbours along the reduction index as parts (igconv_linear_float.hpp): by truncation, so that all parts have x's sign.
__device__ __forceinline__ void store_parts(uint16_t *unit, int slot, const float (&x)[8]) {
    u32x4 part[kFloatParts];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        uint32_t bits[kFloatParts][2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float v = x[2 * e + i];
            const uint32_t all = __builtin_bit_cast(uint32_t, v), sign = all & 0x80000000u;
            const bool finite = (all & 0x7F800000u) != 0x7F800000u;
            uint32_t h = finite ? all & 0xFFFF0000u : (all & 0x007FFFFFu ? 0x7FC00000u : all);   // (an undefined value must not become an infinity)
            const float r = finite ? v - __builtin_bit_cast(float, h) : 0.f;
            uint32_t m = __builtin_bit_cast(uint32_t, r) & 0xFFFF0000u;
            uint32_t l = __builtin_bit_cast(uint32_t, r - __builtin_bit_cast(float, m)) & 0xFFFF0000u;
            const uint32_t least = (all & 0x7FFFFFFFu) != 0u ? sign | 0x00010000u : 0u;   // in place of a part that is zero though x is not
            if ((h & 0x7FFFFFFFu) == 0u) h = least;
            if ((m & 0x7FFFFFFFu) == 0u) m = least;
            if ((l & 0x7FFFFFFFu) == 0u) l = least;
            bits[0][i] = h >> 16; bits[1][i] = m >> 16; bits[2][i] = l >> 16;
        }
#pragma unroll
        for (int q = 0; q < kFloatParts; ++q) part[q][e] = bits[q][0] | bits[q][1] << 16;
    }
#pragma unroll
    for (int q = 0; q < kFloatParts; ++q) *reinterpret_cast<u32x4 *>(unit + (q * kUnitBytes + slot * 16) / 2) = part[q];
}

// A float operand as units of parts.  Reduction index adjacent: a wavefront makes the units of 16 rows by 32 indices, a lane 8 of a row.
// Else a wavefront's lanes take 64 adjacent rows of the operand (columns of the matrix), 8 indices at a time.
__global__ __launch_bounds__(256) void linear_parts_pack_kernel(const PackArgs args) {
    const bool second = (long long)blockIdx.x >= args.o[0].workgroups;
    const PackOperand &p = args.o[second ? 1 : 0];
    const long long task = ((long long)blockIdx.x - (second ? args.o[0].workgroups : 0)) * 4 + (threadIdx.x >> 6);
    const int lane = threadIdx.x & 63, l16 = lane & 15, g = lane >> 4;
    const float *from = static_cast<const float *>(p.from);
    if (!p.strided) {
        const int steps = (p.cols + kFloatStep - 1) / kFloatStep;
        const long long block = task / steps, row = block * 16 + l16;
        const int step = (int)(task % steps), k = step * kFloatStep + g * 8, left = p.cols - k;
        if (block >= p.blocks) return;
        float x[8];
        if (row < p.rows && left >= 8) {
            const EightStored<float> raw = *reinterpret_cast<const EightStored<float> *>(from + row * p.stride + k);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = raw.v[e];
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = 0.f;
                if (row < p.rows && e < left) x[e] = from[row * p.stride + k + e];
            }
        }
        store_parts(p.to + ((long long)step * p.blocks + block) * (kFloatParts * kUnitBytes / 2), lane, x);
    } else {
        const int groups = (p.blocks + 3) / 4;
        const int step = (int)(task / groups), block = (int)(task % groups) * 4 + g, col = block * 16 + l16;
        if ((long long)step * kFloatStep >= p.rows) return;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const long long k = (long long)step * kFloatStep + c * 8;
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = k + e < p.rows && col < p.cols ? from[(k + e) * p.stride + col] : 0.f;
            if (block < p.blocks) store_parts(p.to + ((long long)step * p.blocks + block) * (kFloatParts * kUnitBytes / 2), c * 16 + l16, x);
        }
    }
}

// ---- the choice of a tile and of the ranges -------------------------------------------------------------------------------
struct OperandPlan {
    bool pack = false;
    long long rows = 0, stride = 0, toRow = 0;   // of the matrix in memory
    int cols = 0, blocks = 0;
    size_t at = 0, bytes = 0;                    // its copy in the workspace
};
struct TilePlan {
    bool tiles = false;      // (else the kernel for any layout)
    TileKernel k{};
    int tilesM = 0, tilesN = 0, splits = 1, stepsPerSplit = 0;
    OperandPlan a, b;
    size_t partsAt = 0, sumsAt = 0, bytes = 0;   // of workspace
    double us = 1e300;
};

long long round_up(long long v, long long to) { return (v + to - 1) / to * to; }

TileKernel tile_kernel(bool sa, bool sb, int shape, bool f32_out) {
    return sa ? tile_kernel_columns(shape, f32_out) : (sb ? tile_kernel_rows_columns(shape, f32_out) : tile_kernel_rows(shape, f32_out));
}

// Whether the tiles take an operand as it lies: rows on boundaries of 4 bytes, of whole pieces of 16 along the reduction index (float: of any length), of
// whole words across it; no row inside another; a tile's reach below 2^31 bytes.  (Rows on 4-byte boundaries as against copies on 16: forward 1000^3 9.6 us for 13.5,
// 8192 x 4096 x 4096 212 for 221, filter gradient 208 for 248; on 16-byte boundaries 9.5, 201 and 207.)
bool fits(const OperandPlan &o, bool strided, int elem, const void *p, bool padded = false) {
    const int words = 4 / elem, most = (1 << 23) / elem;
    return (padded || o.cols % (strided || elem == 4 ? words : 16 / elem) == 0) && (o.rows == 1 || (o.stride % words == 0 && o.stride >= o.cols)) &&
           std::max(o.stride, (long long)o.cols) < most && (uintptr_t)p % 4 == 0;
}

// The matrix of an operand, and whether it has to be copied: a bfloat16 one that does not fit, a float one to have its parts.
OperandPlan operand_plan(bool strided, long long n, long long K, long long ns, long long ks, bool f32, const void *p, bool padded = false) {
    OperandPlan o;
    o.rows = strided ? K : n;
    o.cols = (int)(strided ? n : K);
    o.stride = strided ? ks : ns;
    o.pack = f32 || !fits(o, strided, 2, p, padded);
    o.toRow = round_up(o.cols, 8);
    o.blocks = (int)((n + 15) / 16);
    if (o.pack)
        o.bytes = f32 ? (size_t)((K + kFloatStep - 1) / kFloatStep) * o.blocks * (kFloatParts * kUnitBytes) : (size_t)round_up(o.rows * o.toRow * 2, 256);
    return o;
}

// us of a step of a workgroup alone on its compute unit and with another beside it, and of a tile's start and epilogue.  Measured: forward 8192^3 is 512
// steps of 256 x 256, 786 us, or 1024 of 128 x 128 two by two, 1003; 2048^3 32 steps, 44, 21.4 (alone) and, 64 x 128 two by two, 24.7;
// 2048 x 1024 -> 1024 16 steps of 64 x 128 alone, 9.7.  Float 4096^3: 512 steps, 560.  With the pieces through registers a step waits for memory: 8 x 4097 ->
// 8000, 252 workgroups of 17 steps, 34 us, 504 of 9, 24 - with copies first 41; 1000 x 1001 -> 1001, 16 steps, 28, with copies first 16.
struct ShapeCost {
    int per_cu;
    double alone, full, ends;
};
constexpr ShapeCost kShapeCost[kTileShapes] = {{1, 1.40, 1.40, 8.0}, {2, 0.45, 0.98, 2.5}, {2, 0.42, 0.60, 2.0}, {2, 1.65, 2.00, 2.0}};
constexpr ShapeCost kFloatCost = {1, 1.09, 1.09, 4.0}, kDirectCost[kDirectShapes] = {{2, 1.10, 2.00, 2.5}, {2, 0.60, 1.00, 2.0}};
// The second launch that adds the ranges' parts, and their bytes, written and read mostly in the last-level cache; bytes per us from memory, and what one
// workgroup reads of them, whatever its tile (8 x 4096 -> 16384, the filter not in the last-level cache: 128 workgroups 40 us, 256 36, 512 29).
// What the ends for cross entropy add to a tile's, by shape.
constexpr double kCrossEnds[kTileShapes] = {4.0, 2.0, 1.0, 1.0};
constexpr double kPartsLaunch = 2.5, kPartsBytes = 6e6, kMemoryBytes = 4.9e6, kWorkgroupBytes = 16e3;

// cross: null, or the end of a product for cross entropy (of logits: bfloat16 or float, in one range; with rows added: bfloat16)
TilePlan plan_tiles(const igcContext *h, igcDataType in, igcDataType out, const LinearArgs &a, bool sums, size_t room, const CrossKind *cross = nullptr) {
    TilePlan pl;
    const bool f32 = in == IGC_DATA_FLOAT, sa = a.strided_a, sb = a.strided_b;
    const OperandPlan oa = operand_plan(sa, a.M, a.K, a.am, a.ak, f32, a.a, a.padded_a), ob = operand_plan(sb, a.N, a.K, a.bn, a.bk, f32, a.b, a.padded_b);
    double &best = pl.us;
    // the product by kernel k in `splits` ranges of steps of `step`, its operands copied first or not
    auto consider = [&](const TileKernel &k, const ShapeCost &sc, int step, int splits, bool copied) {
        const int steps = (a.K + step - 1) / step, per = (steps + splits - 1) / splits;
        if (!k.kernel || (steps + per - 1) / per != splits) return;
        const size_t at_b = copied ? oa.bytes : 0, at = copied ? oa.bytes + ob.bytes : 0;
        const long long tm = (a.M + k.bm - 1) / k.bm, tn = (a.N + k.bn - 1) / k.bn, units = tm * tn * splits;
        const size_t parts = splits > 1 ? (size_t)splits * a.M * round_up(a.N, 8) * 4 : 0, sum_bytes = sums ? (size_t)(splits * tn) * a.M * 4 : 0;
        // (a launch holds 2^32 threads: of the sum over the ranges one to 32 bytes, of the copies 256 to 4 KB of bfloat16 or 12 KB of parts)
        if (at + parts + sum_bytes > room || units > kMostGroups || parts / splits >= (1ull << 36) || at >= (1ull << 35)) return;
        const long long slots = (long long)h->computeUnits * sc.per_cu, whole = units / slots, rest = units % slots;
        // what a unit, two side by side and one alone, takes: its steps, or what it reads from memory
        const double read = (double)(a.K * ((long long)a.M + a.N) * elem_size(in)) / (double)units;
        const double full = std::max(per * sc.full + sc.ends, read * sc.per_cu * h->computeUnits / kMemoryBytes), one = std::max(per * sc.alone + sc.ends, read / kWorkgroupBytes);
        const double us = whole * full + (rest == 0 ? 0.0 : (rest <= h->computeUnits ? one : full)) + (splits > 1 ? kPartsLaunch + (double)parts * 2 / kPartsBytes : 0.0) +
                          (at > 0 ? kPartsLaunch + (double)at * 2 / kMemoryBytes : 0.0);
        if (us >= best) return;
        best = us;
        pl.tiles = true;
        pl.k = k;
        pl.tilesM = (int)tm; pl.tilesN = (int)tn; pl.splits = splits; pl.stepsPerSplit = per;
        pl.a = oa;
        pl.b = ob;
        pl.a.pack = oa.pack && copied;
        pl.b.pack = ob.pack && copied;
        pl.b.at = at_b;
        pl.partsAt = at;
        pl.sumsAt = at + parts;
        pl.bytes = at + parts + sum_bytes;
    };
    // (no range without a step)
    auto most_splits = [&](int step) { return cross && *cross <= kSlopes ? 1 : std::min(64, (a.K + step - 1) / step); };
    auto more = [&](const ShapeCost &sc, int shape) { return cross && *cross <= kSlopes ? ShapeCost{sc.per_cu, sc.alone, sc.full, sc.ends + kCrossEnds[shape]} : sc; };
    if (f32) {
        // (rows that end inside a piece begin off 16-byte boundaries as well: 1024 x 2050 -> 1000 65 steps of 32 x 128 49 us, 1024 x 2048 -> 1000 64 steps 45;
        // in parts both 42)
        const double steps = a.K % 4 != 0 && !(sa && sb) ? 1.1 : 1.0;
        if (fits(oa, sa, 4, a.a) && fits(ob, sb, 4, a.b))
            for (int shape = 0; shape < kDirectShapes; ++shape) {
                const ShapeCost sc = more(kDirectCost[shape], 2);
                for (int splits = 1; splits <= most_splits(kFloatStep); ++splits)
                    consider(cross ? cross_direct_float_kernel(*cross, shape) : direct_float_kernel(sa, sb, shape), {sc.per_cu, sc.alone * steps, sc.full * steps, sc.ends}, kFloatStep, splits, false);
            }
        for (int splits = 1; splits <= most_splits(kFloatStep); ++splits) consider(cross ? cross_float_kernel(*cross) : float_kernel(), more(kFloatCost, 1), kFloatStep, splits, true);
        return pl;
    }
    // (a tile's reach stays within 31 bits)
    if ((oa.pack ? oa.toRow : oa.stride) >= (1ll << 22) || (ob.pack ? ob.toRow : ob.stride) >= (1ll << 22)) return pl;
    for (int shape = 0; shape < (oa.pack || ob.pack ? kTileShapes : kStagedShape); ++shape)
        for (int splits = 1; splits <= most_splits(kTileStep); ++splits)
            consider(!cross ? tile_kernel(sa, sb, shape, out == IGC_DATA_FLOAT)
                            : (*cross <= kSlopes ? cross_tile_kernel(*cross, shape) : with_rows_tile_kernel(*cross, shape, out == IGC_DATA_FLOAT)),
                     more(kShapeCost[shape], shape), kTileStep, splits, shape < kStagedShape);
    return pl;
}

bool on16(const void *p) { return (uintptr_t)p % 16 == 0; }

// the copies that the plan asks for; the tiles' operands
igcStatus pack_operands(const TilePlan &pl, bool f32, const LinearArgs &a, TileArgs &t, uint8_t *workSpace, void *stream) {
    PackArgs p{};
    long long workgroups = 0;
    int n = 0;
    for (int i = 0; i < 2; ++i) {
        const OperandPlan &o = i ? pl.b : pl.a;
        if (!o.pack) continue;
        const bool strided = i ? a.strided_b : a.strided_a;
        PackOperand &q = p.o[n++];
        q.from = i ? a.b : a.a;
        q.to = reinterpret_cast<uint16_t *>(workSpace + o.at);
        q.rows = o.rows; q.stride = o.stride; q.toRow = o.toRow; q.cols = o.cols; q.groups = (int)(o.toRow / 8);
        q.strided = strided ? 1 : 0; q.blocks = o.blocks;
        const long long steps = (a.K + kFloatStep - 1) / kFloatStep;
        q.workgroups = f32 ? (steps * (strided ? (o.blocks + 3) / 4 : o.blocks) + 3) / 4 : (o.rows * q.groups + 255) / 256;
        workgroups += q.workgroups;
        (i ? t.b : t.a) = q.to;
        (i ? t.bn : t.am) = strided ? 1 : o.toRow;
        (i ? t.bk : t.ak) = strided ? o.toRow : 1;
        (i ? t.blocksB : t.blocksA) = o.blocks;
    }
    if (n == 0) return IGC_STATUS_SUCCESS;
    return launch_kernel(f32 ? reinterpret_cast<const void *>(&linear_parts_pack_kernel) : reinterpret_cast<const void *>(&linear_pack_kernel), p,
                         dim3((unsigned)workgroups), 256, stream);
}

// column sums of dy, [M of the product], beside backward filter
struct SumsOut {
    float *out = nullptr;
    float alpha = 1.f, beta = 0.f;
};

// the plan's tiles in the kernels' arguments, operands copied where it says so
igcStatus begin_tiles(igcHandle_t handle, const TilePlan &pl, igcDataType in, const LinearArgs &a, uint8_t *ws, TileArgs &t) {
    static_cast<LinearArgs &>(t) = a;
    t.tilesM = pl.tilesM; t.tilesN = pl.tilesN;
    t.group = std::min(pl.tilesM, 4);
    t.splits = pl.splits; t.stepsPerSplit = pl.stepsPerSplit;
    t.tilesPerXcd = (int)(((long long)pl.tilesM * pl.tilesN * pl.splits + 7) / 8);
    t.parts = reinterpret_cast<float *>(ws + pl.partsAt);
    t.partsRow = round_up(a.N, 8);
    return pack_operands(pl, in == IGC_DATA_FLOAT, a, t, ws, handle->stream);
}

// after tiles in ranges
igcStatus join_ranges(igcHandle_t handle, igcDataType out, const TileArgs &t) {
    FinishArgs f{};
    static_cast<TileArgs &>(f) = t;
    f.partsGroups = (t.M * (t.partsRow / 8) + 255) / 256;
    return launch_kernel(out == IGC_DATA_FLOAT ? reinterpret_cast<const void *>(&linear_finish_kernel<float>) : reinterpret_cast<const void *>(&linear_finish_kernel<bf16_t>), f,
                         dim3((unsigned)f.partsGroups), 256, handle->stream);
}

dim3 any_grid(const LinearArgs &a) {
    return dim3((unsigned)std::min((long long)((a.M + kAnyTile - 1) / kAnyTile) * ((a.N + kAnyTile - 1) / kAnyTile), kMostGroups));
}

igcStatus run_product(igcHandle_t handle, igcDataType in, igcDataType out, const LinearArgs &a, void *workSpace, size_t bytes, const SumsOut &sums = SumsOut(),
                      bool *summed = nullptr) {
    const TilePlan pl = plan_tiles(handle, in, out, a, sums.out != nullptr, workSpace && on16(workSpace) ? bytes : 0);
    if (pl.tiles) {
        TileArgs t{};
        uint8_t *ws = static_cast<uint8_t *>(workSpace);
        igcStatus rc = begin_tiles(handle, pl, in, a, ws, t);
        if (rc != IGC_STATUS_SUCCESS) return rc;
        t.columnParts = sums.out ? reinterpret_cast<float *>(ws + pl.sumsAt) : nullptr;
        rc = launch_kernel(pl.k.kernel, t, dim3((unsigned)t.tilesPerXcd * 8u), pl.k.threads, handle->stream);
        if (rc == IGC_STATUS_SUCCESS && (pl.splits > 1 || sums.out)) {
            FinishArgs f{};
            static_cast<TileArgs &>(f) = t;
            f.partsGroups = pl.splits > 1 ? (a.M * (t.partsRow / 8) + 255) / 256 : 0;
            f.sumsCount = pl.splits * pl.tilesN;
            f.sums = sums.out; f.sumsAlpha = sums.alpha; f.sumsBeta = sums.beta;
            const long long sum_groups = sums.out ? (a.M + 255) / 256 : 0;
            rc = launch_kernel(out == IGC_DATA_FLOAT ? reinterpret_cast<const void *>(&linear_finish_kernel<float>)
                                                     : reinterpret_cast<const void *>(&linear_finish_kernel<bf16_t>),
                               f, dim3((unsigned)(f.partsGroups + sum_groups)), 256, handle->stream);
            if (summed) *summed = sums.out != nullptr;
        }
        return rc;
    }
    return by_types(in, out, [&](auto ti, auto to) {
        return launch_kernel(reinterpret_cast<const void *>(&linear_any_kernel<decltype(ti), decltype(to)>), a, any_grid(a), 256, handle->stream);
    });
}

// the passes as D[m][n] = sum_k A(m,k) B(n,k)
LinearArgs forward_sizes(const Matrix &x, const igcFilterStruct &w) {
    LinearArgs a{};
    a.am = x.stride; a.ak = 1; a.bn = w.c; a.bk = 1;
    a.M = (int)x.rows; a.N = w.k; a.K = w.c;
    return a;
}
LinearArgs backward_data_sizes(const Matrix &dy, const igcFilterStruct &w) {
    LinearArgs a{};
    a.am = dy.stride; a.ak = 1; a.bn = 1; a.bk = w.c; a.strided_b = true;
    a.M = (int)dy.rows; a.N = w.c; a.K = w.k;
    return a;
}
LinearArgs backward_filter_sizes(const Matrix &x, const Matrix &dy, const igcFilterStruct &dw) {
    LinearArgs a{};
    a.am = 1; a.ak = dy.stride; a.bn = 1; a.bk = x.stride; a.strided_a = a.strided_b = true;
    a.M = dw.k; a.N = dw.c; a.K = (int)x.rows;
    return a;
}
constexpr size_t kNoLimit = ~(size_t)0;

}  // namespace

igcStatus product(igcHandle_t handle, igcDataType in, igcDataType out, const LinearArgs &a, void *workSpace, size_t bytes) {
    return run_product(handle, in, out, a, workSpace, bytes);
}
size_t product_room(igcHandle_t handle, igcDataType in, igcDataType out, const LinearArgs &a) { return plan_tiles(handle, in, out, a, false, kNoLimit).bytes; }
double product_us(igcHandle_t handle, igcDataType in, igcDataType out, const LinearArgs &a, size_t room) { return plan_tiles(handle, in, out, a, false, room).us; }

static CrossPlan cross_plan(const TilePlan &pl) {
    CrossPlan c;
    if (!pl.tiles) return c;
    c.us = pl.us;
    c.room = pl.bytes;
    c.copiesB = pl.b.pack;
    c.tileColumns = pl.k.bn;
    c.sumBlocks = pl.tilesM * pl.k.wavesM;
    return c;
}
CrossPlan plan_cross_product(igcHandle_t handle, CrossKind kind, igcDataType in, const LinearArgs &a, size_t room) {
    return cross_plan(plan_tiles(handle, in, in, a, false, room, &kind));
}
igcStatus cross_product(igcHandle_t handle, CrossKind kind, igcDataType in, const LinearArgs &a, const CrossEnd &end, void *workSpace, size_t bytes, CrossPlan *taken) {
    const TilePlan pl = plan_tiles(handle, in, in, a, false, bytes, &kind);
    *taken = cross_plan(pl);
    if (!pl.tiles) return IGC_STATUS_NOT_SUPPORTED;
    CrossArgs t{};
    const igcStatus rc = begin_tiles(handle, pl, in, a, static_cast<uint8_t *>(workSpace), t);
    if (rc != IGC_STATUS_SUCCESS) return rc;
    t.end = end;
    return launch_kernel(pl.k.kernel, t, dim3((unsigned)t.tilesPerXcd * 8u), pl.k.threads, handle->stream);
}

igcStatus product_with_rows(igcHandle_t handle, CrossKind kind, igcDataType out, const LinearArgs &a, const RowAddend &add, void *workSpace, size_t bytes) {
    const TilePlan pl = plan_tiles(handle, IGC_DATA_BFLOAT16, out, a, false, bytes, &kind);
    if (!pl.tiles) {
        AnyAddendArgs t{};
        static_cast<LinearArgs &>(t) = a;
        t.add = add;
        return launch_kernel(out == IGC_DATA_FLOAT ? reinterpret_cast<const void *>(&linear_any_kernel<bf16_t, float, AnyAddendArgs>)
                                                   : reinterpret_cast<const void *>(&linear_any_kernel<bf16_t, bf16_t, AnyAddendArgs>), t, any_grid(a), 256, handle->stream);
    }
    AddendArgs t{};
    igcStatus rc = begin_tiles(handle, pl, IGC_DATA_BFLOAT16, a, static_cast<uint8_t *>(workSpace), t);
    if (rc != IGC_STATUS_SUCCESS) return rc;
    t.add = add;
    rc = launch_kernel(pl.k.kernel, t, dim3((unsigned)t.tilesPerXcd * 8u), pl.k.threads, handle->stream);
    return rc == IGC_STATUS_SUCCESS && pl.splits > 1 ? join_ranges(handle, out, t) : rc;
}
size_t product_with_rows_room(igcHandle_t handle, CrossKind kind, igcDataType out, const LinearArgs &a) {
    return plan_tiles(handle, IGC_DATA_BFLOAT16, out, a, false, kNoLimit, &kind).bytes;
}

}  // namespace igc

using namespace igc;

extern "C" {

igcStatus igcGetLinearForwardWorkspaceSize(igcHandle_t handle, igcTensorDescriptor_t xDesc, igcFilterDescriptor_t wDesc,
                                           igcTensorDescriptor_t yDesc, size_t *sizeInBytes) {
    if (!handle || !sizeInBytes) return IGC_STATUS_BAD_PARAM;
    Matrix x, y;
    const igcStatus st = check_linear(xDesc, wDesc, yDesc, false, &x, &y);
    if (st != IGC_STATUS_SUCCESS) return st;
    *sizeInBytes = plan_tiles(handle, xDesc->dtype, yDesc->dtype, forward_sizes(x, *wDesc), false, kNoLimit).bytes;
    return IGC_STATUS_SUCCESS;
}

igcStatus igcLinearForward(igcHandle_t handle, const void *alpha, igcTensorDescriptor_t xDesc, const void *x, igcFilterDescriptor_t wDesc,
                           const void *w, void *workSpace, size_t workSpaceSizeInBytes, const void *bias, int activation, const void *beta,
                           igcTensorDescriptor_t rDesc, const void *r, igcTensorDescriptor_t yDesc, void *z, void *y) {
    if (!handle || !alpha || !beta || !x || !w || !y || !known_activation(activation)) return IGC_STATUS_BAD_PARAM;
    Matrix mx, my, mr;
    igcStatus st = check_linear(xDesc, wDesc, yDesc, false, &mx, &my);
    if (st != IGC_STATUS_SUCCESS) return st;
    LinearArgs a = forward_sizes(mx, *wDesc);
    a.alpha = *static_cast<const float *>(alpha);
    a.beta = *static_cast<const float *>(beta);
    if (a.beta != 0.f && (st = check_beside(yDesc, rDesc, r, &mr)) != IGC_STATUS_SUCCESS) return st;
    if (misaligned(x, xDesc->dtype) || misaligned(w, wDesc->dtype) || misaligned(y, yDesc->dtype) || misaligned(z, yDesc->dtype) ||
        misaligned(bias, IGC_DATA_FLOAT))
        return IGC_STATUS_BAD_PARAM;
    a.a = x;
    a.b = w;
    a.bias = static_cast<const float *>(bias);
    a.act = activation;
    a.z = z; a.zs = my.stride;
    a.r = r; a.rs = mr.stride;
    a.y = y; a.ys = my.stride;
    return run_product(handle, xDesc->dtype, yDesc->dtype, a, workSpace, workSpaceSizeInBytes);
}

igcStatus igcGetLinearBackwardDataWorkspaceSize(igcHandle_t handle, igcFilterDescriptor_t wDesc, igcTensorDescriptor_t dyDesc,
                                                igcTensorDescriptor_t dxDesc, size_t *sizeInBytes) {
    if (!handle || !sizeInBytes) return IGC_STATUS_BAD_PARAM;
    Matrix dy, dx;
    const igcStatus st = check_linear(dyDesc, wDesc, dxDesc, true, &dy, &dx);
    if (st != IGC_STATUS_SUCCESS) return st;
    *sizeInBytes = plan_tiles(handle, dyDesc->dtype, dxDesc->dtype, backward_data_sizes(dy, *wDesc), false, kNoLimit).bytes;
    return IGC_STATUS_SUCCESS;
}

igcStatus igcLinearBackwardData(igcHandle_t handle, const void *alpha, igcFilterDescriptor_t wDesc, const void *w, igcTensorDescriptor_t dyDesc,
                                const void *dy, void *workSpace, size_t workSpaceSizeInBytes, int activation, igcTensorDescriptor_t zDesc,
                                const void *z, const void *beta, igcTensorDescriptor_t rDesc, const void *r, igcTensorDescriptor_t dxDesc,
                                void *dx) {
    if (!handle || !alpha || !beta || !w || !dy || !dx || !known_activation(activation)) return IGC_STATUS_BAD_PARAM;
    Matrix mdy, mdx, mz, mr;
    igcStatus st = check_linear(dyDesc, wDesc, dxDesc, true, &mdy, &mdx);
    if (st != IGC_STATUS_SUCCESS) return st;
    LinearArgs a = backward_data_sizes(mdy, *wDesc);
    a.alpha = *static_cast<const float *>(alpha);
    a.beta = *static_cast<const float *>(beta);
    const bool slope = activation != IGC_ACTIVATION_IDENTITY;
    if (slope && (st = check_beside(dxDesc, zDesc, z, &mz)) != IGC_STATUS_SUCCESS) return st;
    if (a.beta != 0.f && (st = check_beside(dxDesc, rDesc, r, &mr)) != IGC_STATUS_SUCCESS) return st;
    if (misaligned(w, wDesc->dtype) || misaligned(dy, dyDesc->dtype) || misaligned(dx, dxDesc->dtype)) return IGC_STATUS_BAD_PARAM;
    a.a = dy;
    a.b = w;
    a.act = activation;
    a.zin = slope ? z : nullptr; a.zs = mz.stride;
    a.r = r; a.rs = mr.stride;
    a.y = dx; a.ys = mdx.stride;
    return run_product(handle, dyDesc->dtype, dxDesc->dtype, a, workSpace, workSpaceSizeInBytes);
}

igcStatus igcGetLinearBackwardFilterWorkspaceSize(igcHandle_t handle, igcTensorDescriptor_t xDesc, igcTensorDescriptor_t dyDesc,
                                                  igcFilterDescriptor_t dwDesc, size_t *sizeInBytes) {
    if (!handle || !sizeInBytes) return IGC_STATUS_BAD_PARAM;
    Matrix x, dy;
    const igcStatus st = check_linear_filter(xDesc, dyDesc, dwDesc, &x, &dy);
    if (st != IGC_STATUS_SUCCESS) return st;
    *sizeInBytes = plan_tiles(handle, xDesc->dtype, dwDesc->dtype, backward_filter_sizes(x, dy, *dwDesc), true, kNoLimit).bytes;
    return IGC_STATUS_SUCCESS;
}

igcStatus igcLinearBackwardFilter(igcHandle_t handle, const void *alpha, igcTensorDescriptor_t xDesc, const void *x, igcTensorDescriptor_t dyDesc,
                                  const void *dy, void *workSpace, size_t workSpaceSizeInBytes, const void *beta, igcFilterDescriptor_t dwDesc,
                                  void *dw, void *dbias) {
    if (!handle || !alpha || !beta || !x || !dy || !dw) return IGC_STATUS_BAD_PARAM;
    Matrix mx, mdy;
    const igcStatus st = check_linear_filter(xDesc, dyDesc, dwDesc, &mx, &mdy);
    if (st != IGC_STATUS_SUCCESS) return st;
    if (misaligned(x, xDesc->dtype) || misaligned(dy, dyDesc->dtype) || misaligned(dw, dwDesc->dtype) || misaligned(dbias, IGC_DATA_FLOAT))
        return IGC_STATUS_BAD_PARAM;
    LinearArgs a = backward_filter_sizes(mx, mdy, *dwDesc);
    a.alpha = *static_cast<const float *>(alpha);
    a.beta = *static_cast<const float *>(beta);
    a.a = dy;
    a.b = x;
    a.act = IGC_ACTIVATION_IDENTITY;
    a.r = dw; a.rs = dwDesc->c;
    a.y = dw; a.ys = dwDesc->c;
    SumsOut sums;
    sums.out = static_cast<float *>(dbias);
    sums.alpha = a.alpha;
    sums.beta = a.beta;
    bool summed = false;
    const igcStatus rc = run_product(handle, xDesc->dtype, dwDesc->dtype, a, workSpace, workSpaceSizeInBytes, sums, &summed);
    if (rc != IGC_STATUS_SUCCESS || !dbias || summed) return rc;
    ColumnArgs c{dy, mdy.stride, (int)mdy.rows, dwDesc->k, a.alpha, a.beta, static_cast<float *>(dbias)};
    const dim3 grid((unsigned)(c.K + 63) / 64u);
    return dyDesc->dtype == IGC_DATA_FLOAT ? launch_kernel(reinterpret_cast<const void *>(&column_sum_kernel<float>), c, grid, 256, handle->stream)
                                           : launch_kernel(reinterpret_cast<const void *>(&column_sum_kernel<bf16_t>), c, grid, 256, handle->stream);
}

}  // extern "C"
