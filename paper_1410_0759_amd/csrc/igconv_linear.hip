// Matrix products over tokens with what follows them in a feed-forward block:
//
//   forward          z = alpha x w^T + bias,  y = f(z) + beta r
//   backward data    dx = alpha (dy w) f'(z) + beta r
//   backward filter  dw = alpha dy^T x + beta dw,  dbias = alpha (column sums of dy) + beta dbias
//
// Products of bfloat16 are accumulated in fp32 by the matrix instructions, in a fixed order.
#include "igconv_linear.h"

namespace igc {
namespace {

// ---- any strides, any alignment, no workspace -------------------------------------------------------------------------
// A workgroup computes 64 x 64 results, its four wavefronts 32 x 32 each, in steps of 32 of the reduction that go element by
// element through LDS, k innermost; the lanes of a load run along whichever index is adjacent in memory.
constexpr int kAnyTile = 64, kAnyStep = 32;

using f32x16 = float __attribute__((ext_vector_type(16)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));

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

template <class T, class TO>
__global__ __launch_bounds__(256) void linear_any_kernel(const LinearArgs p) {
    typedef AnyTile<T> Tile;
    __shared__ __attribute__((aligned(16))) typename Tile::lds_t la[kAnyTile * Tile::ROW], lb[kAnyTile * Tile::ROW];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l32 = lane & 31, half = lane >> 5;
    const int tilesM = (p.M + kAnyTile - 1) / kAnyTile;
    const int m0 = (int)(blockIdx.x % (unsigned)tilesM) * kAnyTile, n0 = (int)(blockIdx.x / (unsigned)tilesM) * kAnyTile;
    const int wm = (wave >> 1) * 32, wn = (wave & 1) * 32;
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
        if (m < p.M && n < p.N) finish_element<TO>(p, m, n, acc[v]);
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

igcStatus run_product(igcHandle_t handle, igcDataType in, igcDataType out, const LinearArgs &a) {
    const long long tiles = (long long)((a.M + kAnyTile - 1) / kAnyTile) * ((a.N + kAnyTile - 1) / kAnyTile);
    if (tiles >= (1ll << 31)) return IGC_STATUS_NOT_SUPPORTED;
    return by_types(in, out, [&](auto ti, auto to) {
        return launch_kernel(reinterpret_cast<const void *>(&linear_any_kernel<decltype(ti), decltype(to)>), a, dim3((unsigned)tiles), 256, handle->stream);
    });
}

}  // namespace
}  // namespace igc

using namespace igc;

extern "C" {

igcStatus igcGetLinearForwardWorkspaceSize(igcHandle_t handle, igcTensorDescriptor_t xDesc, igcFilterDescriptor_t wDesc,
                                           igcTensorDescriptor_t yDesc, size_t *sizeInBytes) {
    if (!handle || !sizeInBytes) return IGC_STATUS_BAD_PARAM;
    Matrix x, y;
    const igcStatus st = check_linear(xDesc, wDesc, yDesc, false, &x, &y);
    if (st != IGC_STATUS_SUCCESS) return st;
    *sizeInBytes = 0;
    return IGC_STATUS_SUCCESS;
}

igcStatus igcLinearForward(igcHandle_t handle, const void *alpha, igcTensorDescriptor_t xDesc, const void *x, igcFilterDescriptor_t wDesc,
                           const void *w, void *workSpace, size_t workSpaceSizeInBytes, const void *bias, int activation, const void *beta,
                           igcTensorDescriptor_t rDesc, const void *r, igcTensorDescriptor_t yDesc, void *z, void *y) {
    if (!handle || !alpha || !beta || !x || !w || !y || !known_activation(activation)) return IGC_STATUS_BAD_PARAM;
    Matrix mx, my, mr;
    igcStatus st = check_linear(xDesc, wDesc, yDesc, false, &mx, &my);
    if (st != IGC_STATUS_SUCCESS) return st;
    LinearArgs a{};
    a.alpha = *static_cast<const float *>(alpha);
    a.beta = *static_cast<const float *>(beta);
    if (a.beta != 0.f && (st = check_beside(yDesc, rDesc, r, &mr)) != IGC_STATUS_SUCCESS) return st;
    if (misaligned(x, xDesc->dtype) || misaligned(w, wDesc->dtype) || misaligned(y, yDesc->dtype) || misaligned(z, yDesc->dtype) ||
        misaligned(bias, IGC_DATA_FLOAT))
        return IGC_STATUS_BAD_PARAM;
    a.a = x; a.am = mx.stride; a.ak = 1;
    a.b = w; a.bn = wDesc->c; a.bk = 1;
    a.M = (int)mx.rows; a.N = wDesc->k; a.K = wDesc->c;
    a.bias = static_cast<const float *>(bias);
    a.act = activation;
    a.z = z; a.zs = my.stride;
    a.r = r; a.rs = mr.stride;
    a.y = y; a.ys = my.stride;
    return run_product(handle, xDesc->dtype, yDesc->dtype, a);
}

igcStatus igcGetLinearBackwardDataWorkspaceSize(igcHandle_t handle, igcFilterDescriptor_t wDesc, igcTensorDescriptor_t dyDesc,
                                                igcTensorDescriptor_t dxDesc, size_t *sizeInBytes) {
    if (!handle || !sizeInBytes) return IGC_STATUS_BAD_PARAM;
    Matrix dy, dx;
    const igcStatus st = check_linear(dyDesc, wDesc, dxDesc, true, &dy, &dx);
    if (st != IGC_STATUS_SUCCESS) return st;
    *sizeInBytes = 0;
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
    LinearArgs a{};
    a.alpha = *static_cast<const float *>(alpha);
    a.beta = *static_cast<const float *>(beta);
    const bool slope = activation != IGC_ACTIVATION_IDENTITY;
    if (slope && (st = check_beside(dxDesc, zDesc, z, &mz)) != IGC_STATUS_SUCCESS) return st;
    if (a.beta != 0.f && (st = check_beside(dxDesc, rDesc, r, &mr)) != IGC_STATUS_SUCCESS) return st;
    if (misaligned(w, wDesc->dtype) || misaligned(dy, dyDesc->dtype) || misaligned(dx, dxDesc->dtype)) return IGC_STATUS_BAD_PARAM;
    a.a = dy; a.am = mdy.stride; a.ak = 1;
    a.b = w; a.bn = 1; a.bk = wDesc->c;
    a.M = (int)mdy.rows; a.N = wDesc->c; a.K = wDesc->k;
    a.act = activation;
    a.zin = slope ? z : nullptr; a.zs = mz.stride;
    a.r = r; a.rs = mr.stride;
    a.y = dx; a.ys = mdx.stride;
    return run_product(handle, dyDesc->dtype, dxDesc->dtype, a);
}

igcStatus igcGetLinearBackwardFilterWorkspaceSize(igcHandle_t handle, igcTensorDescriptor_t xDesc, igcTensorDescriptor_t dyDesc,
                                                  igcFilterDescriptor_t dwDesc, size_t *sizeInBytes) {
    if (!handle || !sizeInBytes) return IGC_STATUS_BAD_PARAM;
    Matrix x, dy;
    const igcStatus st = check_linear_filter(xDesc, dyDesc, dwDesc, &x, &dy);
    if (st != IGC_STATUS_SUCCESS) return st;
    *sizeInBytes = 0;
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
    LinearArgs a{};
    a.alpha = *static_cast<const float *>(alpha);
    a.beta = *static_cast<const float *>(beta);
    a.a = dy; a.am = 1; a.ak = mdy.stride;
    a.b = x; a.bn = 1; a.bk = mx.stride;
    a.M = dwDesc->k; a.N = dwDesc->c; a.K = (int)mx.rows;
    a.act = IGC_ACTIVATION_IDENTITY;
    a.r = dw; a.rs = dwDesc->c;
    a.y = dw; a.ys = dwDesc->c;
    const igcStatus rc = run_product(handle, xDesc->dtype, dwDesc->dtype, a);
    if (rc != IGC_STATUS_SUCCESS || !dbias) return rc;
    ColumnArgs c{dy, mdy.stride, (int)mdy.rows, dwDesc->k, a.alpha, a.beta, static_cast<float *>(dbias)};
    const dim3 grid((unsigned)(c.K + 63) / 64u);
    return dyDesc->dtype == IGC_DATA_FLOAT ? launch_kernel(reinterpret_cast<const void *>(&column_sum_kernel<float>), c, grid, 256, handle->stream)
                                           : launch_kernel(reinterpret_cast<const void *>(&column_sum_kernel<bf16_t>), c, grid, 256, handle->stream);
}

}  // extern "C"
