// Layer norm over the feature maps of every position, forward and backward:
//
//   mean_i = sum_c x_ic / C,   s_i = 1 / sqrt(sum_c (x_ic - mean_i)^2 / C + epsilon)
//   y_ic   = alpha * ((x_ic - mean_i) s_i scale_c + shift_c) + beta * y_ic
//
//   with h = (x - mean) s and q = dy * scale:
//   dx_ic    = alpha * s_i (q_ic - sum_c(q_ic) / C - h_ic sum_c(q_ic h_ic) / C) + beta * r_ic
//   dscale_c = alpha * sum_i dy_ic h_ic + paramBeta * dscale_c,   dshift_c = alpha * sum_i dy_ic + paramBeta * dshift_c
//
// The deviations are taken from the finished mean (a difference of a sum of squares and a squared sum would lose the digits of
// rows whose mean is large against their spread).  Sums are held in float, in double for double tensors, in a fixed order.
#include "igconv_rows.h"

namespace igc {
namespace {

template <class W>
struct NormArgs {
    const void *x, *scale, *shift;
    void *y;
    W *mean, *invstd;
    long long xs, ys;   // elements between rows
    int C;
    W alpha, beta, epsilon;
};

template <class W>
struct NormBackwardArgs {
    const void *x, *dy, *r;
    const W *scale, *mean, *invstd;
    void *dx;
    W *dscale, *dshift, *parts;   // parts: [range][2][C], dscale's and dshift's sums of a range of rows
    long long xs, dys, rs, dxs;
    int M, C;
    int ranges, per;              // rows per range
    W alpha, beta, paramBeta;
};

template <class W>
__device__ __forceinline__ W wave_sum(W v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v += __shfl_xor(v, d);
    return v;
}

// sum over a workgroup of 256 threads, given to all; `slots`: four entries that nothing else uses until the next barrier
template <class W>
__device__ __forceinline__ W group_sum(W v, W *slots) {
    v = wave_sum(v);
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    return (slots[0] + slots[1]) + (slots[2] + slots[3]);
}

// ---- any row length: a workgroup per row, the row read once per pass ------------------------------------------------
template <class TX, class TY>
__global__ __launch_bounds__(256) void layer_norm_rows_kernel(const NormArgs<typename Stored<TX>::wide_t> a) {
    typedef typename Stored<TX>::wide_t W;
    __shared__ W slots[8];
    const TX *x = static_cast<const TX *>(a.x) + (long long)blockIdx.x * a.xs;
    TY *y = static_cast<TY *>(a.y) + (long long)blockIdx.x * a.ys;
    W sum = W(0);
    for (int c = threadIdx.x; c < a.C; c += 256) sum += Stored<TX>::widen(x[c]);
    const W mean = group_sum(sum, slots) / W(a.C);
    W squares = W(0);
    for (int c = threadIdx.x; c < a.C; c += 256) {
        const W d = Stored<TX>::widen(x[c]) - mean;
        squares += d * d;
    }
    const W s = W(1) / sqrt(group_sum(squares, slots + 4) / W(a.C) + a.epsilon);
    const W *scale = static_cast<const W *>(a.scale), *shift = static_cast<const W *>(a.shift);
    for (int c = threadIdx.x; c < a.C; c += 256) {
        W v = (Stored<TX>::widen(x[c]) - mean) * s;
        if (scale) v *= scale[c];
        if (shift) v += shift[c];
        v *= a.alpha;
        if (a.beta != W(0)) v += a.beta * Stored<TY>::widen(y[c]);
        y[c] = Stored<TY>::narrow(v);
    }
    if (threadIdx.x == 0) {
        if (a.mean) a.mean[blockIdx.x] = mean;
        if (a.invstd) a.invstd[blockIdx.x] = s;
    }
}

template <class TX, class TY>
__global__ __launch_bounds__(256) void layer_norm_backward_rows_kernel(const NormBackwardArgs<typename Stored<TX>::wide_t> a) {
    typedef typename Stored<TX>::wide_t W;
    __shared__ W slots[8];
    const long long i = blockIdx.x;
    const TX *x = static_cast<const TX *>(a.x) + i * a.xs;
    const TY *dy = static_cast<const TY *>(a.dy) + i * a.dys;
    const W mean = a.mean[i], s = a.invstd[i];
    W sum = W(0), along = W(0);
    for (int c = threadIdx.x; c < a.C; c += 256) {
        const W q = Stored<TY>::widen(dy[c]) * (a.scale ? a.scale[c] : W(1));
        sum += q;
        along += q * ((Stored<TX>::widen(x[c]) - mean) * s);
    }
    sum = group_sum(sum, slots) / W(a.C);
    along = group_sum(along, slots + 4) / W(a.C);
    const TX *r = static_cast<const TX *>(a.r) + i * a.rs;
    TX *dx = static_cast<TX *>(a.dx) + i * a.dxs;
    for (int c = threadIdx.x; c < a.C; c += 256) {
        const W q = Stored<TY>::widen(dy[c]) * (a.scale ? a.scale[c] : W(1)), h = (Stored<TX>::widen(x[c]) - mean) * s;
        W v = a.alpha * (s * (q - sum - h * along));
        if (a.beta != W(0)) v += a.beta * Stored<TX>::widen(r[c]);
        dx[c] = Stored<TX>::narrow(v);
    }
}

// dscale's and dshift's sums over a range of rows: lanes along 64 feature maps, the four wavefronts on every fourth row
template <class TX, class TY>
__global__ __launch_bounds__(256) void layer_norm_params_kernel(const NormBackwardArgs<typename Stored<TX>::wide_t> a) {
    typedef typename Stored<TX>::wide_t W;
    __shared__ W sums[2][4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = (int)blockIdx.x * 64 + lane;
    const int begin = (int)blockIdx.y * a.per, end = min(begin + a.per, a.M);
    W scale = W(0), shift = W(0);
    if (c < a.C)
        for (int i = begin + wave; i < end; i += 4) {
            const W dy = Stored<TY>::widen(static_cast<const TY *>(a.dy)[i * a.dys + c]);
            const W h = (Stored<TX>::widen(static_cast<const TX *>(a.x)[i * a.xs + c]) - a.mean[i]) * a.invstd[i];
            shift += dy;
            scale += dy * h;
        }
    sums[0][wave][lane] = scale;
    sums[1][wave][lane] = shift;
    __syncthreads();
    if (wave < 2 && c < a.C) {
        const W *s = &sums[wave][0][lane];
        a.parts[((size_t)blockIdx.y * 2 + wave) * a.C + c] = (s[0] + s[64]) + (s[128] + s[192]);
    }
}

// adds the ranges' sums in order; without ranges takes the sums over all rows itself
template <class TX, class TY>
__global__ __launch_bounds__(256) void layer_norm_params_sum_kernel(const NormBackwardArgs<typename Stored<TX>::wide_t> a) {
    typedef typename Stored<TX>::wide_t W;
    __shared__ W sums[2][4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = (int)blockIdx.x * 64 + lane;
    W scale = W(0), shift = W(0);
    if (c < a.C) {
        if (a.parts) {
            for (int r = wave; r < a.ranges; r += 4) {
                scale += a.parts[(size_t)r * 2 * a.C + c];
                shift += a.parts[((size_t)r * 2 + 1) * a.C + c];
            }
        } else {
            for (int i = wave; i < a.M; i += 4) {
                const W dy = Stored<TY>::widen(static_cast<const TY *>(a.dy)[i * a.dys + c]);
                const W h = (Stored<TX>::widen(static_cast<const TX *>(a.x)[i * a.xs + c]) - a.mean[i]) * a.invstd[i];
                shift += dy;
                scale += dy * h;
            }
        }
    }
    sums[0][wave][lane] = scale;
    sums[1][wave][lane] = shift;
    __syncthreads();
    W *out = wave == 0 ? a.dscale : a.dshift;
    if (wave < 2 && c < a.C && out) {
        const W *s = &sums[wave][0][lane];
        W v = a.alpha * ((s[0] + s[64]) + (s[128] + s[192]));
        if (a.paramBeta != W(0)) v += a.paramBeta * out[c];
        out[c] = v;
    }
}

// ---- host ------------------------------------------------------------------------------------------------------------
bool norm_types(igcDataType x, igcDataType y) {
    return (x == IGC_DATA_DOUBLE) == (y == IGC_DATA_DOUBLE);
}

bool misaligned(const void *p, igcDataType t) { return (uintptr_t)p % (size_t)elem_size(t) != 0; }

double host_scalar(const void *p, bool f64) { return f64 ? *static_cast<const double *>(p) : (double)*static_cast<const float *>(p); }

// f(type of x, type of y) for the types a call was accepted with
template <class F>
igcStatus by_types(igcDataType x, igcDataType y, F f) {
    if (x == IGC_DATA_DOUBLE) return f(double(), double());
    if (x == IGC_DATA_FLOAT) return y == IGC_DATA_FLOAT ? f(float(), float()) : f(float(), bf16_t());
    return y == IGC_DATA_FLOAT ? f(bf16_t(), float()) : f(bf16_t(), bf16_t());
}

struct NormProblem {
    Matrix x, y, r, dx;
};

igcStatus check_norm(igcTensorDescriptor_t xDesc, igcTensorDescriptor_t yDesc, NormProblem *p) {
    if (!xDesc || !yDesc) return IGC_STATUS_BAD_PARAM;
    if (!xDesc->set || !yDesc->set) return IGC_STATUS_NOT_INITIALIZED;
    if (!same_positions(*xDesc, *yDesc) || xDesc->dim[1] != yDesc->dim[1]) return IGC_STATUS_BAD_PARAM;
    if (!norm_types(xDesc->dtype, yDesc->dtype) || !matrix_of(*xDesc, &p->x) || !matrix_of(*yDesc, &p->y)) return IGC_STATUS_NOT_SUPPORTED;
    return IGC_STATUS_SUCCESS;
}

igcStatus check_norm_backward(igcTensorDescriptor_t xDesc, igcTensorDescriptor_t dyDesc, igcTensorDescriptor_t dxDesc, NormProblem *p) {
    const igcStatus st = check_norm(xDesc, dyDesc, p);
    if (!dxDesc) return IGC_STATUS_BAD_PARAM;
    if (st != IGC_STATUS_SUCCESS) return st;
    if (!dxDesc->set) return IGC_STATUS_NOT_INITIALIZED;
    if (!same_positions(*xDesc, *dxDesc) || xDesc->dim[1] != dxDesc->dim[1] || !non_aliasing(dxDesc->dim, dxDesc->stride)) return IGC_STATUS_BAD_PARAM;
    if (dxDesc->dtype != xDesc->dtype || !matrix_of(*dxDesc, &p->dx)) return IGC_STATUS_NOT_SUPPORTED;
    return IGC_STATUS_SUCCESS;
}

// ranges of rows whose sums are taken side by side
int param_ranges(const igcContext *h, const Matrix &x) {
    const long long groups = (x.cols + 63) / 64;
    const long long most = (x.rows + 31) / 32, wanted = (4ll * h->computeUnits + groups - 1) / groups;
    return (int)std::max(1ll, std::min(most, wanted));
}

}  // namespace
}  // namespace igc

using namespace igc;

extern "C" {

igcStatus igcLayerNormForward(igcHandle_t handle, const void *alpha, igcTensorDescriptor_t xDesc, const void *x, const void *scale,
                              const void *shift, double epsilon, const void *beta, igcTensorDescriptor_t yDesc, void *y, void *mean,
                              void *invStd) {
    if (!handle || !alpha || !beta || !x || !y) return IGC_STATUS_BAD_PARAM;
    NormProblem p;
    const igcStatus st = check_norm(xDesc, yDesc, &p);
    if (st != IGC_STATUS_SUCCESS) return st;
    if (!non_aliasing(yDesc->dim, yDesc->stride) || !(epsilon >= 0.0) || isinf(epsilon)) return IGC_STATUS_BAD_PARAM;
    const bool f64 = xDesc->dtype == IGC_DATA_DOUBLE;
    const igcDataType wide = f64 ? IGC_DATA_DOUBLE : IGC_DATA_FLOAT;
    if (misaligned(x, xDesc->dtype) || misaligned(y, yDesc->dtype) || misaligned(scale, wide) || misaligned(shift, wide) || misaligned(mean, wide) ||
        misaligned(invStd, wide))
        return IGC_STATUS_BAD_PARAM;
    return by_types(xDesc->dtype, yDesc->dtype, [&](auto tx, auto ty) {
        typedef decltype(tx) TX;
        typedef decltype(ty) TY;
        typedef typename Stored<TX>::wide_t W;
        NormArgs<W> a{};
        a.x = x; a.scale = scale; a.shift = shift; a.y = y;
        a.mean = static_cast<W *>(mean); a.invstd = static_cast<W *>(invStd);
        a.xs = p.x.stride; a.ys = p.y.stride; a.C = p.x.cols;
        a.alpha = (W)host_scalar(alpha, f64); a.beta = (W)host_scalar(beta, f64); a.epsilon = (W)epsilon;
        return launch_kernel(reinterpret_cast<const void *>(&layer_norm_rows_kernel<TX, TY>), a, dim3((unsigned)p.x.rows), 256, handle->stream);
    });
}

igcStatus igcGetLayerNormBackwardWorkspaceSize(igcHandle_t handle, igcTensorDescriptor_t xDesc, igcTensorDescriptor_t dyDesc,
                                               igcTensorDescriptor_t dxDesc, size_t *sizeInBytes) {
    if (!handle || !sizeInBytes) return IGC_STATUS_BAD_PARAM;
    NormProblem p;
    const igcStatus st = check_norm_backward(xDesc, dyDesc, dxDesc, &p);
    if (st != IGC_STATUS_SUCCESS) return st;
    const int ranges = param_ranges(handle, p.x);
    *sizeInBytes = ranges > 1 ? (size_t)ranges * 2 * p.x.cols * (xDesc->dtype == IGC_DATA_DOUBLE ? 8 : 4) : 0;
    return IGC_STATUS_SUCCESS;
}

igcStatus igcLayerNormBackward(igcHandle_t handle, const void *alpha, igcTensorDescriptor_t xDesc, const void *x, igcTensorDescriptor_t dyDesc,
                               const void *dy, const void *scale, const void *mean, const void *invStd, void *workSpace,
                               size_t workSpaceSizeInBytes, const void *beta, igcTensorDescriptor_t rDesc, const void *r,
                               igcTensorDescriptor_t dxDesc, void *dx, const void *paramBeta, void *dscale, void *dshift) {
    if (!handle || !alpha || !beta || !paramBeta || !x || !dy || !mean || !invStd || !dx) return IGC_STATUS_BAD_PARAM;
    NormProblem p;
    const igcStatus st = check_norm_backward(xDesc, dyDesc, dxDesc, &p);
    if (st != IGC_STATUS_SUCCESS) return st;
    const bool f64 = xDesc->dtype == IGC_DATA_DOUBLE;
    const igcDataType wide = f64 ? IGC_DATA_DOUBLE : IGC_DATA_FLOAT;
    const double b = host_scalar(beta, f64);
    if (b != 0.0) {
        if (!rDesc || !r) return IGC_STATUS_BAD_PARAM;
        if (!rDesc->set) return IGC_STATUS_NOT_INITIALIZED;
        if (!same_positions(*xDesc, *rDesc) || xDesc->dim[1] != rDesc->dim[1] || misaligned(r, rDesc->dtype)) return IGC_STATUS_BAD_PARAM;
        if (rDesc->dtype != dxDesc->dtype || !matrix_of(*rDesc, &p.r)) return IGC_STATUS_NOT_SUPPORTED;
    }
    if (misaligned(x, xDesc->dtype) || misaligned(dy, dyDesc->dtype) || misaligned(dx, dxDesc->dtype) || misaligned(scale, wide) ||
        misaligned(mean, wide) || misaligned(invStd, wide) || misaligned(dscale, wide) || misaligned(dshift, wide))
        return IGC_STATUS_BAD_PARAM;
    return by_types(xDesc->dtype, dyDesc->dtype, [&](auto tx, auto ty) {
        typedef decltype(tx) TX;
        typedef decltype(ty) TY;
        typedef typename Stored<TX>::wide_t W;
        NormBackwardArgs<W> a{};
        a.x = x; a.dy = dy; a.r = b != 0.0 ? r : nullptr;
        a.scale = static_cast<const W *>(scale); a.mean = static_cast<const W *>(mean); a.invstd = static_cast<const W *>(invStd);
        a.dx = dx;
        a.dscale = static_cast<W *>(dscale); a.dshift = static_cast<W *>(dshift);
        a.xs = p.x.stride; a.dys = p.y.stride; a.rs = p.r.stride; a.dxs = p.dx.stride;
        a.M = (int)p.x.rows; a.C = p.x.cols;
        a.alpha = (W)host_scalar(alpha, f64); a.beta = (W)b; a.paramBeta = (W)host_scalar(paramBeta, f64);
        igcStatus rc = launch_kernel(reinterpret_cast<const void *>(&layer_norm_backward_rows_kernel<TX, TY>), a, dim3((unsigned)a.M), 256, handle->stream);
        if (rc != IGC_STATUS_SUCCESS || (!dscale && !dshift)) return rc;
        const unsigned groups = (unsigned)(a.C + 63) / 64u;
        a.ranges = param_ranges(handle, p.x);
        const size_t need = (size_t)a.ranges * 2 * (size_t)a.C * sizeof(W);
        if (a.ranges > 1 && workSpace && workSpaceSizeInBytes >= need && (uintptr_t)workSpace % sizeof(W) == 0) {
            a.parts = static_cast<W *>(workSpace);
            a.per = (a.M + a.ranges - 1) / a.ranges;
            a.ranges = (a.M + a.per - 1) / a.per;
            rc = launch_kernel(reinterpret_cast<const void *>(&layer_norm_params_kernel<TX, TY>), a, dim3(groups, (unsigned)a.ranges), 256, handle->stream);
            if (rc != IGC_STATUS_SUCCESS) return rc;
        }
        return launch_kernel(reinterpret_cast<const void *>(&layer_norm_params_sum_kernel<TX, TY>), a, dim3(groups), 256, handle->stream);
    });
}

}  // extern "C"
