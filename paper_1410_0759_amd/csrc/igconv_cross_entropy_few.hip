// Sixteen tokens at most: bfloat16 logits for cross entropy straight from registers.  A workgroup computes the tokens by 16 KB vocabulary entries; its eight wavefronts take the
// blocks of 128 features in turns, two blocks requested at once, and add their sums in LDS.  The vocabulary's bytes are all there is to it: 8 x 8192 -> 8000 39.5 us with the
// joining of the statistics (131 MB; as tiles of 128 x 128 77), 8 x 4096 -> 32768 64.6 (66.6).  Beyond 128 entries for each compute unit the tiles, whose loads run further
// ahead, are the faster: 8 x 4096 -> 131072 195 us, this way 224; with more than sixteen tokens, and for float, everywhere (30 x 1024 -> 50000 27 for 43; float 58 for 97).
#include "igconv_cross_entropy.h"
#include "igconv_linear_tiles.hpp"

namespace igc {
namespace {

constexpr int kBlock = 128, kWaves = 8;

__device__ __forceinline__ u32x4 load8_bits(const uint16_t *from, int there) {
    if (there >= 8) return __builtin_bit_cast(u32x4, *reinterpret_cast<const Adjacent<uint16_t, 8> *>(from));
    u32x4 v;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        uint32_t lo = 0, hi = 0;
        if (2 * e < there) lo = from[2 * e];
        if (2 * e + 1 < there) hi = from[2 * e + 1];
        v[e] = lo | hi << 16;
    }
    return v;
}

template <int KB, bool SLOPES>
__global__ __launch_bounds__(64 * kWaves) void cross_few_kernel(const CrossArgs p) {
    constexpr int BATCH = 2, TOKENS = kFewTokens, COLUMNS = 16 * KB;
    __shared__ f32x4 sums[kWaves][KB][64];
    __shared__ float z[TOKENS][COLUMNS + 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l16 = lane & 15, g = lane >> 4;
    const int blocks = (p.K + kBlock - 1) / kBlock;
    const uint16_t *token = static_cast<const uint16_t *>(p.a) + (long long)min(l16, p.M - 1) * p.am + 8 * g;
    for (int tile = blockIdx.x; tile < p.tilesN; tile += gridDim.x) {
        const int n0 = tile * COLUMNS;
        const uint16_t *row[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) row[kb] = static_cast<const uint16_t *>(p.b) + (long long)min(n0 + 16 * kb + l16, p.N - 1) * p.bn + 8 * g;
        f32x4 total[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) total[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int first = wave; first < blocks; first += BATCH * kWaves) {
            u32x4 w[BATCH][4][KB], x[BATCH][4];
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const int s = first + b * kWaves;
                if (s >= blocks) continue;
                const bool whole = (s + 1) * kBlock <= p.K;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int c = s * kBlock + 32 * i, there = whole ? 8 : p.K - c - 8 * g;
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) w[b][i][kb] = load8_bits(row[kb] + c, there);
                    x[b][i] = load8_bits(token + c, there);
                }
            }
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                if (first + b * kWaves >= blocks) continue;
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb)
                        total[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w[b][i][kb]), __builtin_bit_cast(bf16x8, x[b][i]), total[kb], 0, 0, 0);
            }
        }
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
            if (l16 < p.M) sums[wave][kb][lane] = total[kb];
        __syncthreads();
        // the logits, minus infinity right of the matrix
        for (int at = threadIdx.x; at < KB * 64; at += 64 * kWaves) {
            const int block = at >> 6, l = at & 63, m = l & 15, n = 16 * block + 4 * (l >> 4);
            if (m >= p.M) continue;
            f32x4 d = sums[0][block][l];
#pragma unroll
            for (int v = 1; v < kWaves; ++v) d += sums[v][block][l];
#pragma unroll
            for (int e = 0; e < 4; ++e) z[m][n + e] = n0 + n + e < p.N ? d[e] + (p.bias ? p.bias[n0 + n + e] : 0.f) : -INFINITY;
        }
        __syncthreads();
        if constexpr (!SLOPES) {
            // sixteen lanes to a token
            const int m = threadIdx.x >> 4, part = threadIdx.x & 15;
            if (m < min(TOKENS, p.M)) {
                float most = -INFINITY;
#pragma unroll
                for (int i = 0; i < KB; ++i) most = fmaxf(most, z[m][part + 16 * i]);
#pragma unroll
                for (int d = 1; d < 16; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
                const float from = most == -INFINITY ? 0.f : most;
                float sum = 0.f;
#pragma unroll
                for (int i = 0; i < KB; ++i) sum += exp_of(z[m][part + 16 * i] - from);
                sum = lanes_sum<16>(sum);
                if (part == 0) {
                    p.end.parts[(long long)tile * p.M + m] = {most, sum};
                    const int t = p.end.targets[m], at = t >= p.end.first && t - p.end.first < p.N ? t - p.end.first - n0 : -1;
                    if (at >= 0 && at < COLUMNS) p.end.picked[m] = z[m][at];
                }
            }
        } else {
            // a thread two columns of a token
            for (int at = threadIdx.x; at < TOKENS * COLUMNS / 2; at += 64 * kWaves) {
                const int m = at / (COLUMNS / 2), n = at % (COLUMNS / 2) * 2;
                if (m >= p.M || n0 + n >= (p.N + 7) / 8 * 8) continue;
                const int t = p.end.targets[m];
                const bool there = t >= 0 && t < p.end.V;
                const float slope = p.end.alpha * (p.end.dloss ? p.end.dloss[m] : 1.f), log_sum = p.end.logSum[m];
                float d[2], rest[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    float v = exp_of(z[m][n + e] - log_sum);
                    if (there && t - p.end.first == n0 + n + e) v -= 1.f;
                    d[e] = there && n0 + n + e < p.N ? slope * v : 0.f;
                    z[m][n + e] = d[e];
                    rest[e] = rest_of(d[e]);
                }
                uint16_t *to = static_cast<uint16_t *>(p.y) + m * p.ys + n0 + n;
                *reinterpret_cast<uint32_t *>(to) = to_bf16_pair(d[0], d[1]);
                *reinterpret_cast<uint32_t *>(to + p.M * p.ys) = to_bf16_pair(rest[0], rest[1]);
            }
            __syncthreads();
            if (p.end.sums && threadIdx.x < COLUMNS && n0 + (int)threadIdx.x < p.N) {
                float sum = 0.f;
                for (int m = 0; m < p.M; ++m) sum += z[m][threadIdx.x];
                p.end.sums[n0 + threadIdx.x] = sum;
            }
        }
        __syncthreads();
    }
    if constexpr (SLOPES) {
        // x, once for each part, as rows below each other
        const int eights = (p.K + 7) / 8;
        uint16_t *to = static_cast<uint16_t *>(p.z);
        if (to)
            for (long long id = (long long)blockIdx.x * (64 * kWaves) + threadIdx.x; id < (long long)p.M * eights; id += (long long)gridDim.x * (64 * kWaves)) {
                const long long m = id / eights;
                const int c = (int)(id % eights) * 8;
                const u32x4 v = load8_bits(static_cast<const uint16_t *>(p.a) + m * p.am + c, p.K - c);
                *reinterpret_cast<u32x4 *>(to + m * p.zs + c) = v;
                *reinterpret_cast<u32x4 *>(to + (p.M + m) * p.zs + c) = v;
            }
    }
}

}  // namespace

int cross_few_columns(igcHandle_t handle, int N) { return N >= 64 * handle->computeUnits / 2 ? 64 : 16; }

igcStatus cross_few(igcHandle_t handle, CrossKind kind, const LinearArgs &a, const CrossEnd &end) {
    CrossArgs t{};
    static_cast<LinearArgs &>(t) = a;
    t.end = end;
    const int columns = cross_few_columns(handle, a.N);
    t.tilesM = 1;
    t.tilesN = (a.N + columns - 1) / columns;
    const void *const kernels[2][2] = {{reinterpret_cast<const void *>(&cross_few_kernel<1, false>), reinterpret_cast<const void *>(&cross_few_kernel<4, false>)},
                                       {reinterpret_cast<const void *>(&cross_few_kernel<1, true>), reinterpret_cast<const void *>(&cross_few_kernel<4, true>)}};
    return launch_kernel(kernels[kind == kSlopes][columns == 64], t, dim3((unsigned)std::min(t.tilesN, 1 << 20)), 64 * kWaves, handle->stream);
}

}  // namespace igc
