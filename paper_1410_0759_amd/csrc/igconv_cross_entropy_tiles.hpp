// The ends of linear_tiles_kernel and linear_float_kernel for cross entropy.  A lane holds, of FM x FN blocks of 16 x 16 results, row 16 i + lane % 16, columns
// 16 j + 4 (lane / 16) + 0..3: of each of its rows 4 FN logits, which are a quarter of the wavefront's, so that a row's largest and sum are 4 FN - 1 steps within the
// lane and two between lanes.  Nothing of this has matrix instructions beside it; 8192 x 4096 -> 131072 is 6270 us that way, against 7633 with float logits in memory.
#ifndef IGCONV_CROSS_ENTROPY_TILES_HPP_
#define IGCONV_CROSS_ENTROPY_TILES_HPP_

#include "igconv_cross_entropy.h"
#include "igconv_linear_float.hpp"

namespace igc {

// z = accumulated + bias, minus infinity right of the matrix
template <int FM, int FN>
__device__ __forceinline__ void finish_logits(const CrossArgs &p, int n0, int lane, f32x4 (&acc)[FM][FN]) {
    const int g = lane >> 4;
#pragma unroll
    for (int j = 0; j < FN; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int n = n0 + 16 * j + 4 * g + e;
            const float b = p.bias && n < p.N ? p.bias[n] : 0.f;
#pragma unroll
            for (int i = 0; i < FM; ++i) acc[i][j][e] = n < p.N ? acc[i][j][e] + b : -INFINITY;
        }
}

// four neighbours of a row of bfloat16 numbers (zeros behind its N elements)
__device__ __forceinline__ f32x4 four_of(const uint16_t *row, int n, int N) {
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    if (n + 4 <= N) {
        const Adjacent<uint16_t, 4> q = *reinterpret_cast<const Adjacent<uint16_t, 4> *>(row + n);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = bf16_bits_to_float(q.v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < N) v[e] = bf16_bits_to_float(row[n + e]);
    }
    return v;
}

template <class Cfg>
struct TileEnd<Cfg, RowStatistics, CrossArgs> {
    template <int FM, int FN>
    static __device__ __forceinline__ void run(const CrossArgs &p, uint8_t *lds, int lane, int wave, int, int tm, int tn, int m0, int n0, f32x4 (&acc)[FM][FN]) {
        RowPart *share = reinterpret_cast<RowPart *>(lds);     // [row of the tile][wavefront across]
        static_assert(Cfg::BM * Cfg::WAVES_N * sizeof(RowPart) <= Cfg::LDS_BYTES, "");
        const int l16 = lane & 15, g = lane >> 4, row0 = m0 - tm * Cfg::BM, across = wave % Cfg::WAVES_N;
        finish_logits<FM, FN>(p, n0, lane, acc);
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            float most = acc[i][0][0];
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) most = fmaxf(most, acc[i][j][e]);
            most = fmaxf(most, __shfl_xor(most, 16));
            most = fmaxf(most, __shfl_xor(most, 32));
            // (nothing but minus infinities: no differences of them, and what is undefined among them stays so)
            const float from = most == -INFINITY ? 0.f : most;
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) sum += exp_of(acc[i][j][e] - from);
            sum += __shfl_xor(sum, 16);
            sum += __shfl_xor(sum, 32);
            if (g == 0) share[(row0 + 16 * i + l16) * Cfg::WAVES_N + across] = {most, sum};
            const int m = m0 + 16 * i + l16;
            if (m < p.M) {
                const int t = p.end.targets[m], at = t >= p.end.first && t - p.end.first < p.N ? t - p.end.first - n0 - 4 * g : -1;
#pragma unroll
                for (int j = 0; j < FN; ++j)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (at == 16 * j + e) p.end.picked[m] = acc[i][j][e];
            }
        }
        __syncthreads();
        for (int r = threadIdx.x; r < Cfg::BM; r += Cfg::THREADS) {
            const int m = tm * Cfg::BM + r;
            if (m >= p.M) continue;
            RowPart all = share[r * Cfg::WAVES_N];
#pragma unroll
            for (int w = 1; w < Cfg::WAVES_N; ++w) {
                const RowPart q = share[r * Cfg::WAVES_N + w];
                const float most = fmaxf(all.most, q.most);
                all = most == -INFINITY ? RowPart{most, all.sum + q.sum} : RowPart{most, all.sum * exp_of(all.most - most) + q.sum * exp_of(q.most - most)};
            }
            p.end.parts[(long long)tn * p.M + m] = all;
        }
    }
};

template <class Cfg, class TZ>
struct TileEnd<Cfg, Slopes<TZ>, CrossArgs> {
    template <int FM, int FN>
    static __device__ __forceinline__ void run(const CrossArgs &p, uint8_t *lds, int lane, int wave, int split, int tm, int tn, int m0, int n0, f32x4 (&acc)[FM][FN]) {
        const int l16 = lane & 15, g = lane >> 4;
        finish_logits<FM, FN>(p, n0, lane, acc);
        f32x4 sums[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) sums[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            const int m = m0 + 16 * i + l16, row = m < p.M ? m : p.M - 1, t = p.end.targets[row];
            const bool there = m < p.M && t >= 0 && t < p.end.V;
            const int at = there ? t - p.end.first - n0 - 4 * g : -1;
            const float slope = p.end.alpha * (p.end.dloss ? p.end.dloss[row] : 1.f), log_sum = p.end.logSum[row];
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float v = sizeof(TZ) == 4 ? expf(acc[i][j][e] - log_sum) : exp_of(acc[i][j][e] - log_sum);
                    if (at == 16 * j + e) v -= 1.f;
                    v = there && n0 + 16 * j + 4 * g + e < p.N ? slope * v : 0.f;
                    if (sizeof(TZ) == 2 && p.end.rests && at == 16 * j + e && n0 + 16 * j + 4 * g + e < p.N) p.end.rests[m] = rest_of(v);
                    acc[i][j][e] = v;
                    sums[j][e] += v;
                }
        }
        if (p.end.sums) {
            const long long block = (long long)tm * Cfg::WAVES_M + wave / Cfg::WAVES_N;
#pragma unroll
            for (int j = 0; j < FN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float v = lanes_sum<16>(sums[j][e]);
                    const int n = n0 + 16 * j + 4 * g + e;
                    if (l16 == 0 && n < p.N) p.end.sums[block * p.end.sumStride + n] = v;
                }
        }
        // (stored as an ordinary product's results are, up to the next eighth column)
        TileArgs q = p;
        q.alpha = 1.f;
        q.beta = 0.f;
        q.bias = nullptr;
        q.z = nullptr;
        q.zin = nullptr;
        q.act = IGC_ACTIVATION_IDENTITY;
        q.splits = 1;
        q.N = (p.N + 7) / 8 * 8;
        uint8_t *share = lds + wave * (Cfg::LDS_BYTES / Cfg::WAVES);
        write_results<FM, FN, Cfg::LDS_BYTES / Cfg::WAVES, TZ>(q, share, lane, split, m0, n0, acc);
        if constexpr (sizeof(TZ) == 2) {
            if (p.end.twoParts) {
#pragma unroll
                for (int i = 0; i < FM; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j][e] = rest_of(acc[i][j][e]);
                q.y = static_cast<TZ *>(q.y) + q.M * q.ys;
                write_results<FM, FN, Cfg::LDS_BYTES / Cfg::WAVES, TZ>(q, share, lane, split, m0, n0, acc);
            }
        }
    }
};

template <class Cfg, class TO>
struct TileEnd<Cfg, WithRows<TO>, AddendArgs> {
    template <int FM, int FN>
    static __device__ __forceinline__ void run(const AddendArgs &p, uint8_t *lds, int lane, int wave, int split, int, int, int m0, int n0, f32x4 (&acc)[FM][FN]) {
        const int l16 = lane & 15, g = lane >> 4;
        if (split == 0) {
            uint32_t at[FM];
            float factor[FM];
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                const int m = m0 + 16 * i + l16;
                at[i] = m < p.M ? (uint32_t)p.add.rowOf[m] - (uint32_t)p.add.first : 0xFFFFFFFFu;
                factor[i] = 1.f;
                if (m < p.M && p.add.factor) factor[i] = p.add.factor[m];
            }
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                if (at[i] >= (uint32_t)p.add.count) continue;
                const uint16_t *from = p.add.from + (long long)at[i] * p.add.stride;
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    const f32x4 row = four_of(from, n0 + 16 * j + 4 * g, p.N);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[i][j][e] += factor[i] * row[e];
                }
            }
        }
        write_results<FM, FN, Cfg::LDS_BYTES / Cfg::WAVES, TO>(p, lds + wave * (Cfg::LDS_BYTES / Cfg::WAVES), lane, split, m0, n0, acc);
    }
};

}  // namespace igc
#endif
