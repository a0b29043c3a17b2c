// Filters held in four bits, and products with them:
//
//   y = f(alpha x W^T + bias) + beta r,   W[k][c] = scale[c / group][k] q[k][c],  q of 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives (e2m1)
//
// The q are bfloat16 numbers, and one instruction makes two of them: the products x q are exact in the matrix instructions, and a group's sum is
// multiplied by its scale in fp32.  A scaled weight, which has up to eleven bits, is never rounded.  Float x goes in as three bfloat16 parts
// of eight bits, whose products are exact too.
//
// Layout.  A row of W is cut into blocks of 128 features in 64 bytes; word 4 g + i of a block holds features 32 i + 8 g to + 7, the first in the lowest bits.
// So the 16 bytes that lane group g of a wavefront (16 lanes each) loads are its share of four matrix instructions of 32 features each, and every instruction's features
// lie in one group of any size.  Scales are kept with the rows next to each other: a lane's four results have theirs in 8 bytes.
#include "igconv_linear4.h"

namespace igc {
namespace {

constexpr int kBlock = kCodeBlock, kBlockBytes = kCodeBlockBytes;

// ---- into four bits and back --------------------------------------------------------------------------------------------
struct StoreArgs {
    const void *w;
    void *out;            // (back)
    uint8_t *codes;
    uint16_t *scales;
    int K, C, group;
    long long tiles;
};

// A workgroup takes 64 rows of a block: a lane one word of it, sixteen lanes a row, so that a group's largest is found among 4, 8 or 16 lanes
// and 64 rows' scales of a group go out next to each other.  The scale is the smallest bfloat16 number not below a sixth of the largest.  (16384 x 4096 bfloat16:
// 46 to 50 us for 171 MB; with a sixth in double precision 55 to 63, with a comparison for each border between codes 77.)
template <class T>
__global__ __launch_bounds__(256) void to_four_bits_kernel(const StoreArgs p) {
    const int lane = threadIdx.x & 63, word = lane & 15;
    const int blocks = (p.C + kBlock - 1) / kBlock;
    // (lane j of the sixteen: features 8 j to 8 j + 7, which word 4 (j % 4) + j / 4 holds)
    const int at = 4 * (word & 3) + (word >> 2);
    for (long long tile = blockIdx.x; tile < p.tiles; tile += gridDim.x) {
        const int block = (int)(tile % blocks), c = block * kBlock + word * 8;
        const long long k0 = tile / blocks * 64 + (threadIdx.x >> 4);
        float w[4][8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const long long k = k0 + 16 * i;
#pragma unroll
            for (int e = 0; e < 8; ++e) w[i][e] = 0.f;
            if (k >= p.K) continue;
            const T *from = static_cast<const T *>(p.w) + k * p.C + c;
            if (c + 8 <= p.C) {
                const Adjacent<T, 8> q = *reinterpret_cast<const Adjacent<T, 8> *>(from);
#pragma unroll
                for (int e = 0; e < 8; ++e) w[i][e] = Stored<T>::widen(q.v[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (c + e < p.C) w[i][e] = Stored<T>::widen(from[e]);
            }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const long long k = k0 + 16 * i;
            uint32_t most = 0;      // (magnitudes as whole numbers: what is infinite or undefined lies above all others)
#pragma unroll
            for (int e = 0; e < 8; ++e) most = max(most, __builtin_bit_cast(uint32_t, w[i][e]) & 0x7FFFFFFFu);
            for (int d = 1; d < p.group / 8; d *= 2) most = max(most, (uint32_t)__shfl_xor((int)most, d));
            uint32_t scale = 0x7FC00000u;
            if (most < 0x7F800000u) {
                // (six times a bfloat16 number is exact; a sixth is off by a last digit, so that at most two steps are missing)
                const float largest = __builtin_bit_cast(float, most);
                scale = __builtin_bit_cast(uint32_t, largest * (1.f / 6.f)) & 0xFFFF0000u;
#pragma unroll
                for (int n = 0; n < 2; ++n)
                    if (6.f * __builtin_bit_cast(float, scale) < largest) scale += 0x10000u;
            }
            // w / scale, rounded once: the inverse's product and its remainder's, which is exact.  It is a border between codes only where w is one times the scale (borders
            // have three bits, scales eight: no other w of 24 is within half a step of that).  Below 2^-100, where inverses overflow, both are taken 2^64 times.
            uint32_t codes = 0;
            if (scale != 0) {
                const float s = __builtin_bit_cast(float, scale), up = s < 0x1p-100f ? 0x1p64f : 1.f, su = s * up, inverse = 1.f / su;
                float q[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float v = w[i][e] * up, near = v * inverse;
                    q[e] = __builtin_fmaf(__builtin_fmaf(-near, su, v), inverse, near);
                }
                codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, q[0], q[1], 1.f, 0);
                codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, q[2], q[3], 1.f, 1);
                codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, q[4], q[5], 1.f, 2);
                codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, q[6], q[7], 1.f, 3);
                // (no negative zeros)
                const uint32_t size = codes & 0x77777777u, some = (size | size >> 1 | size >> 2) & 0x11111111u;
                codes = size | (codes & some << 3);
            }
            if (k >= p.K) continue;
            *reinterpret_cast<uint32_t *>(p.codes + k * code_row(p.C) + block * kBlockBytes + at * 4) = codes;
            if (word % (p.group / 8) == 0 && c < p.C) p.scales[(long long)(c / p.group) * p.K + k] = (uint16_t)(scale >> 16);
        }
    }
}

// A workgroup takes 64 rows of a block: a lane four features, so that the lanes of a store write next to each other (16384 x 4096 into float: 51 us for 306 MB; with
// stores that stay in the caches 72, with eight features to a lane, whose stores of 16 bytes lie 32 apart, 92).
template <class T>
__global__ __launch_bounds__(256) void from_four_bits_kernel(const StoreArgs p) {
    const int four = threadIdx.x & 31;
    // (features 4 j to 4 j + 3 of a block: half of word 4 (j / 2 % 4) + j / 8)
    const int at = (4 * ((four >> 1) & 3) + (four >> 3)) * 4 + (four & 1) * 2;
    const int blocks = (p.C + kBlock - 1) / kBlock;
    for (long long tile = blockIdx.x; tile < p.tiles; tile += gridDim.x) {
        const int block = (int)(tile % blocks), c = block * kBlock + four * 4;
        const long long k0 = tile / blocks * 64 + (threadIdx.x >> 5);
        if (c >= p.C) continue;
        uint32_t codes[8];
        float scale[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const long long k = k0 + 8 * i < p.K ? k0 + 8 * i : p.K - 1;
            codes[i] = *reinterpret_cast<const uint16_t *>(p.codes + k * code_row(p.C) + block * kBlockBytes + at);
            scale[i] = bf16_bits_to_float(p.scales[(long long)(c / p.group) * p.K + k]);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const long long k = k0 + 8 * i;
            if (k >= p.K) continue;
            const bf16x8 q = widen8(codes[i]);
            Adjacent<T, 4> v;
#pragma unroll
            for (int e = 0; e < 4; ++e) v.v[e] = Stored<T>::narrow((float)q[e] * scale[i]);
            T *to = static_cast<T *>(p.out) + k * p.C + c;
            if (c + 4 <= p.C) {
                typedef uint32_t Words __attribute__((ext_vector_type(sizeof(T)), aligned(sizeof(T))));
                __builtin_nontemporal_store(__builtin_bit_cast(Words, v), reinterpret_cast<Words *>(to));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (c + e < p.C) to[e] = v.v[e];
            }
        }
    }
}

// ---- products -----------------------------------------------------------------------------------------------------------
// A lane's eight features of a token, in registers and as bfloat16 parts.
template <class T> struct Features;
template <> struct Features<bf16_t> {
    static constexpr int PARTS = 1;
    u32x4 v;
    __device__ __forceinline__ void load(const bf16_t *from, long long = 0) { v = __builtin_bit_cast(u32x4, *reinterpret_cast<const Adjacent<bf16_t, 8> *>(from)); }
    __device__ __forceinline__ void load_some(const bf16_t *from, int there, long long = 0) {
        if (there >= 8) return load(from);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t lo = 0, hi = 0;
            if (2 * e < there) lo = from[2 * e].bits;
            if (2 * e + 1 < there) hi = from[2 * e + 1].bits;
            v[e] = lo | hi << 16;
        }
    }
    __device__ __forceinline__ void split(bf16x8 (&p)[1]) const { p[0] = __builtin_bit_cast(bf16x8, v); }
};
template <> struct Features<float> {
    static constexpr int PARTS = 3;
    f32x4 v[2];
    __device__ __forceinline__ void load(const float *from, long long = 0) {
        const Adjacent<float, 8> q = *reinterpret_cast<const Adjacent<float, 8> *>(from);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e / 4][e % 4] = q.v[e];
    }
    __device__ __forceinline__ void load_some(const float *from, int there, long long = 0) {
        if (there >= 8) return load(from);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e / 4][e % 4] = 0.f;
            if (e < there) v[e / 4][e % 4] = from[e];
        }
    }
    // by truncation: 24 bits are three times eight.  (An infinity has no rest; an undefined number must not become one.)
    __device__ __forceinline__ void split(bf16x8 (&p)[3]) const {
        u32x4 h, m, l;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            uint32_t hb[2], mb[2], lb[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float x = v[(2 * e + i) / 4][(2 * e + i) % 4];
                const uint32_t all = __builtin_bit_cast(uint32_t, x);
                const bool finite = (all & 0x7F800000u) != 0x7F800000u;
                hb[i] = (!finite && (all & 0x007FFFFFu)) ? 0x7FC00000u : all & 0xFFFF0000u;
                const float r = finite ? x - __builtin_bit_cast(float, hb[i]) : 0.f;
                mb[i] = __builtin_bit_cast(uint32_t, r) & 0xFFFF0000u;
                lb[i] = __builtin_bit_cast(uint32_t, r - __builtin_bit_cast(float, mb[i]));
            }
            h[e] = __builtin_amdgcn_perm(hb[1], hb[0], 0x07060302u);
            m[e] = __builtin_amdgcn_perm(mb[1], mb[0], 0x07060302u);
            l[e] = __builtin_amdgcn_perm(lb[1], lb[0], 0x07060302u);
        }
        p[0] = __builtin_bit_cast(bf16x8, h);
        p[1] = __builtin_bit_cast(bf16x8, m);
        p[2] = __builtin_bit_cast(bf16x8, l);
    }
};

// float features laid out in three parts (lay_out_kernel), `parts` elements apart; rows end with a whole eight
struct Laid {
    uint16_t bits;
};
template <> struct Features<Laid> {
    static constexpr int PARTS = 3;
    u32x4 v[3];
    __device__ __forceinline__ void load(const Laid *from, long long parts) {
#pragma unroll
        for (int n = 0; n < 3; ++n) v[n] = *reinterpret_cast<const u32x4 *>(from + n * parts);
    }
    __device__ __forceinline__ void load_some(const Laid *from, int there, long long parts) {
#pragma unroll
        for (int n = 0; n < 3; ++n) {
            v[n] = u32x4{0u, 0u, 0u, 0u};
            if (there > 0) v[n] = *reinterpret_cast<const u32x4 *>(from + n * parts);
        }
    }
    __device__ __forceinline__ void split(bf16x8 (&p)[3]) const {
#pragma unroll
        for (int n = 0; n < 3; ++n) p[n] = __builtin_bit_cast(bf16x8, v[n]);
    }
};

// A workgroup computes 16 TB tokens x 16 KB rows of W; its wavefronts take the blocks of 128 features in turns and add their sums at the end, so that a few rows of W keep a
// compute unit's loads under way.  The last part of all of them: the sums, from LDS, with the epilogue.
template <int KB, int TB, int WAVES, class TO>
__device__ __forceinline__ void finish_sums(const Linear4Args &p, f32x4 (&sums)[WAVES][KB * TB][64], const f32x4 (&total)[KB][TB], int lane, int wave, long long m0, int n0,
                                            int split) {
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int tb = 0; tb < TB; ++tb)
            if (m0 + 16 * tb + (lane & 15) < p.M) sums[wave][kb * TB + tb][lane] = total[kb][tb];
    __syncthreads();
    for (int at = threadIdx.x; at < KB * TB * 64; at += 64 * WAVES) {
        const int block = at >> 6, l = at & 63;
        const long long m = m0 + 16 * (block % TB) + (l & 15);
        const int n = n0 + 16 * (block / TB) + 4 * (l >> 4);
        if (m >= p.M) continue;
        f32x4 d = sums[0][block][l];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) d += sums[w][block][l];
        if (p.splits > 1) {
            if (n < p.N) *reinterpret_cast<f32x4 *>(p.parts + ((long long)split * p.M + m) * p.partsRow + n) = d;
            continue;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < p.N) finish_element<TO>(p, (int)m, n + e, d[e]);
    }
    __syncthreads();
}

// Sixteen tokens: everything that a wavefront needs for BATCH blocks is requested at once - at 4096 features that is all it needs - because each trip to memory that waits for
// another shows (1 x 4096 -> 16384, groups of 128: 14.3 us block after block, 15.7 with the next block under way, 11.4 to 12.2 this way).
template <int KB, int GROUP, class TX, class TO>
__global__ __launch_bounds__(512) void linear4_few_kernel(const Linear4Args p) {
    constexpr int WAVES = 8, N = Features<TX>::PARTS, SCALES = kBlock / GROUP, IN_GROUP = GROUP / 32;
    constexpr int BATCH = GROUP == 32 || N == 3 ? 2 : 4;     // (registers)
    __shared__ f32x4 sums[WAVES][KB][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l16 = lane & 15, g = lane >> 4;
    const int blocks = (p.K + kBlock - 1) / kBlock, groups = (p.K + GROUP - 1) / GROUP;
    const long long row_bytes = code_row(p.K);
    for (long long unit = blockIdx.x; unit < (long long)p.tilesM * p.tilesN * p.splits; unit += gridDim.x) {
        const long long tile = unit / p.splits;
        const int split = (int)(unit % p.splits), begin = split * p.stepsPerSplit, end = min(blocks, begin + p.stepsPerSplit);
        const int n0 = (int)(tile % p.tilesN) * (16 * KB);
        const long long m0 = tile / p.tilesN * 16;
        const uint8_t *row[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) row[kb] = p.codes + (long long)min(n0 + 16 * kb + l16, p.N - 1) * row_bytes + g * 16;
        const TX *token = static_cast<const TX *>(p.a) + min(m0 + l16, (long long)p.M - 1) * p.am + 8 * g;
        f32x4 total[KB][1];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) total[kb][0] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int first = begin + wave; first < end; first += BATCH * WAVES) {
            u32x4 codes[BATCH][KB];
            u32x2 scales[BATCH][SCALES][KB];
            Features<TX> x[BATCH][4];
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                const int s = first + b * WAVES;
                if (s >= end) continue;
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) codes[b][kb] = *reinterpret_cast<const u32x4 *>(row[kb] + (long long)s * kBlockBytes);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if ((s + 1) * kBlock <= p.K) x[b][i].load(token + s * kBlock + 32 * i);
                    else x[b][i].load_some(token + s * kBlock + 32 * i, p.K - s * kBlock - 8 * g - 32 * i);
                }
#pragma unroll
                for (int q = 0; q < SCALES; ++q)      // (behind the row: zeros times the last group's)
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) scales[b][q][kb] = load_scales(p.scales + (long long)min(s * SCALES + q, groups - 1) * p.N, n0 + 16 * kb + 4 * g, p.N);
            }
#pragma unroll
            for (int b = 0; b < BATCH; ++b) {
                if (first + b * WAVES >= end) continue;
#pragma unroll
                for (int q = 0; q < SCALES; ++q) {
                    f32x4 sum[KB];
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) sum[kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int i = 0; i < IN_GROUP; ++i) {
                        bf16x8 parts[N];
                        x[b][q * IN_GROUP + i].split(parts);
#pragma unroll
                        for (int kb = 0; kb < KB; ++kb) {
                            const bf16x8 w = widen8(codes[b][kb][q * IN_GROUP + i]);
#pragma unroll
                            for (int n = 0; n < N; ++n) sum[kb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, parts[n], sum[kb], 0, 0, 0);
                        }
                    }
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) {
                        const f32x4 scale = widen_scales(scales[b][q][kb]);
#pragma unroll
                        for (int e = 0; e < 4; ++e) total[kb][0][e] += scale[e] * sum[kb][e];
                    }
                }
            }
        }
        finish_sums<KB, 1, WAVES, TO>(p, sums, total, lane, wave, m0, n0, split);
    }
}

// More tokens, TB pieces of sixteen: a block's codes and scales are requested while the block before is multiplied.  Sums are multiplied by their scales every 32 features,
// whatever the group: that needs no room for sums under way.
template <int KB, int TB, class TX, class TO>
__global__ __launch_bounds__(512) void linear4_pieces_kernel(const Linear4Args p) {
    constexpr int WAVES = 8, N = Features<TX>::PARTS;
    __shared__ f32x4 sums[WAVES][KB * TB][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), l16 = lane & 15, g = lane >> 4;
    const int blocks = (p.K + kBlock - 1) / kBlock, groups = (p.K + p.group4 - 1) / p.group4, shift = p.group4 == 32 ? 0 : (p.group4 == 64 ? 1 : 2);
    const long long row_bytes = code_row(p.K);
    for (long long unit = blockIdx.x; unit < (long long)p.tilesM * p.tilesN * p.splits; unit += gridDim.x) {
        const long long tile = unit / p.splits;
        const int split = (int)(unit % p.splits), begin = split * p.stepsPerSplit, end = min(blocks, begin + p.stepsPerSplit);
        const int n0 = (int)(tile % p.tilesN) * (16 * KB);
        const long long m0 = tile / p.tilesN * (16 * TB);
        const uint8_t *row[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) row[kb] = p.codes + (long long)min(n0 + 16 * kb + l16, p.N - 1) * row_bytes + g * 16;
        const TX *token[TB];
#pragma unroll
        for (int tb = 0; tb < TB; ++tb) {
            const long long m = min(m0 + 16 * tb + l16, (long long)p.M - 1);
            token[tb] = static_cast<const TX *>(p.a) + (sizeof(TX) == 2 && N == 3 ? m / kPartsTokens * (3 * kPartsTokens) + m % kPartsTokens : m) * p.am + 8 * g;
        }
        f32x4 total[KB][TB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int tb = 0; tb < TB; ++tb) total[kb][tb] = f32x4{0.f, 0.f, 0.f, 0.f};
        u32x4 codes[KB], next_codes[KB];
        u32x2 scales[4][KB], next_scales[4][KB];
        auto load = [&](int s) __attribute__((always_inline)) {
            if (s >= end) return;
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) next_codes[kb] = *reinterpret_cast<const u32x4 *>(row[kb] + (long long)s * kBlockBytes);
#pragma unroll
            for (int i = 0; i < 4; ++i)      // (behind the row: zeros times the last group's)
#pragma unroll
                for (int kb = 0; kb < KB; ++kb)
                    next_scales[i][kb] = load_scales(p.scales + (long long)min((4 * s + i) >> shift, groups - 1) * p.N, n0 + 16 * kb + 4 * g, p.N);
        };
        load(begin + wave);
        for (int s = begin + wave; s < end; s += WAVES) {
#pragma unroll
            for (int kb = 0; kb < KB; ++kb) codes[kb] = next_codes[kb];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) scales[i][kb] = next_scales[i][kb];
            load(s + WAVES);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                bf16x8 parts[TB][N];
#pragma unroll
                for (int tb = 0; tb < TB; ++tb) {
                    Features<TX> here;
                    const TX *from = token[tb] + s * kBlock + 32 * i;
                    if ((s + 1) * kBlock <= p.K) here.load(from, kPartsTokens * p.am);
                    else here.load_some(from, p.K - s * kBlock - 8 * g - 32 * i, kPartsTokens * p.am);
                    here.split(parts[tb]);
                }
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) {
                    const bf16x8 q = widen8(codes[kb][i]);
                    const f32x4 scale = widen_scales(scales[i][kb]);
#pragma unroll
                    for (int tb = 0; tb < TB; ++tb) {
                        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                        for (int n = 0; n < N; ++n) sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q, parts[tb][n], sum, 0, 0, 0);
#pragma unroll
                        for (int e = 0; e < 4; ++e) total[kb][tb][e] += scale[e] * sum[e];
                    }
                }
            }
        }
        finish_sums<KB, TB, WAVES, TO>(p, sums, total, lane, wave, m0, n0, split);
    }
}

// The sum of the parts of a cut reduction, with the epilogue: a thread four neighbours of a row.
template <class TO>
__global__ __launch_bounds__(256) void linear4_finish_kernel(const Linear4Args p) {
    const long long groups = p.partsRow / 4, tasks = p.M * groups;
    for (long long id = (long long)blockIdx.x * 256 + threadIdx.x; id < tasks; id += (long long)gridDim.x * 256) {
        const int m = (int)(id / groups), n = (int)(id % groups) * 4;
        f32x4 d = *reinterpret_cast<const f32x4 *>(p.parts + m * p.partsRow + n);
#pragma unroll 4
        for (int s = 1; s < p.splits; ++s) d += *reinterpret_cast<const f32x4 *>(p.parts + ((long long)s * p.M + m) * p.partsRow + n);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < p.N) finish_element<TO>(p, m, n + e, d[e]);
    }
}

// ---- x and scales for the tiles ------------------------------------------------------------------------------------------------
struct Lay4Args {
    const void *x;
    uint16_t *to;
    long long stride;
    int M, C, toRow;
    unsigned groupsX;           // workgroups for x; the others lay out scales
    const uint16_t *scales;
    uint16_t *toScales;
    int N;
    long long scaleGroups, scaleRow;
};
// x: bfloat16 in rows on 16-byte boundaries, zeros up to the next eighth feature; float in three parts, kPartsTokens rows of each in turn, and zeros for the last rows.
// Scales: in rows of an even length.
template <class T>
__global__ __launch_bounds__(256) void lay_out_kernel(const Lay4Args p) {
    constexpr int N = Features<T>::PARTS;
    if (blockIdx.x >= p.groupsX) {
        for (long long id = (long long)(blockIdx.x - p.groupsX) * 256 + threadIdx.x; id < p.scaleGroups * p.scaleRow; id += (long long)(gridDim.x - p.groupsX) * 256) {
            const long long group = id / p.scaleRow, n = id % p.scaleRow;
            p.toScales[id] = n < p.N ? p.scales[group * p.N + n] : (uint16_t)0;
        }
        return;
    }
    const int groups = p.toRow / 8;
    const long long rows = N == 1 ? p.M : ((long long)p.M + kPartsTokens - 1) / kPartsTokens * kPartsTokens;
    for (long long id = (long long)blockIdx.x * 256 + threadIdx.x; id < rows * groups; id += (long long)p.groupsX * 256) {
        const long long m = id / groups;
        const int c = (int)(id % groups) * 8;
        Features<T> v;
        const T *from = static_cast<const T *>(p.x) + m * p.stride + c;
        if (m < p.M && c + 8 <= p.C) v.load(from);
        else v.load_some(from, m < p.M ? p.C - c : 0);
        bf16x8 parts[N];
        v.split(parts);
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const long long row = N == 1 ? m : (m / kPartsTokens * N + n) * kPartsTokens + m % kPartsTokens;
            *reinterpret_cast<bf16x8 *>(p.to + row * p.toRow + c) = parts[n];
        }
    }
}

// ---- host ---------------------------------------------------------------------------------------------------------------
bool off(const void *p, size_t to) { return (uintptr_t)p % to != 0; }

igcStatus check_filter(igcFilterDescriptor_t w, int group) {
    if (!w) return IGC_STATUS_BAD_PARAM;
    if (!w->set) return IGC_STATUS_NOT_INITIALIZED;
    if (w->r != 1 || w->s != 1) return IGC_STATUS_BAD_PARAM;
    if ((w->dtype != IGC_DATA_FLOAT && w->dtype != IGC_DATA_BFLOAT16) || (group != 32 && group != 64 && group != 128) || w->k > kMostColumns || w->c > kMostColumns)
        return IGC_STATUS_NOT_SUPPORTED;
    return IGC_STATUS_SUCCESS;
}

igcStatus check_product(igcTensorDescriptor_t x, igcFilterDescriptor_t w, int group, igcTensorDescriptor_t y, Matrix *mx, Matrix *my) {
    if (!x || !w || !y) return IGC_STATUS_BAD_PARAM;
    if (!x->set || !y->set) return IGC_STATUS_NOT_INITIALIZED;
    const igcStatus st = check_filter(w, group);
    if (st != IGC_STATUS_SUCCESS) return st;
    if (x->dim[1] != w->c || y->dim[1] != w->k || !same_positions(*x, *y) || !non_aliasing(y->dim, y->stride)) return IGC_STATUS_BAD_PARAM;
    if ((x->dtype != IGC_DATA_BFLOAT16 && x->dtype != IGC_DATA_FLOAT) || (y->dtype != IGC_DATA_FLOAT && !(x->dtype == IGC_DATA_BFLOAT16 && y->dtype == IGC_DATA_BFLOAT16)) ||
        !matrix_of(*x, mx) || !matrix_of(*y, my))
        return IGC_STATUS_NOT_SUPPORTED;
    return IGC_STATUS_SUCCESS;
}

constexpr long long kMostGroups = 1ll << 21;   // workgroups of a launch (times 1024 threads: a 32-bit number); more tiles are taken in turns

template <class F>
igcStatus with_types(igcDataType in, igcDataType out, F f) {
    if (in == IGC_DATA_FLOAT) return f(float(), float());
    return out == IGC_DATA_FLOAT ? f(bf16_t(), float()) : f(bf16_t(), bf16_t());
}

long long round_up(long long v, long long to) { return (v + to - 1) / to * to; }

// Few tokens: pieces of 16 TB tokens and 16 KB rows of W, the reduction in ranges where those are few; x in parts first where several pieces of float tokens would make
// them again and again.
struct FewPlan {
    int kb = 1, tb = 1, splits = 1, per = 0;      // per: blocks to a range
    bool lay = false;
    size_t partsAt = 0, room = 0;
    double us = 0.0;
};
// us, measured, for the choice between kernels.  Of a block of 128 features: by the shape of a tile (of 64 x 128 one on a compute unit and two; float in parts: 64 x 256 and
// 64 x 128), at groups of 64; of 17 to 32 and more tokens in the few-token kernels, a block to each wavefront (kCrooked: bfloat16 rows off 16-byte boundaries); of a launch and a
// tile's start; bytes per us of ranges' sums that are stored and read.  2048 x 4096 -> 8192 one round of 256 x 256, after some calls 128 us, or two of 128 x 256, 157; 64 x 4096 -> 16384, groups of
// 128: 64 x 128 in one, two, four and eight ranges 27.7, 23.1, 23.8 and 31.5 us, 128 x 128 39.5, 29.1, 35.7 and 46.8, few-token kernel 44.8; 64 x 1024 -> 2048 tiles 9.5, few-token
// kernel 7.4; float 64 x 4096 -> 10880 30 and 77; 100 x 5001 -> 2003 20 and 36.
constexpr double kBlockUs[kTile4Shapes] = {2.45, 1.2, 4.0, 0.8}, kTwoBlocksUs = 1.45, kPartsBlockUs[kTile4Shapes] = {2.1, 0.0, 0.0, 1.35}, kFewBlockUs[3] = {0.0, 2.5, 4.6},
                 kFewPartsBlockUs[3] = {0.0, 4.5, 11.5}, kCrooked = 1.7, kLaunchUs = 3.5, kStartUs = 1.5, kSumBytes = 6e6;
double sums_us(long long splits, const Linear4Args &a) { return splits > 1 ? kLaunchUs + (double)splits * a.M * a.N * 8 / kSumBytes : 0.0; }
FewPlan plan_few(const igcContext *h, igcDataType in, const Linear4Args &a, size_t room) {
    FewPlan p;
    const int blocks = (a.K + kBlock - 1) / kBlock;
    p.tb = a.M <= 16 ? 1 : (a.M <= 32 ? 2 : 4);
    const long long tm = (a.M + 16 * p.tb - 1) / (16 * p.tb);
    auto tiles = [&](int kb) { return tm * ((a.N + 16 * kb - 1) / (16 * kb)); };
    const int most = p.tb == 1 ? 4 : 2;      // (registers)
    p.per = blocks;
    if (in == IGC_DATA_FLOAT && p.tb > 1) {
        const size_t bytes = (size_t)round_up(round_up(a.M, kPartsTokens) * 3 * round_up(a.K, 8) * 2, 256);
        if (bytes <= room) p.lay = true, p.partsAt = p.room = bytes;
    }
    const bool parts = in == IGC_DATA_FLOAT;
    const bool crooked = !parts && (a.K % 8 != 0 || a.am % 8 != 0), small = a.group4 == 32;
    // a block: of sixteen tokens by rows of W and tokens (1 x 4096 -> 4096, groups of 128: 16 rows and no ranges 5.8 us, 64 rows and four ranges 8.9; 16 x 16000 -> 333 one and
    // twelve ranges 17 and 10), of more by its shape
    auto block_us = [&](int kb) {
        if (p.tb > 1) return (parts ? kFewPartsBlockUs : kFewBlockUs)[p.tb / 2] * (crooked ? kCrooked : 1.0);
        const double tokens = a.M * (crooked ? 0.15 : 0.045) + (crooked && small ? 0.9 : 0.0);
        return tokens + (parts ? (small ? 1.05 + 0.85 * kb : 1.2 + 0.6 * kb) : (small ? 0.35 + 0.65 * kb : 0.35 + 0.4 * kb));
    };
    auto cost = [&](const FewPlan &q) {
        const long long rounds = (tiles(q.kb) * q.splits + h->computeUnits - 1) / h->computeUnits;
        return rounds * ((q.per + 7) / 8) * block_us(q.kb) + kLaunchUs * (1 + q.lay) + sums_us(q.splits, a);
    };
    // Without ranges: of sixteen tokens as many rows of W to a workgroup as cost least (1 x 4096 -> 10880, groups of 128: 16, 32 and 64 rows 15.8, 14.6 and 12.1 us,
    // 1 x 8192 -> 8192 16.6, 14.4 and 19.7), of more 32 where that leaves one workgroup for each compute unit.
    p.us = cost(p);
    for (FewPlan q = p; q.kb < most;) {
        q.kb *= 2;
        if (p.tb > 1 && tiles(q.kb) < h->computeUnits) break;
        q.us = cost(q);
        if (q.us < p.us || p.tb > 1) p.kb = q.kb, p.us = q.us;
    }
    // Ranges, each of a block for every wavefront at least, where they cost less with the second launch.
    if (p.kb < most || p.tb == 1) {
        // (no more workgroups than compute units: 64 x 5001 -> 2003 bfloat16 in 5 ranges 32 us, in 4 23; 1 x 4096 -> 10880 float in two 21, in one 16)
        const int splits = (int)std::min<long long>(std::max(1ll, h->computeUnits / tiles(most)), (blocks + 7) / 8);
        const size_t bytes = (size_t)splits * a.M * round_up(a.N, 4) * 4;
        FewPlan q = p;
        q.kb = most;
        q.per = (blocks + splits - 1) / splits;
        q.splits = (blocks + q.per - 1) / q.per;
        q.room = p.partsAt + bytes;
        q.us = cost(q);
        if (splits > 1 && q.room <= room && q.us < p.us) return q;
    }
    return p;
}

template <int KB, int TB, class TX, class TO>
const void *few_kernel(int group) {
    if constexpr (TB == 1)
        return group == 32 ? reinterpret_cast<const void *>(&linear4_few_kernel<KB, 32, TX, TO>)
                           : (group == 64 ? reinterpret_cast<const void *>(&linear4_few_kernel<KB, 64, TX, TO>) : reinterpret_cast<const void *>(&linear4_few_kernel<KB, 128, TX, TO>));
    else
        return reinterpret_cast<const void *>(&linear4_pieces_kernel<KB, TB, TX, TO>);
}
template <class TX, class TO>
const void *few_kernel(const FewPlan &p, int group) {
    if (p.tb == 1) return p.kb == 4 ? few_kernel<4, 1, TX, TO>(group) : (p.kb == 2 ? few_kernel<2, 1, TX, TO>(group) : few_kernel<1, 1, TX, TO>(group));
    if constexpr (sizeof(TX) == 4) {
        if (p.lay) {
            if (p.tb == 2) return p.kb == 2 ? few_kernel<2, 2, Laid, TO>(group) : few_kernel<1, 2, Laid, TO>(group);
            return p.kb == 2 ? few_kernel<2, 4, Laid, TO>(group) : few_kernel<1, 4, Laid, TO>(group);
        }
    }
    if (p.tb == 2) return p.kb == 2 ? few_kernel<2, 2, TX, TO>(group) : few_kernel<1, 2, TX, TO>(group);
    return p.kb == 2 ? few_kernel<2, 4, TX, TO>(group) : few_kernel<1, 4, TX, TO>(group);
}

// to, toScales: null where x, the scales stay as they are
igcStatus lay_out(igcHandle_t handle, igcDataType in, Linear4Args &t, void *to, void *toScales = nullptr) {
    Lay4Args q{t.a, static_cast<uint16_t *>(to), t.am, t.M, t.K, (int)round_up(t.K, 8), 0, t.scales, static_cast<uint16_t *>(toScales), t.N,
               (t.K + t.group4 - 1) / t.group4, round_up(t.N, 2)};
    long long groups = 0;
    if (to) {
        q.groupsX = (unsigned)std::min((round_up(t.M, kPartsTokens) * (q.toRow / 8) + 255) / 256, kMostGroups);
        t.a = to;
        t.am = q.toRow;
    }
    if (toScales) {
        groups = std::min((q.scaleGroups * q.scaleRow + 255) / 256, kMostGroups);
        t.scales = q.toScales;
        t.scaleRow = q.scaleRow;
    }
    return launch_kernel(in == IGC_DATA_FLOAT ? reinterpret_cast<const void *>(&lay_out_kernel<float>) : reinterpret_cast<const void *>(&lay_out_kernel<bf16_t>), q,
                         dim3((unsigned)(q.groupsX + groups)), 256, handle->stream);
}

igcStatus finish(igcHandle_t handle, igcDataType out, const Linear4Args &t) {
    return launch_kernel(out == IGC_DATA_FLOAT ? reinterpret_cast<const void *>(&linear4_finish_kernel<float>) : reinterpret_cast<const void *>(&linear4_finish_kernel<bf16_t>), t,
                         dim3((unsigned)std::min((t.M * (t.partsRow / 4) + 255) / 256, kMostGroups)), 256, handle->stream);
}

template <class TX, class TO>
igcStatus run_few(igcHandle_t handle, const Linear4Args &a, const FewPlan &p, void *workSpace) {
    Linear4Args t = a;
    igcStatus st = IGC_STATUS_SUCCESS;
    if (p.lay && (st = lay_out(handle, IGC_DATA_FLOAT, t, workSpace)) != IGC_STATUS_SUCCESS) return st;
    t.tilesM = (a.M + 16 * p.tb - 1) / (16 * p.tb);
    t.tilesN = (a.N + 16 * p.kb - 1) / (16 * p.kb);
    t.splits = p.splits;
    t.stepsPerSplit = p.per;
    t.parts = reinterpret_cast<float *>(static_cast<uint8_t *>(workSpace) + p.partsAt);
    t.partsRow = round_up(a.N, 4);
    st = launch_kernel(few_kernel<TX, TO>(p, a.group4), t, dim3((unsigned)std::min((long long)t.tilesM * t.tilesN * t.splits, kMostGroups)), 512, handle->stream);
    if (st != IGC_STATUS_SUCCESS || p.splits == 1) return st;
    return finish(handle, sizeof(TO) == 4 ? IGC_DATA_FLOAT : IGC_DATA_BFLOAT16, t);
}

// The tiles for a call, or none: few tokens, or more workgroups than a launch holds.
struct Tile4Plan {
    TileKernel k{};
    bool lay = false, layScales = false;       // x, the scales are laid out first, in `room` bytes
    size_t scalesAt = 0, partsAt = 0, room = 0;
    int splits = 1, per = 0;      // per: blocks to a range
    long long tilesM = 0, tilesN = 0;
    double us = 1e300;
};
Tile4Plan plan_tiles4(const igcContext *h, igcDataType in, igcDataType out, const Linear4Args &a) {
    Tile4Plan best;
    if (a.M <= 16 || a.K > (1 << 22)) return best;
    const bool parts = in == IGC_DATA_FLOAT;
    const long long row = round_up(a.K, 8);
    Tile4Plan p;
    // (as they lie: rows on 4-byte boundaries of whole pieces of 16 bytes, none inside another, a tile's reach below 2^31 bytes)
    p.lay = parts || a.K % 8 != 0 || (uintptr_t)a.a % 4 != 0 || (a.M > 1 && (a.am % 2 != 0 || a.am < a.K)) || a.am >= (1 << 22);
    p.layScales = a.N % 2 != 0 || (uintptr_t)a.scales % 4 != 0;
    p.scalesAt = p.lay ? (size_t)round_up((parts ? round_up(a.M, kPartsTokens) * 3 : a.M) * row * 2, 256) : 0;
    p.partsAt = p.scalesAt + (p.layScales ? (size_t)round_up((a.K + a.group4 - 1) / a.group4 * round_up(a.N, 2) * 2, 256) : 0);
    const int blocks = (a.K + kBlock - 1) / kBlock;
    // (groups' sums and scales)
    const double scaled = a.group4 == 32 ? 1.15 : (a.group4 == 64 ? 1.0 : 0.9);
    for (int shape = 0; shape < kTile4Shapes; ++shape) {
        p.k = tile4_kernel(shape, a.group4, parts, out == IGC_DATA_FLOAT);
        if (!p.k.kernel) continue;
        p.tilesM = (a.M + p.k.bm - 1) / p.k.bm;
        p.tilesN = (a.N + p.k.bn - 1) / p.k.bn;
        if (p.tilesM * p.tilesN > kMostGroups) continue;
        const double one = scaled * (parts ? kPartsBlockUs : kBlockUs)[shape], two = shape == 3 && !parts ? scaled * kTwoBlocksUs : 2.0 * one;
        // the reduction in ranges of two blocks and more
        for (int splits = 1; splits == 1 || (shape != 2 && splits <= std::min(16, blocks / 2) && p.tilesM * p.tilesN * (splits - 1) < 2 * h->computeUnits); ++splits) {
            p.per = (blocks + splits - 1) / splits;
            p.splits = (blocks + p.per - 1) / p.per;
            const long long rounds = (p.tilesM * p.tilesN * p.splits + h->computeUnits - 1) / h->computeUnits;
            p.us = kStartUs + p.per * (rounds / 2 * two + rounds % 2 * one) + kLaunchUs * (1 + (p.lay || p.layScales)) + sums_us(p.splits, a);
            if (p.us >= best.us) continue;
            best = p;
            best.room = p.partsAt + (p.splits > 1 ? (size_t)p.splits * a.M * round_up(a.N, 8) * 4 : 0);
        }
    }
    return best;
}

igcStatus run_tiles4(igcHandle_t handle, igcDataType in, igcDataType out, const Linear4Args &a, const Tile4Plan &pl, void *workSpace) {
    Linear4Args t = a;
    igcStatus st = IGC_STATUS_SUCCESS;
    t.scaleRow = a.N;
    uint8_t *ws = static_cast<uint8_t *>(workSpace);
    if ((pl.lay || pl.layScales) && (st = lay_out(handle, in, t, pl.lay ? ws : nullptr, pl.layScales ? ws + pl.scalesAt : nullptr)) != IGC_STATUS_SUCCESS) return st;
    t.tilesM = (int)pl.tilesM; t.tilesN = (int)pl.tilesN;
    t.splits = pl.splits;
    t.stepsPerSplit = pl.per;
    t.parts = reinterpret_cast<float *>(ws + pl.partsAt);
    t.partsRow = round_up(a.N, 8);
    t.tilesPerXcd = (int)((pl.tilesM * pl.tilesN * pl.splits + 7) / 8);
    t.group = std::min(t.tilesM, 4);
    st = launch_kernel(pl.k.kernel, t, dim3((unsigned)t.tilesPerXcd * 8u), pl.k.threads, handle->stream);
    if (st != IGC_STATUS_SUCCESS || pl.splits == 1) return st;
    return finish(handle, out, t);
}

Linear4Args sizes_of(const Matrix &x, const igcFilterStruct &w, int group) {
    Linear4Args a{};
    a.am = x.stride; a.ak = 1;
    a.M = (int)x.rows; a.N = w.k; a.K = w.c;
    a.group4 = group;
    return a;
}

}  // namespace
}  // namespace igc

using namespace igc;

extern "C" {

igcStatus igcGetFilter4Size(igcFilterDescriptor_t wDesc, int group, size_t *codeBytes, size_t *scaleBytes) {
    if (!codeBytes || !scaleBytes) return IGC_STATUS_BAD_PARAM;
    const igcStatus st = check_filter(wDesc, group);
    if (st != IGC_STATUS_SUCCESS) return st;
    *codeBytes = (size_t)(wDesc->k * code_row(wDesc->c));
    *scaleBytes = (size_t)((wDesc->c + group - 1) / group) * wDesc->k * 2;
    return IGC_STATUS_SUCCESS;
}

igcStatus igcQuantizeFilter4(igcHandle_t handle, igcFilterDescriptor_t wDesc, const void *w, int group, void *codes, void *scales) {
    if (!handle || !w || !codes || !scales) return IGC_STATUS_BAD_PARAM;
    const igcStatus st = check_filter(wDesc, group);
    if (st != IGC_STATUS_SUCCESS) return st;
    if (off(w, elem_size(wDesc->dtype)) || off(codes, 16) || off(scales, 2)) return IGC_STATUS_BAD_PARAM;
    StoreArgs a{};
    a.w = w;
    a.codes = static_cast<uint8_t *>(codes);
    a.scales = static_cast<uint16_t *>(scales);
    a.K = wDesc->k; a.C = wDesc->c; a.group = group;
    a.tiles = (long long)((a.C + kBlock - 1) / kBlock) * ((a.K + 63) / 64);
    const void *kernel = wDesc->dtype == IGC_DATA_FLOAT ? reinterpret_cast<const void *>(&to_four_bits_kernel<float>) : reinterpret_cast<const void *>(&to_four_bits_kernel<bf16_t>);
    return launch_kernel(kernel, a, dim3((unsigned)std::min(a.tiles, kMostGroups)), 256, handle->stream);
}

igcStatus igcDequantizeFilter4(igcHandle_t handle, int group, const void *codes, const void *scales, igcFilterDescriptor_t wDesc, void *w) {
    if (!handle || !w || !codes || !scales) return IGC_STATUS_BAD_PARAM;
    const igcStatus st = check_filter(wDesc, group);
    if (st != IGC_STATUS_SUCCESS) return st;
    if (off(w, elem_size(wDesc->dtype)) || off(codes, 16) || off(scales, 2)) return IGC_STATUS_BAD_PARAM;
    StoreArgs a{};
    a.out = w;
    a.codes = const_cast<uint8_t *>(static_cast<const uint8_t *>(codes));
    a.scales = const_cast<uint16_t *>(static_cast<const uint16_t *>(scales));
    a.K = wDesc->k; a.C = wDesc->c; a.group = group;
    a.tiles = (long long)((a.C + kBlock - 1) / kBlock) * ((a.K + 63) / 64);
    const void *kernel = wDesc->dtype == IGC_DATA_FLOAT ? reinterpret_cast<const void *>(&from_four_bits_kernel<float>) : reinterpret_cast<const void *>(&from_four_bits_kernel<bf16_t>);
    return launch_kernel(kernel, a, dim3((unsigned)std::min(a.tiles, kMostGroups)), 256, handle->stream);
}

igcStatus igcGetLinear4ForwardWorkspaceSize(igcHandle_t handle, igcTensorDescriptor_t xDesc, igcFilterDescriptor_t wDesc, int group, igcTensorDescriptor_t yDesc,
                                            size_t *sizeInBytes) {
    if (!handle || !sizeInBytes) return IGC_STATUS_BAD_PARAM;
    Matrix x, y;
    const igcStatus st = check_product(xDesc, wDesc, group, yDesc, &x, &y);
    if (st != IGC_STATUS_SUCCESS) return st;
    Linear4Args a = sizes_of(x, *wDesc, group);
    const FewPlan few = plan_few(handle, xDesc->dtype, a, ~(size_t)0);
    *sizeInBytes = 0;
    for (int off_words : {0, 1}) {      // (x and scales on 4-byte boundaries and off them)
        if (off_words) a.a = a.scales = reinterpret_cast<const uint16_t *>(2);
        const Tile4Plan pl = plan_tiles4(handle, xDesc->dtype, yDesc->dtype, a);
        *sizeInBytes = std::max(*sizeInBytes, pl.us <= few.us ? pl.room : few.room);
    }
    return IGC_STATUS_SUCCESS;
}

igcStatus igcLinear4Forward(igcHandle_t handle, const void *alpha, igcTensorDescriptor_t xDesc, const void *x, igcFilterDescriptor_t wDesc, int group,
                            const void *codes, const void *scales, void *workSpace, size_t workSpaceSizeInBytes, const void *bias, int activation, const void *beta,
                            igcTensorDescriptor_t rDesc, const void *r, igcTensorDescriptor_t yDesc, void *y) {
    if (!handle || !alpha || !beta || !x || !codes || !scales || !y || activation < IGC_ACTIVATION_IDENTITY || activation > IGC_ACTIVATION_SILU) return IGC_STATUS_BAD_PARAM;
    Matrix mx, my, mr;
    const igcStatus st = check_product(xDesc, wDesc, group, yDesc, &mx, &my);
    if (st != IGC_STATUS_SUCCESS) return st;
    Linear4Args a = sizes_of(mx, *wDesc, group);
    a.alpha = *static_cast<const float *>(alpha);
    a.beta = *static_cast<const float *>(beta);
    if (a.beta != 0.f) {
        if (!rDesc || !r) return IGC_STATUS_BAD_PARAM;
        if (!rDesc->set) return IGC_STATUS_NOT_INITIALIZED;
        if (!same_positions(*yDesc, *rDesc) || yDesc->dim[1] != rDesc->dim[1] || off(r, elem_size(rDesc->dtype))) return IGC_STATUS_BAD_PARAM;
        if (rDesc->dtype != yDesc->dtype || !matrix_of(*rDesc, &mr)) return IGC_STATUS_NOT_SUPPORTED;
    }
    if (off(x, elem_size(xDesc->dtype)) || off(y, elem_size(yDesc->dtype)) || off(bias, 4) || off(codes, 16) || off(scales, 2)) return IGC_STATUS_BAD_PARAM;
    a.a = x;
    a.bias = static_cast<const float *>(bias);
    a.act = activation;
    a.r = r; a.rs = mr.stride;
    a.y = y; a.ys = my.stride;
    a.codes = static_cast<const uint8_t *>(codes);
    a.scales = static_cast<const uint16_t *>(scales);
    const Tile4Plan pl = plan_tiles4(handle, xDesc->dtype, yDesc->dtype, a);
    const size_t room = workSpace && !off(workSpace, 16) ? workSpaceSizeInBytes : 0;
    const FewPlan few = plan_few(handle, xDesc->dtype, a, room);
    if (pl.room <= room && pl.us <= few.us) return run_tiles4(handle, xDesc->dtype, yDesc->dtype, a, pl, workSpace);
    return with_types(xDesc->dtype, yDesc->dtype, [&](auto tx, auto ty) { return run_few<decltype(tx), decltype(ty)>(handle, a, few, workSpace); });
}

}  // extern "C"
