// Products of matrices whose rows lie on 4-byte boundaries: bfloat16, and float with few tokens, where reading the filter is what takes the
// time (more of them: igconv_linear_float.hpp).
//
// A workgroup computes a BM x BN tile in steps of 128 bytes of the reduction, a wavefront of it FM x FN blocks of 16 x 16 with
// v_mfma_f32_16x16x32_bf16 or v_mfma_f32_16x16x4_f32.  (Blocks of 32 x 32 were slower: 8192^3
// 814 us instead of 754 with two places in LDS for each operand; it is 736 now.)  Both operands go from global memory straight into LDS (16 bytes per lane, no
// registers), two steps ahead.  An operand whose reduction index is adjacent in memory lies in LDS row by row (128 bytes a row) and is
// read 16 bytes per lane; one whose reduction index runs along the rows (w for backward data, x and dy for backward filter)
// lies there as it is, k by k, and is read with the transposing 8-byte reads (float: 4 bytes at a time) - no operand is transposed in memory.  In both cases
// the 16-byte (32-, 64-byte) pieces of a row are permuted by an exclusive or with the row's number so that the lanes of a read lie
// in different banks; the permutation is made on the global side of the copy, whose LDS side is fixed.
//
// Float rows may end inside a piece (their starts then lie off 16-byte boundaries too): what follows in the last piece is cleared in LDS, between two barriers
// before the last step.  8 x 4001 -> 16384 61 us that way, its data gradient 53 (the filter in no cache: 53 at a copy's rate); in bfloat16 parts, made of the
// whole filter for eight tokens, 204 and 213.
//
// A step is 2 x FM slots of FN matrix instructions.  Fragments of the first operand are read two slots ahead; those of the second operand's
// second half in the first quarter of the step, after which its place in LDS is free: there, at a first barrier, the step after next is
// requested (three places for the first operand, two for the second: all of the LDS with 256 x 256).  Two slots before the end, at a second
// barrier, the next step has to be there; the remaining matrix instructions cover its first reads.
//
// Tried at 8192^3 and slower: workgroups that stay and take several tiles (798 us for 743: a store before the next tile's copies holds up their
// waits), raised priority of the multiplying wavefronts (783 for 761), rings of four places (below).  Tiles taken 4 or 8 rows at a time: alike.
#ifndef IGCONV_LINEAR_TILES_HPP_
#define IGCONV_LINEAR_TILES_HPP_

#include "igconv_linear.h"

namespace igc {

using f32x4 = float __attribute__((ext_vector_type(4)));
using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using i16x4 = short __attribute__((ext_vector_type(4)));
using u32x2 = uint32_t __attribute__((ext_vector_type(2)));
using u32x4 = uint32_t __attribute__((ext_vector_type(4)));

constexpr uint32_t kNowhere = 0x80000000u;        // an offset outside every buffer: the load brings zeros

// neighbours in memory, on no boundary but their own
template <class T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Adjacent {
    T v[N];
};

// 16 bytes per lane from global memory into LDS at `to`, lane after lane; past the buffer's end: zeros.  In assembly (there is no register that
// it writes) because the compiler puts a wait for every such copy under way before each transposing read, which no alias information keeps
// it from: 8192^3 by backward filter 1060 us as against 796.  The waits are the kernels' own: `arrived`.
__device__ __forceinline__ void copy_to_lds(const u32x4 &buffer, uint32_t to, uint32_t offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(buffer) : "m0");
}
__device__ __forceinline__ uint32_t lds_address(const uint8_t *p) { return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t *)p; }
// the words of a raw buffer descriptor
__device__ __forceinline__ u32x4 raw_buffer(const void *base, uint32_t bytes) {
    const uint64_t at = (uint64_t)(uintptr_t)base;
    return u32x4{(uint32_t)at, (uint32_t)(at >> 32) & 0xFFFFu, bytes, 0x00020000u};
}

// One operand's copies into a stage: ROWS rows of the tile, from row `row0` of the operand; elements of ELEM bytes.
// STRIDED: the reduction index runs along the rows of the matrix in memory (`stride` elements apart), the tile's rows are adjacent.
// STAGED (bfloat16): the rows begin off 4-byte boundaries or end inside a piece, which copies straight into LDS do not serve; the lanes load the same pieces into
// registers, element by element where one is cut by the matrix's end, and write them to LDS a step later.
template <int ROWS, int WAVES, bool STRIDED, int ELEM, bool STAGED>
struct OperandCopy {
    static constexpr int REQUESTS = ROWS / 8 / WAVES;      // of 1 KB per wavefront and step
    static constexpr int PIECES = ROWS * ELEM / 16;        // (strided) 16-byte pieces of a k row
    static constexpr int KROWS = 64 / PIECES;              // (strided) k rows per request
    static constexpr int IN_PIECE = 16 / ELEM;
    const uint8_t *base;
    long long left;             // bytes from `base` to the end of the operand
    uint32_t stride_bytes, first;   // (descriptors hold strides below 2^31 elements: below 2^32 bytes where rows are read through registers)
    int k_piece, k_row;         // (not strided) the lane's first reduction index within a step, and its first row

    // (strided) the exclusive or of the pieces of k row k: the rows that a read takes at once lie in different banks
    static __device__ __forceinline__ int twist(int k) { return ELEM == 2 ? ((k & 3) | ((k >> 3) & 1) << 2) << 1 : ((k >> 2) & 3) << 2; }

    __device__ __forceinline__ void init(const void *matrix, long long row_stride, long long k_stride, int row0, int rows, int K, int lane, int wave) {
        rows_left = rows - row0;
        cols_left = rows - row0;
        k_row = wave * REQUESTS * 8 + (lane >> 3);
        // (Rows of bfloat16 end with a whole piece along the reduction index, of float anywhere: what follows the row in its last piece is cleared in LDS
        // (`cut`).  Strided, rows end with a whole word of 4 bytes: the last piece of a row may hold what follows the
        // row, which only reaches results outside the product.  Of a piece across the end of the buffer the words inside it are read, the
        // others are zeros, as was measured.)
        if constexpr (STRIDED) {
            base = static_cast<const uint8_t *>(matrix) + (long long)row0 * ELEM;
            left = ((K - 1) * k_stride + (rows + IN_PIECE / 4 - 1) / (IN_PIECE / 4) * (IN_PIECE / 4) - row0) * ELEM;
            stride_bytes = (uint32_t)k_stride * ELEM;
            const int k = lane / PIECES, at = lane % PIECES;
            k_piece = wave * REQUESTS * KROWS + k;       // (the k row of the first request)
            first = at;
        } else {
            base = static_cast<const uint8_t *>(matrix) + row0 * row_stride * ELEM;
            left = ((rows - row0 - 1) * row_stride + (ELEM == 4 ? K : (K + IN_PIECE - 1) / IN_PIECE * IN_PIECE)) * ELEM;
            stride_bytes = (uint32_t)row_stride * ELEM;
            const int row = lane >> 3, piece = (lane & 7) ^ row;
            first = (uint32_t)(wave * REQUESTS * 8 + row) * stride_bytes + piece * 16u;
            k_piece = piece * IN_PIECE;
        }
    }

    // the step that begins at reduction index k (of K), to be copied to `to`; not live: reads nothing, the counts of requests stay alike
    u32x4 buf;
    uint32_t to;
    int k, K;
    // (staged) rows and columns of the matrix from the tile's first on, the pieces in registers and where they go
    int rows_left, cols_left;
    u32x4 held[STAGED ? REQUESTS : 1];
    uint8_t *held_to, *next_to;
    __device__ __forceinline__ void begin(uint8_t *stage, int wave, int k_, int K_, bool live) {
        if constexpr (STAGED) {
            held_to = next_to;
            next_to = stage + wave * REQUESTS * 1024 + (threadIdx.x & 63) * 16;
            k = k_;
            K = live ? K_ : 0;
            return;
        }
        const long long skip = STRIDED ? (long long)k_ * stride_bytes : 0, bytes = left - skip;
        buf = raw_buffer(base + skip, live ? (uint32_t)(bytes < 0x7FFFFFFFll ? bytes : 0x7FFFFFFFll) : 0u);
        to = lds_address(stage) + wave * REQUESTS * 1024;
        k = k_;
        K = K_;
    }
    __device__ __forceinline__ void store(int i) { *reinterpret_cast<u32x4 *>(held_to + i * 1024) = held[i]; }
    __device__ __forceinline__ void request(int i) {
        if constexpr (STAGED) {
            const int row = STRIDED ? k + k_piece + i * KROWS : k_row + i * 8, col = STRIDED ? (int)(first ^ (uint32_t)twist(k_piece + i * KROWS)) * IN_PIECE : k + k_piece;
            const int there = row < (STRIDED ? K : rows_left) ? (STRIDED ? cols_left : K) - col : 0;   // elements
            const uint16_t *from = reinterpret_cast<const uint16_t *>(base + (long long)row * stride_bytes) + col;
            if (there >= 8) {
                held[i] = __builtin_bit_cast(u32x4, *reinterpret_cast<const Adjacent<uint16_t, 8> *>(from));
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t lo = 0, hi = 0;
                    if (2 * e < there) lo = from[2 * e];
                    if (2 * e + 1 < there) hi = from[2 * e + 1];
                    held[i][e] = lo | hi << 16;
                }
            }
            return;
        }
        uint32_t off;
        if constexpr (STRIDED) {
            const int kr = k_piece + i * KROWS;
            off = (uint32_t)kr * stride_bytes + (first ^ (uint32_t)twist(kr)) * 16u;
        } else {
            off = k + k_piece < K ? first + (uint32_t)i * 8u * stride_bytes + (uint32_t)k * ELEM : kNowhere;
        }
        copy_to_lds(buf, to + i * 1024, off);
    }

    // (float, not strided) The tile's rows end with index `end` of the step in `stage`: zeros in the rest of that index's piece, by all of the workgroup.
    static __device__ __forceinline__ void cut(uint8_t *stage, int end) {
        if constexpr (!STRIDED)
            for (int row = threadIdx.x; row < ROWS; row += 64 * WAVES) {
                float *piece = reinterpret_cast<float *>(stage + row * 128 + (((end / IN_PIECE) ^ (row & 7)) * 16));
                for (int e = end % IN_PIECE; e < IN_PIECE; ++e) piece[e] = 0.f;
            }
    }
};

// Fragments: eight bfloat16 or four float reduction indices of a row per lane.  Products of a block of 16 x 16 with half a step's indices (float: four
// instructions, each taking one of every lane's four).
template <int ELEM> struct Fragment;
template <> struct Fragment<2> {
    typedef bf16x8 type;
    static __device__ __forceinline__ f32x4 multiply(bf16x8 b, bf16x8 a, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(b, a, c, 0, 0, 0); }
};
template <> struct Fragment<4> {
    typedef f32x4 type;
    static __device__ __forceinline__ f32x4 multiply(f32x4 b, f32x4 a, f32x4 c) {
#pragma unroll
        for (int q = 0; q < 4; ++q) c = __builtin_amdgcn_mfma_f32_16x16x4f32(b[q], a[q], c, 0, 0, 0);
        return c;
    }
};

// One operand's fragments: F of them, 16 rows each, from row `row0` of the tile on.
template <int ROWS, int F, bool STRIDED, int ELEM>
struct OperandReads {
    typedef typename Fragment<ELEM>::type fragment_t;
    uint32_t at[STRIDED ? F : 2];
    __device__ __forceinline__ void init(int row0, int lane) {
        const int l16 = lane & 15, g = lane >> 4;
        if constexpr (STRIDED && ELEM == 2) {
            const int r = l16 >> 2, twist = r | (g & 1) << 2;
#pragma unroll
            for (int i = 0; i < F; ++i) at[i] = (uint32_t)((8 * g + r) * ROWS * 2 + (((row0 >> 4) + i) ^ twist) * 32 + (l16 & 3) * 8);
        } else if constexpr (STRIDED) {
#pragma unroll
            for (int i = 0; i < F; ++i) at[i] = (uint32_t)(4 * g * ROWS * 4 + (((row0 >> 4) + i) ^ g) * 64 + l16 * 4);
        } else {
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) at[kk] = (uint32_t)((row0 + l16) * 128 + ((g + 4 * kk) ^ (l16 & 7)) * 16);
        }
    }
    // fragment i of the step's half kk
    __device__ __forceinline__ fragment_t read(const uint8_t *stage, int kk, int i) const {
        if constexpr (STRIDED && ELEM == 2) {
            typedef __attribute__((address_space(3))) i16x4 *lds4;
            const uint8_t *p = stage + at[i] + kk * 32 * ROWS * 2;
            const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)p);
            const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds4)(p + 4 * ROWS * 2));
            return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else if constexpr (STRIDED) {
            f32x4 r;
#pragma unroll
            for (int q = 0; q < 4; ++q) r[q] = *reinterpret_cast<const float *>(stage + at[i] + (kk * 16 + q) * ROWS * 4);
            return r;
        } else {
            return *reinterpret_cast<const fragment_t *>(stage + at[kk] + i * 2048);
        }
    }
};

// eight neighbours of a row (which need not lie on a 16-byte boundary)
struct Eight {
    float v[8];
};
template <class TO>
__device__ __forceinline__ Eight load8(const void *p, long long at) {
    Eight r;
    if constexpr (sizeof(TO) == 4) {
        const Adjacent<float, 8> q = *reinterpret_cast<const Adjacent<float, 8> *>(static_cast<const float *>(p) + at);
#pragma unroll
        for (int e = 0; e < 8; ++e) r.v[e] = q.v[e];
    } else {
        const Adjacent<uint16_t, 8> a = *reinterpret_cast<const Adjacent<uint16_t, 8> *>(static_cast<const uint16_t *>(p) + at);
        const u32x4 q = __builtin_bit_cast(u32x4, a);
#pragma unroll
        for (int e = 0; e < 4; ++e) r.v[2 * e] = bf16_bits_to_float(q[e]), r.v[2 * e + 1] = __builtin_bit_cast(float, q[e] & 0xFFFF0000u);
    }
    return r;
}
template <class TO>
__device__ __forceinline__ void store8(void *p, long long at, const Eight &r) {
    if constexpr (sizeof(TO) == 4) {
        *reinterpret_cast<Adjacent<float, 8> *>(static_cast<float *>(p) + at) = __builtin_bit_cast(Adjacent<float, 8>, r);
    } else {
        u32x4 q;
#pragma unroll
        for (int e = 0; e < 4; ++e) q[e] = to_bf16_pair(r.v[2 * e], r.v[2 * e + 1]);
        *reinterpret_cast<Adjacent<uint16_t, 8> *>(static_cast<uint16_t *>(p) + at) = __builtin_bit_cast(Adjacent<uint16_t, 8>, q);
    }
}
// finish_element for eight results at once
template <class TO>
__device__ __forceinline__ void finish8(const LinearArgs &a, int m, int n, Eight d, const Eight &bias) {
    constexpr bool FINE = sizeof(TO) == 4;
#pragma unroll
    for (int e = 0; e < 8; ++e) d.v[e] = a.alpha * d.v[e] + bias.v[e];
    if (a.z) store8<TO>(a.z, m * a.zs + n, d);
    if (a.zin) {
        const Eight z = load8<TO>(a.zin, m * a.zs + n);
        by_activation(a.act, [&](auto act) {
#pragma unroll
            for (int e = 0; e < 8; ++e) d.v[e] *= activation_slope<FINE>(decltype(act)::value, z.v[e]);
        });
    } else {
        by_activation(a.act, [&](auto act) {
#pragma unroll
            for (int e = 0; e < 8; ++e) d.v[e] = activation<FINE>(decltype(act)::value, d.v[e]);
        });
    }
    if (a.beta != 0.f) {
        const Eight r = load8<TO>(a.r, m * a.rs + n);
#pragma unroll
        for (int e = 0; e < 8; ++e) d.v[e] += a.beta * r.v[e];
    }
    store8<TO>(a.y, m * a.ys + n, d);
}

template <int BM_, int BN_, int WAVES_M_, int WAVES_N_, bool SA_, bool SB_, int ELEM_ = 2, bool STAGED_ = false>
struct TileConfig {
    static constexpr bool STAGED = STAGED_;
    static constexpr int BM = BM_, BN = BN_, WAVES_M = WAVES_M_, WAVES_N = WAVES_N_, WAVES = WAVES_M * WAVES_N;
    static constexpr bool SA = SA_, SB = SB_;
    static constexpr int ELEM = ELEM_, STEP = 128 / ELEM;   // bytes of the operands' elements, reduction indices per step
    static constexpr int FM = BM / WAVES_M / 16, FN = BN / WAVES_N / 16;
    // Steps requested ahead, and the places of both operands' rings: a step of B is free again within its own step, one of A after it.  (Four ahead, for
    // 128 x 128 tiles that leave room: 1000^3 17 us, two ahead 13.)
    static constexpr int AHEAD = 2, SLOTS_A = AHEAD + 1, SLOTS_B = AHEAD, BYTES_A = BM * 128, BYTES_B = BN * 128;
    static constexpr int LDS_BYTES = SLOTS_A * BYTES_A + SLOTS_B * BYTES_B;
    static_assert(LDS_BYTES <= 160 * 1024, "");
    static constexpr int THREADS = 64 * WAVES, SUM_ROWS = THREADS / (BM * ELEM / 16);   // k rows that the threads cover, a piece each
};

__device__ __forceinline__ bool tile_of(const TileArgs &p, int *tm, int *tn, int *split) {
    const int tiles = p.tilesM * p.tilesN, unit = (int)(blockIdx.x & 7u) * p.tilesPerXcd + (int)(blockIdx.x >> 3);
    if (unit >= tiles * p.splits) return false;
    *split = unit / tiles;
    const int t = unit - *split * tiles, width = p.group * p.tilesN, g = t / width, first = g * p.group;
    const int rows = p.tilesM - first < p.group ? p.tilesM - first : p.group, in = t - g * width;
    *tm = first + in % rows;
    *tn = in / rows;
    return true;
}

// A wavefront's results, FM x FN blocks of 16 x 16 from row m0, column n0 on: lane l holds row 16 i + l % 16, columns 16 j + 4 (l / 16) + 0..3.
// They go through the wavefront's share of the LDS (its 16-byte pieces permuted within a row by the row's number), as many rows at a time as
// it has room for, so that eight lanes write 128 or 256 adjacent bytes of a row of y.
template <int FM, int FN, int SHARE, class TO>
__device__ __forceinline__ void write_results(const TileArgs &p, uint8_t *share, int lane, int split, int m0, int n0, const f32x4 (&acc)[FM][FN]) {
    constexpr int WN = FN * 16, PIECES = WN / 4;
    constexpr int ROOM = SHARE / (16 * WN * 4), PASS_FRAGS = ROOM >= FM ? FM : (ROOM >= 4 ? 4 : (ROOM >= 2 ? 2 : 1));
    constexpr int PASSES = FM / PASS_FRAGS, LANES = WN / 8, AT_ONCE = 64 / LANES;
    static_assert(PASSES * PASS_FRAGS == FM, "whole passes");
    f32x4 *mine = reinterpret_cast<f32x4 *>(share);
    const int l16 = lane & 15, g = lane >> 4, c8 = lane % LANES, n = n0 + c8 * 8;
    Eight bias;
#pragma unroll
    for (int e = 0; e < 8; ++e) bias.v[e] = p.bias && n + e < p.N ? p.bias[n + e] : 0.f;
    for (int pass = 0; pass < PASSES; ++pass) {
        // (which accumulators is known at compile time: an index into registers)
#pragma unroll
        for (int q = 0; q < PASSES; ++q)
            if (pass == q)
#pragma unroll
                for (int i = 0; i < PASS_FRAGS; ++i)
#pragma unroll
                    for (int j = 0; j < FN; ++j) mine[(i * 16 + l16) * PIECES + ((j * 4 + g) ^ (l16 & (PIECES - 1)))] = acc[q * PASS_FRAGS + i][j];
        __builtin_amdgcn_wave_barrier();
        for (int r = lane / LANES; r < PASS_FRAGS * 16; r += AT_ONCE) {
            const int m = m0 + pass * PASS_FRAGS * 16 + r;
            const f32x4 lo = mine[r * PIECES + ((2 * c8) ^ (r & 15 & (PIECES - 1)))], hi = mine[r * PIECES + ((2 * c8 + 1) ^ (r & 15 & (PIECES - 1)))];
            if (m >= p.M || n >= p.N) continue;
            const Eight d = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
            if (p.splits > 1) store8<float>(p.parts, ((long long)split * p.M + m) * p.partsRow + n, d);
            else if (n + 8 <= p.N) finish8<TO>(p, m, n, d, bias);
            else
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (n + e < p.N) finish_element<TO>(p, m, n + e, d.v[e]);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

// What a workgroup does with its tile's results, all of whose LDS is free: its wavefront's are those from row m0, column n0 on.  Another TO or Args: another end.
template <class Cfg, class TO, class Args>
struct TileEnd {
    template <int FM, int FN>
    static __device__ __forceinline__ void run(const Args &p, uint8_t *lds, int lane, int wave, int split, int tm, int tn, int m0, int n0, f32x4 (&acc)[FM][FN]) {
        write_results<FM, FN, Cfg::LDS_BYTES / Cfg::WAVES, TO>(p, lds + wave * (Cfg::LDS_BYTES / Cfg::WAVES), lane, split, m0, n0, acc);
    }
};

template <class Cfg, class TO, class Args = TileArgs>
__global__ __launch_bounds__(Cfg::THREADS, 2) void linear_tiles_kernel(const Args p) {
    constexpr int BM = Cfg::BM, BN = Cfg::BN, FM = Cfg::FM, FN = Cfg::FN, SLOTS = 2 * FM, FREE = FM / 2;
    __shared__ __attribute__((aligned(16))) uint8_t lds[Cfg::LDS_BYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave / Cfg::WAVES_N, wn = wave % Cfg::WAVES_N;
    int tm, tn, split;
    if (!tile_of(p, &tm, &tn, &split)) return;
    const int m0 = tm * BM, n0 = tn * BN;
    OperandCopy<BM, Cfg::WAVES, Cfg::SA, Cfg::ELEM, Cfg::STAGED> copyA;
    OperandCopy<BN, Cfg::WAVES, Cfg::SB, Cfg::ELEM, Cfg::STAGED> copyB;
    copyA.init(p.a, p.am, p.ak, m0, p.M, p.K, lane, wave);
    copyB.init(p.b, p.bn, p.bk, n0, p.N, p.K, lane, wave);
    OperandReads<BM, FM, Cfg::SA, Cfg::ELEM> readA;
    OperandReads<BN, FN, Cfg::SB, Cfg::ELEM> readB;
    readA.init(wm * FM * 16, lane);
    readB.init(wn * FN * 16, lane);

    const int kBegin = split * p.stepsPerSplit * Cfg::STEP;
    const int kEnd = min(p.K, kBegin + p.stepsPerSplit * Cfg::STEP);
    const int steps = (kEnd - kBegin + Cfg::STEP - 1) / Cfg::STEP;
    int k = kBegin, slotA = 0, slotB = 0;       // of the next request
    uint8_t *const ldsB = lds + Cfg::SLOTS_A * Cfg::BYTES_A;
    constexpr int RA = decltype(copyA)::REQUESTS, RB = decltype(copyB)::REQUESTS, R = RA + RB;
    auto begin_requests = [&]() __attribute__((always_inline)) {
        const bool live = k < kEnd;
        copyA.begin(lds + slotA * Cfg::BYTES_A, wave, k, kEnd, live);
        copyB.begin(ldsB + slotB * Cfg::BYTES_B, wave, k, kEnd, live);
        k += Cfg::STEP;
        slotA = slotA == Cfg::SLOTS_A - 1 ? 0 : slotA + 1;
        slotB = slotB == Cfg::SLOTS_B - 1 ? 0 : slotB + 1;
    };
    auto request = [&](int i) __attribute__((always_inline)) {
        if (i < RA) copyA.request(i);
        else copyB.request(i - RA);
    };
    auto store = [&](int i) __attribute__((always_inline)) {
        if (i < RA) copyA.store(i);
        else copyB.store(i - RA);
    };
    constexpr int LATER = (Cfg::AHEAD - 1) * R;
    auto arrived = [&]() __attribute__((always_inline)) {     // all but the steps after the next
        if (Cfg::STAGED) __builtin_amdgcn_s_waitcnt(0xC07F);   // (this wavefront's writes)
        else __builtin_amdgcn_s_waitcnt(0x0F70 | (LATER & 15) | ((LATER >> 4) << 14));
        asm volatile("s_barrier" ::: "memory");
    };
    // The last step of float rows that end inside a piece, once it has arrived: the rest of the piece may be anything, the next row's infinities too.
    constexpr bool CUT = Cfg::ELEM == 4 && !(Cfg::SA && Cfg::SB);
    const int tail = CUT && kEnd % 4 != 0 ? kEnd - kBegin - (steps - 1) * Cfg::STEP : 0;
    auto cut = [&](int step, uint8_t *stageA, uint8_t *stageB) __attribute__((always_inline)) {
        if (!CUT || tail == 0 || step != steps - 1) return;
        decltype(copyA)::cut(stageA, tail);
        decltype(copyB)::cut(stageB, tail);
        __builtin_amdgcn_s_waitcnt(0xC07F);
        asm volatile("s_barrier" ::: "memory");
    };

    f32x4 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int n = 0; n < Cfg::AHEAD; ++n) {
        begin_requests();
#pragma unroll
        for (int i = 0; i < R; ++i) {
            if (Cfg::STAGED && n > 0) store(i);
            request(i);
        }
    }
    arrived();
    cut(0, lds, ldsB);
    typename Fragment<Cfg::ELEM>::type a[4], b[2][FN];
    a[0] = readA.read(lds, 0, 0);
    a[1] = readA.read(lds, 0, 1);
#pragma unroll
    for (int j = 0; j < FN; ++j) b[0][j] = readB.read(ldsB, 0, j);

    // (backward filter) The sums of the first operand's rows over the reduction: the tiles of a row of tiles, which share these rows, take them
    // in turns, a step each, from the step's stage: a thread the 16-byte pieces of one place of every SUM_ROWS-th k row, which hold the same
    // rows of the operand.  (A second body of the step with products with ones among the others spilled registers.  So the sums cost nothing
    // that shows: 8192 x 4096 -> 4096, 252 us with them and 253 without, and the sum over the tiles 4 us.)
    Eight sum = {};
    int turn = Cfg::SA && p.columnParts ? tn : -1;   // steps until the next one whose sums are this tile's

    constexpr int PER_SLOT = (R + SLOTS - 2 - FREE - 1) / (SLOTS - 2 - FREE);
    int atA = 0, atB = 0;
    for (int s = 0; s < steps; ++s) {
        const uint8_t *hereA = lds + atA * Cfg::BYTES_A, *hereB = ldsB + atB * Cfg::BYTES_B;
        atA = atA == Cfg::SLOTS_A - 1 ? 0 : atA + 1;
        atB = atB == Cfg::SLOTS_B - 1 ? 0 : atB + 1;
        uint8_t *nextA = lds + atA * Cfg::BYTES_A, *nextB = ldsB + atB * Cfg::BYTES_B;
        if constexpr (Cfg::SA) {
            if (turn == 0)
#pragma unroll
                for (int i = 0; i < Cfg::STEP / Cfg::SUM_ROWS; ++i) {
                    const uint8_t *piece = hereA + ((int)threadIdx.x + i * Cfg::THREADS) * 16;
                    if constexpr (Cfg::ELEM == 2) {
                        const Eight q = load8<bf16_t>(piece, 0);
#pragma unroll
                        for (int e = 0; e < 8; ++e) sum.v[e] += q.v[e];
                    } else {
                        const f32x4 q = *reinterpret_cast<const f32x4 *>(piece);
#pragma unroll
                        for (int e = 0; e < 4; ++e) sum.v[e] += q[e];
                    }
                }
            turn = turn == 0 ? p.tilesN - 1 : turn - 1;
        }
#pragma unroll
        for (int t = 0; t < SLOTS; ++t) {
            if (t == FREE) {
                __builtin_amdgcn_s_waitcnt(0xC07F);   // this wavefront's reads of B's step, and of A's step before, are done
                asm volatile("s_barrier" ::: "memory");
                begin_requests();
            }
            if (t == SLOTS - 2) {
                arrived();
                cut(s + 1, nextA, nextB);
            }
            // (a few to a slot: eight wavefronts with eight requests each at once wait for each other's)
#pragma unroll
            for (int i = 0; i < R; ++i)
                if (t == FREE + i / PER_SLOT) {
                    if (Cfg::STAGED) store(i);
                    request(i);
                }
            if (t + 2 < SLOTS) a[(t + 2) % 4] = readA.read(hereA, (t + 2) / FM, (t + 2) % FM);
            else a[(t + 2) % 4] = readA.read(nextA, 0, t + 2 - SLOTS);
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                if (t == j * FREE / FN) b[1][j] = readB.read(hereB, 1, j);
                if (t >= SLOTS - 2 && j / ((FN + 1) / 2) == t - (SLOTS - 2)) b[0][j] = readB.read(nextB, 0, j);
            }
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[t % FM][j] = Fragment<Cfg::ELEM>::multiply(b[t / FM][j], a[t % 4], acc[t % FM][j]);
            __builtin_amdgcn_sched_barrier(0);
        }
    }

    __builtin_amdgcn_s_waitcnt(0x0F70);   // (nothing may be on its way into LDS)
    __syncthreads();
    TileEnd<Cfg, TO, Args>::template run<FM, FN>(p, lds, lane, wave, split, tm, tn, m0 + wm * FM * 16, n0 + wn * FN * 16, acc);
    if constexpr (Cfg::SA) {
        if (p.columnParts) {
            typedef decltype(copyA) Copy;
            static_assert(Cfg::SUM_ROWS % 16 == 0 && Cfg::STEP % Cfg::SUM_ROWS == 0 && Cfg::SUM_ROWS * BM * 4 <= Cfg::LDS_BYTES, "");
            float *sums = reinterpret_cast<float *>(lds);   // [SUM_ROWS][BM]
            const int kr = (int)threadIdx.x / Copy::PIECES, piece = ((int)threadIdx.x % Copy::PIECES) ^ Copy::twist(kr);
            __syncthreads();
#pragma unroll
            for (int e = 0; e < Copy::IN_PIECE; ++e) sums[kr * BM + piece * Copy::IN_PIECE + e] = sum.v[e];
            __syncthreads();
            for (int m = threadIdx.x; m < BM && m0 + m < p.M; m += Cfg::THREADS) {
                float v = 0.f;
#pragma unroll
                for (int i = 0; i < Cfg::SUM_ROWS; ++i) v += sums[i * BM + m];
                p.columnParts[(long long)(split * p.tilesN + tn) * p.M + m0 + m] = v;
            }
        }
    }
}

}  // namespace igc
#endif
