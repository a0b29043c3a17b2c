// Many tokens times a filter in four bits.  A workgroup computes a BM x BN tile.  Everything goes from memory straight into LDS: x up to six steps of 64 features ahead, codes
// and scales three blocks of 128 ahead; the wavefronts make bfloat16 of their codes in registers.  No load goes into registers in the loop: the compiler, which does not
// know of the copies, would wait for all of them with it (2048 x 4096 -> 8192, groups of 64, tiles of 128 x 256: 198 us that way, 160 this way).
//
// A group's products are summed from zero, and multiplied by the group's scale into the result: 4 multiply-adds for each matrix instruction that ends
// a group (groups of 32: all of them, of 128: every fourth).  They follow the next unit's matrix instructions, which do not wait for them nor they for these.  Few tiles: the
// reduction in ranges of blocks, added by linear4_finish_kernel.
#ifndef IGCONV_LINEAR4_TILES_HPP_
#define IGCONV_LINEAR4_TILES_HPP_

#include "igconv_linear4.h"

namespace igc {

// PARTS: 3: a tile's rows of x are BM rows of each part in turn.
template <int BM_, int BN_, int WAVES_M_, int WAVES_N_, int PARTS_, int GROUP_, int X_SLOTS_>
struct Tile4Config {
    static constexpr int BM = BM_, BN = BN_, WAVES_M = WAVES_M_, WAVES_N = WAVES_N_, WAVES = WAVES_M * WAVES_N, THREADS = 64 * WAVES;
    static constexpr int PARTS = PARTS_, GROUP = GROUP_, ROWS = BM * PARTS;
    static constexpr int FM = BM / WAVES_M / 16, FN = BN / WAVES_N / 16;
    static constexpr int SCALES = kCodeBlock / GROUP;      // groups in a block
    // Places: of a step's x, a block's codes, a block's scales (which are read until the block's end, codes only at its start).
    static constexpr int X_SLOTS = X_SLOTS_, X_BYTES = ROWS * 128, CODE_SLOTS = 3, CODE_BYTES = BN * kCodeBlockBytes, SCALE_SLOTS = 4;
    static constexpr int SCALE_REQUESTS = (SCALES * (BN / 128) + WAVES - 1) / WAVES;            // of 256 bytes a wavefront and block
    static constexpr int CODE_REQUESTS = BN / 16 / WAVES, SCALE_BYTES = SCALES * BN * 2;
    static constexpr int LDS_BYTES = X_SLOTS * X_BYTES + CODE_SLOTS * CODE_BYTES + SCALE_SLOTS * SCALE_BYTES + 256 /* where requests beyond a block's go */;
    static_assert(LDS_BYTES <= 160 * 1024 && CODE_REQUESTS * 16 * WAVES == BN, "");
};

// 4 bytes per lane from global memory into LDS, as copy_to_lds
__device__ __forceinline__ void copy_words_to_lds(const u32x4 &buffer, uint32_t to, uint32_t offset) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(to), "v"(offset), "s"(buffer) : "m0");
}

// What a tile's wavefronts copy: x by steps, codes and scales by blocks, in rings of places.
template <class Cfg>
struct Copies4 {
    typedef OperandCopy<Cfg::ROWS, Cfg::WAVES, false, 2, false> CopyX;
    static constexpr int R = CopyX::REQUESTS, RC = Cfg::CODE_REQUESTS + Cfg::SCALE_REQUESTS, SCALES = Cfg::SCALES;
    CopyX x;
    uint8_t *lds, *lds_codes, *lds_scales;
    const uint8_t *codes_from;
    const uint16_t *scales_from;
    long long codes_left, scale_row;
    uint32_t row_bytes, code_at;
    int t0, N, K, lane, wave, first, blocks, groups, steps;     // blocks, steps: the range's ends
    int x_requested, x_slot = 0, requested, code_slot = 0, scale_slot = 0;
    u32x4 code_buf;
    uint32_t code_to, scale_to;
    int code_block;

    // (the range `split` of the blocks)
    __device__ __forceinline__ void init(const Linear4Args &p, uint8_t *lds_, int tm, int tn, int split, int lane_, int wave_) {
        lds = lds_;
        lds_codes = lds + Cfg::X_SLOTS * Cfg::X_BYTES;
        lds_scales = lds_codes + Cfg::CODE_SLOTS * Cfg::CODE_BYTES;
        lane = lane_;
        wave = wave_;
        t0 = tn * Cfg::BN;
        N = p.N;
        K = p.K;
        x.init(p.a, p.am, 1, tm * Cfg::ROWS, Cfg::PARTS == 1 ? p.M : p.tilesM * Cfg::ROWS, K, lane, wave);
        first = requested = split * p.stepsPerSplit;
        blocks = min((K + kCodeBlock - 1) / kCodeBlock, first + p.stepsPerSplit);
        x_requested = 2 * first;
        groups = (K + Cfg::GROUP - 1) / Cfg::GROUP;
        steps = min((K + 63) / 64, 2 * blocks);
        // Codes: a request of a wavefront is 16 rows' blocks of 64 bytes, four lanes a row, so that neighbours read neighbours; the four pieces of a row are permuted by
        // an exclusive or with the row's number, for the lanes of a read, which go down the rows, to lie in different banks.
        row_bytes = (uint32_t)code_row(K);
        codes_from = p.codes + (long long)t0 * row_bytes;
        codes_left = (long long)(N - t0) * row_bytes;
        code_at = (uint32_t)(wave * Cfg::CODE_REQUESTS * 16 + lane / 4) * row_bytes + (((lane & 3) ^ ((lane >> 4) & 3)) * 16u);
        scales_from = p.scales;
        scale_row = p.scaleRow;
    }
    __device__ __forceinline__ void begin_x() {
        x.begin(lds + x_slot * Cfg::X_BYTES, wave, x_requested * 64, K, x_requested < steps);
        ++x_requested;
        x_slot = x_slot == Cfg::X_SLOTS - 1 ? 0 : x_slot + 1;
    }
    __device__ __forceinline__ void request_x(int i) { x.request(i); }
    // (past the last block nothing is read, the counts stay alike)
    __device__ __forceinline__ void begin_codes() {
        const long long skip = (long long)requested * kCodeBlockBytes, left = codes_left - skip;
        code_buf = raw_buffer(codes_from + skip, requested < blocks ? (uint32_t)(left < 0x7FFFFFFFll ? left : 0x7FFFFFFFll) : 0u);
        code_to = lds_address(lds_codes) + code_slot * Cfg::CODE_BYTES + wave * Cfg::CODE_REQUESTS * 1024;
        scale_to = lds_address(lds_scales) + scale_slot * Cfg::SCALE_BYTES;
        code_block = requested;
        ++requested;
        code_slot = code_slot == Cfg::CODE_SLOTS - 1 ? 0 : code_slot + 1;
        scale_slot = scale_slot == Cfg::SCALE_SLOTS - 1 ? 0 : scale_slot + 1;
    }
    __device__ __forceinline__ void request_codes(int i) {
        if (i < Cfg::CODE_REQUESTS) {
            copy_to_lds(code_buf, code_to + i * 1024, code_at + (uint32_t)i * 16u * row_bytes);
            return;
        }
        // Scales: request q of the block takes 128 rows' of a group.  (Groups' rows begin on 4-byte boundaries.)
        const int q = wave * Cfg::SCALE_REQUESTS + i - Cfg::CODE_REQUESTS, in = q / (Cfg::BN / 128), group = code_block * SCALES + in, n = t0 + q % (Cfg::BN / 128) * 128;
        const bool there = in < SCALES && group < groups && n < N;
        const u32x4 rows = raw_buffer(there ? scales_from + (long long)group * scale_row + n : scales_from, there ? 2u * (uint32_t)min(128, N - n + (N & 1)) : 0u);
        copy_words_to_lds(rows, in < SCALES ? scale_to + q * 256 : lds_address(lds + Cfg::LDS_BYTES - 256), lane * 4u);
    }
    // a step's x, a block's codes and scales at once (in front of the loop)
    __device__ __forceinline__ void all_x() {
        begin_x();
#pragma unroll
        for (int i = 0; i < R; ++i) request_x(i);
    }
    __device__ __forceinline__ void all_codes() {
        begin_codes();
#pragma unroll
        for (int i = 0; i < RC; ++i) request_codes(i);
    }
    // where a wavefront's fragment j of a block's codes lies, four groups of eight to a lane
    __device__ __forceinline__ const uint8_t *codes_of(int slot, int fragment) const {
        const int l16 = lane & 15;
        return lds_codes + slot * Cfg::CODE_BYTES + fragment * 1024 + l16 * 64 + (((lane >> 4) ^ (l16 >> 2)) * 16);
    }
    __device__ __forceinline__ u32x2 scales_of(int slot, int in, int fragment) const {
        return *reinterpret_cast<const u32x2 *>(lds_scales + slot * Cfg::SCALE_BYTES + in * (Cfg::BN * 2) + (fragment * 16 + 4 * (lane >> 4)) * 2);
    }
};

// of all requests of a wavefront, `later` may be under way; its own reads of LDS are done
constexpr int requests_left(int later) { return 0x0070 | (later & 15) | ((later >> 4) << 14); }

template <class Cfg, class TO>
__global__ __launch_bounds__(Cfg::THREADS, 2) void linear4_tiles_kernel(const Linear4Args p) {
    constexpr int FM = Cfg::FM, FN = Cfg::FN, PARTS = Cfg::PARTS;
    __shared__ __attribute__((aligned(16))) uint8_t lds[Cfg::LDS_BYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave / Cfg::WAVES_N, wn = wave % Cfg::WAVES_N;
    int tm, tn, split;
    if (!tile_of(p, &tm, &tn, &split)) return;
    const int m0 = tm * Cfg::BM, n0 = tn * Cfg::BN + wn * FN * 16;
    Copies4<Cfg> copies;
    copies.init(p, lds, tm, tn, split, lane, wave);
    constexpr int R = Copies4<Cfg>::R, RC = Copies4<Cfg>::RC;
    OperandReads<Cfg::ROWS, FM, false, 2> reads;
    reads.init(wm * FM * 16, lane);

    bf16x8 x[2][PARTS][FM];
    auto read_x = [&](int slot, int kk) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < PARTS; ++n)
#pragma unroll
            for (int i = 0; i < FM; ++i) x[kk][n][i] = reads.read(lds + slot * Cfg::X_BYTES, kk, i + n * (Cfg::BM / 16));
    };
    u32x4 codes[FN], next_codes[FN];
    auto read_codes = [&](int slot, u32x4 (&to)[FN]) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < FN; ++j) to[j] = *reinterpret_cast<const u32x4 *>(copies.codes_of(slot, wn * FN + j));
    };
    constexpr int IN_GROUP = Cfg::GROUP / 32, SUMS = IN_GROUP == 1 ? 2 : FN;    // sums of groups that are under way, or wait for their scales
    f32x4 total[FM][FN], part[SUMS][FM];
    u32x2 scales[FN], ended_scale = {0u, 0u};
#pragma unroll
    for (int i = 0; i < FM; ++i) {
#pragma unroll
        for (int j = 0; j < FN; ++j) total[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 0; b < SUMS; ++b) part[b][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // the multiply-adds of a group that has ended
    auto add = [&](int b, int j) __attribute__((always_inline)) {
        const f32x4 s = widen_scales(ended_scale);
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) total[i][j][e] += s[e] * part[b][i][e];
    };
    // What a wavefront has requested after its x of step s + 1, in the middle of step s: x of S - 2 steps, and codes and scales with every other one of them.  (Codes are
    // requested five steps before they are waited for: 4 R + 2 RC after them.)
    constexpr int S = Cfg::X_SLOTS, LATER = (S - 2) * R + (S - 1) / 2 * RC;
    static_assert(S >= 3 && S <= 6 && LATER <= 4 * R + 2 * RC && LATER < 64 && (S - 1) * R < 64, "");
#pragma unroll
    for (int i = -6; i < 0; ++i) {       // (as in the middle of the steps before the first)
        if (i >= -S) copies.all_x();
        if (i % 2 == 0) copies.all_codes();
    }
    __builtin_amdgcn_s_waitcnt(requests_left((S - 1) * R));
    asm volatile("s_barrier" ::: "memory");
    read_x(0, 0);
    read_codes(0, codes);
    bf16x8 q = widen8(codes[0][0]);
    int xs = 0, cs = 0, ss = 0;       // places of the step's x, the block's codes and scales
    for (int block = copies.first; block < copies.blocks; ++block) {
        int ended = FN - 1, ended_in = IN_GROUP == 1 ? (FN - 1) & 1 : FN - 1;      // column of the group that ended last, with the block before, and where its sum is
#pragma unroll
        for (int i32 = 0; i32 < 4; ++i32) {
            const int kk = i32 & 1;
            if (kk == 0) {
                read_x(xs, 1);
            } else {
                // The next step's x, and its block's codes and scales, have landed; behind the barrier all wavefronts' have, and their reads of this step's x and of this
                // block's codes are done: S steps (three blocks) ahead goes to the same place.
                __builtin_amdgcn_s_waitcnt(requests_left(LATER));
                asm volatile("s_barrier" ::: "memory");
                copies.begin_x();
                xs = xs == Cfg::X_SLOTS - 1 ? 0 : xs + 1;
                read_x(xs, 0);
                if (i32 == 3) {
                    cs = cs == Cfg::CODE_SLOTS - 1 ? 0 : cs + 1;
                    read_codes(cs, next_codes);
                }
            }
            if (i32 == 2) copies.begin_codes();
            const bool ends = i32 % IN_GROUP == IN_GROUP - 1;
            if (ends)
#pragma unroll
                for (int j = 0; j < FN; ++j)
                    scales[j] = copies.scales_of(ss, i32 / IN_GROUP, wn * FN + j);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const int b = IN_GROUP == 1 ? j & 1 : j;
                // (a request to a unit: all wavefronts' at once wait for each other; codes and scales of a block between the first middle and the second)
                if (kk == 1)
#pragma unroll
                    for (int r = j; r < R; r += FN) copies.request_x(r);
                if (i32 == 2)
#pragma unroll
                    for (int r = j; r < RC; r += FN) copies.request_codes(r);
                const bf16x8 then = widen8(j + 1 < FN ? codes[j + 1][i32] : (i32 < 3 ? codes[0][i32 + 1] : next_codes[0][0]));
#pragma unroll
                for (int n = 0; n < PARTS; ++n)
#pragma unroll
                    for (int i = 0; i < FM; ++i) {
                        const f32x4 from = i32 % IN_GROUP == 0 && n == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : part[b][i];
                        part[b][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q, x[kk][n][i], from, 0, 0, 0);
                    }
                if (ended >= 0) add(ended_in, ended);
                ended = -1;
                if (ends) {
                    ended = j;
                    ended_in = b;
                    ended_scale = scales[j];
                }
                q = then;
                // (a few vector instructions between each two of the matrix unit's, which takes four times as long)
#pragma unroll
                for (int i = 0; i < FM * PARTS; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x2, PARTS == 1 ? 6 : 2, 0);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        ss = ss == Cfg::SCALE_SLOTS - 1 ? 0 : ss + 1;
#pragma unroll
        for (int j = 0; j < FN; ++j) codes[j] = next_codes[j];
    }
    add(IN_GROUP == 1 ? (FN - 1) & 1 : FN - 1, FN - 1);
    __builtin_amdgcn_s_waitcnt(requests_left(0));   // (nothing may be on its way into LDS)
    __syncthreads();
    write_results<FM, FN, Cfg::LDS_BYTES / Cfg::WAVES / 256 * 256, TO>(p, lds + wave * (Cfg::LDS_BYTES / Cfg::WAVES / 256 * 256), lane, split, m0 + wm * FM * 16, n0, total);
}

// The same with 256 x 256 results: a wavefront's 128 tokens share its 64 rows' decoded codes, a step's at a time, and go through one block of 16 tokens after the other, so that
// the groups' sums are 16 tokens by 64 rows at a time.  A group of 128 is added in two halves.  (2048 x 4096 -> 8192, groups of 64, the first 50 calls: 143 us, 160 with tiles of 128 x 256: half
// the decoding, twice the matrix instructions between barriers.  After 150 calls 124.)
template <class Cfg, class TO>
__global__ __launch_bounds__(Cfg::THREADS, 2) void linear4_wide_kernel(const Linear4Args p) {
    static_assert(Cfg::GROUP >= 64, "");      // a step's sums are one group's, or half of one
    constexpr int FM = Cfg::FM, FN = Cfg::FN;
    __shared__ __attribute__((aligned(16))) uint8_t lds[Cfg::LDS_BYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave / Cfg::WAVES_N, wn = wave % Cfg::WAVES_N;
    int tm, tn, split;
    if (!tile_of(p, &tm, &tn, &split)) return;
    Copies4<Cfg> copies;
    copies.init(p, lds, tm, tn, 0, lane, wave);      // (never in ranges)
    constexpr int R = Copies4<Cfg>::R, RC = Copies4<Cfg>::RC;
    OperandReads<Cfg::ROWS, FM, false, 2> reads;
    reads.init(wm * FM * 16, lane);

    f32x4 total[FM][FN], part[2][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) total[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    // At the end of a step the next one's x has landed, and its block's codes and scales: after that x a wavefront has requested x R times, and codes and scales RC times, with
    // the same step or the one before.  Behind the barrier all wavefronts' have, and this step's places are free.
    static_assert(Cfg::X_SLOTS == 3 && R + RC < 64, "");
    auto arrived = [&]() __attribute__((always_inline)) {
        __builtin_amdgcn_s_waitcnt(requests_left(R + RC));
        asm volatile("s_barrier" ::: "memory");
    };
    auto add = [](f32x4 &to, u32x2 scale, const f32x4 &sum) __attribute__((always_inline)) {
        const f32x4 s = widen_scales(scale);
#pragma unroll
        for (int e = 0; e < 4; ++e) to[e] += s[e] * sum[e];
    };
    copies.all_codes();      // (as in the steps before the first)
    copies.all_x();
    copies.all_codes();
    copies.all_x();
    __builtin_amdgcn_s_waitcnt(requests_left(R));
    asm volatile("s_barrier" ::: "memory");
    int xs = 0, cs = 0, ss = 0;       // places of the step's x, the block's codes and scales
    for (int block = copies.first; block < copies.blocks; ++block) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const uint8_t *here = lds + xs * Cfg::X_BYTES;
            bf16x8 q[2][FN], x[2][2];
            u32x2 scale[FN];
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) x[0][kk] = reads.read(here, kk, 0);
#pragma unroll
            for (int j = 0; j < FN; ++j) {
                const u32x2 c = *reinterpret_cast<const u32x2 *>(copies.codes_of(cs, wn * FN + j) + half * 8);
                q[0][j] = widen8(c[0]);
                q[1][j] = widen8(c[1]);
                scale[j] = copies.scales_of(ss, half * 64 / Cfg::GROUP, wn * FN + j);
            }
            copies.begin_x();
            if (half == 0) copies.begin_codes();
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                if (i + 1 < FM)
#pragma unroll
                    for (int kk = 0; kk < 2; ++kk) x[(i + 1) & 1][kk] = reads.read(here, kk, i + 1);
                // (a request to a unit: x goes where the step before had its own, codes and scales where the block before had)
                static_assert(R + RC <= FM, "");
                if (i < R) copies.request_x(i);
                else if (half == 0 && i - R < RC) copies.request_codes(i - R);
#pragma unroll
                for (int kk = 0; kk < 2; ++kk) {
                    const int b = i & 1;
#pragma unroll
                    for (int j = 0; j < FN; ++j) part[b][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[kk][j], x[b][kk], kk == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : part[b][j], 0, 0, 0);
                    // the sums that ended before these began
                    if (i == 0 || kk == 0) continue;
#pragma unroll
                    for (int j = 0; j < FN; ++j) add(total[i - 1][j], scale[j], part[b ^ 1][j]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int j = 0; j < FN; ++j) add(total[FM - 1][j], scale[j], part[(FM - 1) & 1][j]);
            arrived();
            xs = xs == Cfg::X_SLOTS - 1 ? 0 : xs + 1;
        }
        cs = cs == Cfg::CODE_SLOTS - 1 ? 0 : cs + 1;
        ss = ss == Cfg::SCALE_SLOTS - 1 ? 0 : ss + 1;
    }
    __builtin_amdgcn_s_waitcnt(requests_left(0));   // (nothing may be on its way into LDS)
    __syncthreads();
    write_results<FM, FN, Cfg::LDS_BYTES / Cfg::WAVES / 256 * 256, TO>(p, lds + wave * (Cfg::LDS_BYTES / Cfg::WAVES / 256 * 256), lane, 0, tm * Cfg::BM + wm * FM * 16,
                                                                        tn * Cfg::BN + wn * FN * 16, total);
}

}  // namespace igc
#endif
