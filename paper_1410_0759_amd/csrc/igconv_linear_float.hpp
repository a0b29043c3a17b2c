// Products of float matrices as products of bfloat16 parts.
//
// x = h + m + l, the upper, middle and lower 8 bits of its significand, each exact in bfloat16; a product a b is
//   l h + h l + m m + m h + h m + h h
// summed in that order (smallest first) in fp32; m l, l m and l l, below 2^-21 of the product together and about 2^-24 of it on average, are
// left out.  The matrix instructions do 16 times as many bfloat16 products as float ones in a cycle, so that six of them take a third
// of the time of one.  Parts have x's sign, and where a part would be zero though x is not it is the smallest subnormal number of
// that sign, 2^-133, which the matrix instructions take as it is: an infinite factor then meets no zero but in a product with zero itself.
// Parts end at 2^-133 too, so that of a number below 2^-110 the last bits are lost: x is off by less than 2^-131 in all (a float unit that flushes
// subnormal operands: 2^-126), which for a product a b comes to less than 2^-131 (|a| + |b|) beside what is left out.
//
// The parts lie in memory as they are wanted in LDS (linear_parts_pack_kernel): units of 1 KB, 16 rows by 32 reduction indices of one
// part, 16 bytes for each lane of a fragment in turn; the three parts of a block of rows next to each other, block after block of rows,
// then the next 32 reduction indices.  A step's copy is one run of memory per operand, a fragment one conflict-free read.
//
// A workgroup of eight wavefronts computes BM x BN results in steps of 32: three parts of both operands per step, copied two steps
// ahead into a ring of three stages.  A wavefront's slot is a block of 16 rows: 6 FN matrix instructions, with the next block's
// fragments on their way; before the last one the wavefronts meet, the stage after is complete and the one read is given to the copies.
//
// Bound by the matrix instructions: 4096^3 608 to 614 us, of them 51 for the parts, 226 TFLOP/s or 1.36 PFLOP/s in bfloat16 products (the float instruction's
// own tiles: 999 us).  1023 x 2050 -> 1000 takes 41 us: 9 for the parts, 27 for 256 workgroups of 17 steps, 6.6 for the sum of their ranges.
// 256 x 128 tiles (719 us for 656 at the time) and fragments taken column by column (651 for 626) were slower.
#ifndef IGCONV_LINEAR_FLOAT_HPP_
#define IGCONV_LINEAR_FLOAT_HPP_

#include "igconv_linear_tiles.hpp"

namespace igc {

constexpr int kFloatParts = 3, kUnitBytes = 1024;

template <int BM_, int BN_, int WAVES_M_, int WAVES_N_>
struct FloatConfig {
    static constexpr int BM = BM_, BN = BN_, WAVES_M = WAVES_M_, WAVES_N = WAVES_N_, WAVES = WAVES_M * WAVES_N, THREADS = 64 * WAVES;
    static constexpr int FM = BM / WAVES_M / 16, FN = BN / WAVES_N / 16, SF = FM / WAVES_N;
    static constexpr int UNITS_A = BM / 16 * kFloatParts, UNITS_B = BN / 16 * kFloatParts, REQUESTS = (UNITS_A + UNITS_B) / WAVES;
    static constexpr int STAGES = 3, STAGE_BYTES = (UNITS_A + UNITS_B) * kUnitBytes, LDS_BYTES = STAGES * STAGE_BYTES;
    static_assert(UNITS_A % REQUESTS == 0 && (UNITS_A + UNITS_B) % WAVES == 0, "a wavefront copies units of one operand");
    static_assert(LDS_BYTES <= 160 * 1024 && SF * WAVES_N == FM, "");
};

// SF sums of 16 rows of the first operand each, the same in all columns of a block (the products with ones)
template <int SF>
__device__ __forceinline__ void write_sums(const TileArgs &p, int lane, int range, int m0, const f32x4 (&sums)[SF]) {
#pragma unroll
    for (int i = 0; i < SF; ++i) {
        const int m = m0 + i * 16 + lane;
        if (lane < 16 && m < p.M) p.columnParts[(long long)range * p.M + m] = sums[i][0];
    }
}

template <class Cfg>
__global__ __launch_bounds__(Cfg::THREADS, 2) void linear_float_kernel(const TileArgs p) {
    constexpr int FM = Cfg::FM, FN = Cfg::FN, SF = Cfg::SF, R = Cfg::REQUESTS;
    __shared__ __attribute__((aligned(16))) uint8_t lds[Cfg::LDS_BYTES];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int wm = wave / Cfg::WAVES_N, wn = wave % Cfg::WAVES_N;
    int tm, tn, split;
    if (!tile_of(p, &tm, &tn, &split)) return;
    const int steps_all = (p.K + kFloatStep - 1) / kFloatStep, begin = split * p.stepsPerSplit, steps = min(p.stepsPerSplit, steps_all - begin);

    // this wavefront's share of the copies: R units of one operand
    const bool of_a = wave * R < Cfg::UNITS_A;
    const long long step_bytes = (long long)(of_a ? p.blocksA : p.blocksB) * (kFloatParts * kUnitBytes);
    const int unit0 = of_a ? wave * R : wave * R - Cfg::UNITS_A;
    const long long skip = begin * step_bytes + ((of_a ? tm * (Cfg::BM / 16) : tn * (Cfg::BN / 16)) * kFloatParts + unit0) * (long long)kUnitBytes;
    const uint8_t *from = static_cast<const uint8_t *>(of_a ? p.a : p.b) + skip;
    long long left = steps_all * step_bytes - skip;      // bytes from there to the operand's end (past it: zeros)
    int to_request = steps, request_stage = 0;
    u32x4 buf;
    uint32_t to;
    auto begin_requests = [&]() __attribute__((always_inline)) {
        // (past the last step: nothing is read, the counts stay alike)
        buf = raw_buffer(from, to_request > 0 && left > 0 ? (uint32_t)(left < 0x7FFFFFFFll ? left : 0x7FFFFFFFll) : 0u);
        to = lds_address(lds) + request_stage * Cfg::STAGE_BYTES + wave * R * kUnitBytes;
        --to_request;
        from += step_bytes;
        left -= step_bytes;
        request_stage = request_stage == Cfg::STAGES - 1 ? 0 : request_stage + 1;
    };
    // third g of a step's requests (a few to a slot: eight wavefronts with all of theirs at once wait for each other's)
    auto request = [&](int g) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (i * 3 / R == g) copy_to_lds(buf, to + i * kUnitBytes, (uint32_t)(i * kUnitBytes + lane * 16));
    };
    constexpr int kAllButOneStep = 0x0F70 | (R & 15) | ((R >> 4) << 14);

    const uint32_t at_a = (uint32_t)(wm * FM * kFloatParts * kUnitBytes + lane * 16), at_b = (uint32_t)((Cfg::UNITS_A + wn * FN * kFloatParts) * kUnitBytes + lane * 16);
    auto read = [&](bf16x8(&f)[kFloatParts], const uint8_t *at) __attribute__((always_inline)) {
#pragma unroll
        for (int q = 0; q < kFloatParts; ++q) f[q] = *reinterpret_cast<const bf16x8 *>(at + q * kUnitBytes);
    };
    f32x4 acc[FM][FN], sums[SF];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < SF; ++i) sums[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    bf16x8 ones;
#pragma unroll
    for (int e = 0; e < 8; ++e) ones[e] = (__bf16)1.f;
    // the sums of the first operand's rows are products with ones, the tiles of a row of tiles in turns, a step each
    int turn = p.columnParts ? tn : -1;

#pragma unroll
    for (int n = 0; n < 2; ++n) {
        begin_requests();
        request(0);
        request(1);
        request(2);
    }
    __builtin_amdgcn_s_waitcnt(kAllButOneStep);
    asm volatile("s_barrier" ::: "memory");
    begin_requests();
    request(0);
    bf16x8 a[2][kFloatParts], b[2][FN][kFloatParts];
    read(a[0], lds + at_a);
#pragma unroll
    for (int j = 0; j < FN; ++j) read(b[0][j], lds + at_b + j * kFloatParts * kUnitBytes);

    int stage = 0;
    auto step = [&](auto parity, auto with_sums) __attribute__((always_inline)) {
        constexpr int P = decltype(parity)::value;
        const uint8_t *here = lds + stage * Cfg::STAGE_BYTES;
        stage = stage == Cfg::STAGES - 1 ? 0 : stage + 1;
        const uint8_t *next = lds + stage * Cfg::STAGE_BYTES;
#pragma unroll
        for (int t = 0; t < FM; ++t) {
            if (t == FM - 1) {
                __builtin_amdgcn_s_waitcnt(0xC07F);            // this wavefront's reads of the stage are done
                __builtin_amdgcn_s_waitcnt(kAllButOneStep);    // its copies into the next one have landed
                asm volatile("s_barrier" ::: "memory");
                begin_requests();
                request(0);
                read(a[(t + 1) & 1], next + at_a);
#pragma unroll
                for (int j = 0; j < FN; ++j) read(b[P ^ 1][j], next + at_b + j * kFloatParts * kUnitBytes);
            } else {
                read(a[(t + 1) & 1], here + at_a + (t + 1) * kFloatParts * kUnitBytes);
            }
            if (t < 2) request(t + 1);   // (of the step that the barrier before gave its place)
            constexpr int part_a[6] = {2, 0, 1, 1, 0, 0}, part_b[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
            for (int q = 0; q < 6; ++q)
#pragma unroll
                for (int j = 0; j < FN; ++j)
                    acc[t][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[P][j][part_b[q]], a[t & 1][part_a[q]], acc[t][j], 0, 0, 0);
            if (decltype(with_sums)::value != 0 && wn == t / SF)
#pragma unroll
                for (int q = kFloatParts - 1; q >= 0; --q) sums[t % SF] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, a[t & 1][q], sums[t % SF], 0, 0, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    auto either = [&](auto parity) __attribute__((always_inline)) {
        if (turn == 0) step(parity, Constant<1>());
        else step(parity, Constant<0>());
        turn = turn == 0 ? p.tilesN - 1 : turn - 1;
    };
    static_assert(FM % 2 == 0 && FM > 2, "a step leaves the fragments where the next expects them");
    int s = 0;
    for (; s + 1 < steps; s += 2) {
        either(Constant<0>());
        either(Constant<1>());
    }
    if (s < steps) either(Constant<0>());

    __builtin_amdgcn_s_waitcnt(0x0F70);   // (nothing may be on its way into LDS)
    __syncthreads();
    write_results<FM, FN, Cfg::LDS_BYTES / Cfg::WAVES, float>(p, lds + wave * (Cfg::LDS_BYTES / Cfg::WAVES), lane, split, tm * Cfg::BM + wm * FM * 16,
                                                              tn * Cfg::BN + wn * FN * 16, acc);
    if (p.columnParts) write_sums<SF>(p, lane, split * p.tilesN + tn, tm * Cfg::BM + (wm * FM + wn * SF) * 16, sums);
}

}  // namespace igc
#endif
