// Cross entropy over a vocabulary, straight from the features in front of the last product:
//
//   z = x w^T + bias,  logSum_i = log sum_v exp z_iv,  loss_i = logSum_i - z_it
//   dz_iv = alpha dloss_i (exp(z_iv - logSum_i) - [v = t]),  dx = dz w + beta dx,  dw = dz^T x + paramBeta dw,  dbias = column sums of dz + paramBeta dbias
//
// The logits are never held whole: pieces of the vocabulary are multiplied, taken in and overwritten by the next piece's.  Forward, a piece leaves the largest
// logit of each row and range of columns and the sum of exp(z - largest); a last kernel joins them.  Backward, the piece's logits are made again, become dz, and go
// into two products.
#include "igconv_cross_entropy.h"
#include "igconv_linear_tiles.hpp"

namespace igc {
namespace {

constexpr int kRange = 2048;                         // columns of one entry of the row statistics
constexpr size_t kPieceBytes = (size_t)512 << 20;    // of logits (or dz) at a time

// (nothing but minus infinities: a sum of zero, and no difference of infinities)
__device__ __forceinline__ RowPart joined(RowPart a, RowPart b) {
    const float most = fmaxf(a.most, b.most);
    if (most == -INFINITY) return {most, a.sum + b.sum};
    return {most, a.sum * exp_of(a.most - most) + b.sum * exp_of(b.most - most)};
}

__device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

// ---- forward ------------------------------------------------------------------------------------------------------------
struct RowPartsArgs {
    const float *logits;        // [M][stride]
    long long stride;
    int M, columns, ranges;
    int first;                  // the piece's first vocabulary entry
    const int *targets;
    RowPart *parts;             // [range][M], from the piece's first range on
    float *picked;              // the targets' logits
};

// A wavefront takes a row's range of columns.
__global__ __launch_bounds__(256) void row_parts_kernel(const RowPartsArgs a) {
    const int lane = threadIdx.x & 63;
    const long long tasks = (long long)a.M * a.ranges;
    for (long long task = (long long)blockIdx.x * 4 + (threadIdx.x >> 6); task < tasks; task += (long long)gridDim.x * 4) {
        const int range = (int)(task / a.M);
        const long long m = task % a.M;
        const float *row = a.logits + m * a.stride;
        float z[kRange / 64];
#pragma unroll
        for (int i = 0; i < kRange / 256; ++i) {
            const int n = range * kRange + i * 256 + lane * 4;
#pragma unroll
            for (int e = 0; e < 4; ++e) z[4 * i + e] = -INFINITY;
            if (n + 4 <= a.columns) {
                const float4 q = *reinterpret_cast<const float4 *>(row + n);
                z[4 * i] = q.x; z[4 * i + 1] = q.y; z[4 * i + 2] = q.z; z[4 * i + 3] = q.w;
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (n + e < a.columns) z[4 * i + e] = row[n + e];
            }
        }
        float most = z[0];
#pragma unroll
        for (int i = 1; i < kRange / 64; ++i) most = fmaxf(most, z[i]);
        most = lanes_max(most);
        float sum = 0.f;
        if (most > -INFINITY)
#pragma unroll
            for (int i = 0; i < kRange / 64; ++i) sum += exp_of(z[i] - most);
        else
#pragma unroll
            for (int i = 0; i < kRange / 64; ++i) sum += z[i] == z[i] ? 0.f : z[i];     // (what is undefined stays so)
        sum = lanes_sum<64>(sum);
        if (lane == 0) {
            a.parts[(long long)range * a.M + m] = {most, sum};
            const long long t = (long long)a.targets[m] - a.first;
            if (t >= (long long)range * kRange && t < (long long)(range + 1) * kRange && t < a.columns) a.picked[m] = row[t];
        }
    }
}

struct LossArgs {
    const RowPart *parts;
    int M, V, ranges;
    const int *targets;
    const float *picked;
    float *loss, *logSum;
};

__device__ __forceinline__ void finish_loss(const LossArgs &a, long long m, RowPart row) {
    const float log_sum = row.most == -INFINITY ? row.most + row.sum : row.most + logf(row.sum);
    const int t = a.targets[m];
    a.loss[m] = t >= 0 && t < a.V ? log_sum - a.picked[m] : 0.f;
    if (a.logSum) a.logSum[m] = log_sum;
}

// 64 rows to a workgroup, its sixteen wavefronts on every sixteenth range.
__global__ __launch_bounds__(1024) void loss_kernel(const LossArgs a) {
    __shared__ RowPart parts[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (long long first = (long long)blockIdx.x * 64; first < a.M; first += (long long)gridDim.x * 64) {
        const long long m = first + lane;
        RowPart mine{-INFINITY, 0.f};
        if (m < a.M)
#pragma unroll 4
            for (int r = wave; r < a.ranges; r += 16) mine = joined(mine, a.parts[(long long)r * a.M + m]);
        parts[wave][lane] = mine;
        __syncthreads();
        if (wave == 0 && m < a.M) {
#pragma unroll
            for (int w = 1; w < 16; ++w) mine = joined(mine, parts[w][lane]);
            finish_loss(a, m, mine);
        }
        __syncthreads();
    }
}

// Few rows: a workgroup to a row, its threads on the ranges.
__global__ __launch_bounds__(1024) void loss_row_kernel(const LossArgs a) {
    __shared__ RowPart parts[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = blockIdx.x;
    RowPart mine{-INFINITY, 0.f};
#pragma unroll 4
    for (int r = threadIdx.x; r < a.ranges; r += 1024) mine = joined(mine, a.parts[(long long)r * a.M + m]);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) mine = joined(mine, {__shfl_xor(mine.most, d), __shfl_xor(mine.sum, d)});
    if (lane == 0) parts[wave] = mine;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int w = 1; w < 16; ++w) mine = joined(mine, parts[w]);
        finish_loss(a, m, mine);
    }
}
// Rows up to which each has a workgroup of its own (1024 ranges, 8, 300, 1000 and 2000 rows: 5.3, 7.6, 14.4 and 23.6 us, with 64 rows to a workgroup 26; 40 ranges, 1023
// rows: 7.3 and 4.9).
constexpr int kRowLosses = 1024, kFewRowLosses = 256, kManyRanges = 256;

// ---- backward -----------------------------------------------------------------------------------------------------------
struct SlopeArgs {
    const float *logits;        // [M][stride]
    void *dz;                   // [M][stride], in place where it is float; zeros from `columns` up to the next eighth column
    long long stride;
    int M, columns, first;
    float alpha;
    const int *targets;
    int V;
    const float *logSum, *dloss;
    float *sums;                // [rows / rowsEach][stride]: column sums, or null
    int rowsEach;
    int parts;                  // dz in two parts, the second M rows below
    float *rests;               // [M]: what rounding left of dz at the targets, or null
};
// Rows to a workgroup, and where there would be less than one for each compute unit (40 rows of 5003: 24 us with 32 rows to each, 5.2 with 4).
constexpr int kSlopeRows = 32, kSlopeRowsFew = 4;

// A thread takes four columns of rowsEach rows.
template <class TZ>
__global__ __launch_bounds__(256) void slope_kernel(const SlopeArgs a) {
    const int across = (int)((a.stride + 1023) / 1024);
    const long long tasks = (long long)across * ((a.M + a.rowsEach - 1) / a.rowsEach);
    for (long long task = blockIdx.x; task < tasks; task += gridDim.x) {
        const int n = (int)(task % across) * 1024 + (int)threadIdx.x * 4;
        const long long block = task / across, m0 = block * a.rowsEach;
        if (n >= a.columns && (n & ~7) >= a.columns) continue;      // (nothing of the last eight)
        float sums[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int r = 0; r < a.rowsEach; ++r) {
            const long long m = m0 + r;
            if (m >= a.M) break;
            const float4 q = *reinterpret_cast<const float4 *>(a.logits + m * a.stride + n);
            const float z[4] = {q.x, q.y, q.z, q.w};
            const int t = a.targets[m];
            const bool there = t >= 0 && t < a.V;
            const float slope = a.alpha * (a.dloss ? a.dloss[m] : 1.f), log_sum = a.logSum[m];
            float d[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float p = sizeof(TZ) == 4 ? expf(z[e] - log_sum) : exp_of(z[e] - log_sum);
                d[e] = there && n + e < a.columns ? slope * (t - a.first == n + e ? p - 1.f : p) : 0.f;
                sums[e] += d[e];
                if (a.rests && there && n + e < a.columns && t - a.first == n + e) a.rests[m] = rest_of(d[e]);
            }
            TZ *to = static_cast<TZ *>(a.dz) + m * a.stride + n;
            if constexpr (sizeof(TZ) == 4) *reinterpret_cast<float4 *>(to) = float4{d[0], d[1], d[2], d[3]};
            else *reinterpret_cast<uint2 *>(to) = uint2{to_bf16_pair(d[0], d[1]), to_bf16_pair(d[2], d[3])};
            if (a.parts) *reinterpret_cast<uint2 *>(to + a.M * a.stride) = uint2{to_bf16_pair(rest_of(d[0]), rest_of(d[1])), to_bf16_pair(rest_of(d[2]), rest_of(d[3]))};
        }
        if (a.sums) *reinterpret_cast<float4 *>(a.sums + block * a.stride + n) = float4{sums[0], sums[1], sums[2], sums[3]};
    }
}

struct JoinArgs {
    const float *from, *more;      // packed; more: null, or added
    void *to;
    long long stride;
    int M, C;
    float beta;
};
// The sum over the pieces and over dz's parts into dx.
template <class TO>
__global__ __launch_bounds__(256) void join_kernel(const JoinArgs a) {
    const int groups = (a.C + 3) / 4;
    const long long tasks = (long long)a.M * groups;
    for (long long id = (long long)blockIdx.x * 256 + threadIdx.x; id < tasks; id += (long long)gridDim.x * 256) {
        const long long m = id / groups;
        const int c = (int)(id % groups) * 4;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < a.C) {
                TO *to = static_cast<TO *>(a.to) + m * a.stride + c + e;
                float v = a.from[m * a.C + c + e];
                if (a.more) v += a.more[m * a.C + c + e];
                if (a.beta != 0.f) v += a.beta * Stored<TO>::widen(*to);
                *to = Stored<TO>::narrow(v);
            }
    }
}

struct TwiceArgs {
    const uint16_t *from;
    uint16_t *to;
    long long stride, toRow;
    int M, C;
};
// x once for each part of dz, rows from 16-byte boundaries below each other
__global__ __launch_bounds__(256) void twice_kernel(const TwiceArgs a) {
    const long long tasks = (long long)a.M * a.toRow;
    for (long long id = (long long)blockIdx.x * 256 + threadIdx.x; id < tasks; id += (long long)gridDim.x * 256) {
        const long long m = id / a.toRow, c = id % a.toRow;
        const uint16_t v = c < a.C ? a.from[m * a.stride + c] : (uint16_t)0;
        a.to[id] = v;
        a.to[a.M * a.toRow + id] = v;
    }
}

// ---- what rounding dz leaves at the targets -------------------------------------------------------------------------------
// Nearly all of a row's gradient is its target's, and its rounding would be half of what the results are off by (with their own: 1.41 times theirs).  The rest of it goes
// back in: dx[m] += rest[m] w[t], dw[v] += the sum of rest[m] x[m] over the rows m with target v, which the first of these rows makes.  (Beside the products: 4096 x 4096 -> 65536
// 30 us of 5100, 777 x 1000 -> 10007 16 of 110.)
struct AfterSlopesArgs {
    // the bias gradient
    const float *sums;
    long long stride, blocks;
    float beta;
    float *out;
    int biasGroups;             // workgroups that make it, in front of the others
    // the targets
    const int *targets;
    int M, first, columns;
    int *firstOf, *lastOf;      // [columns]: the first and last row with this target, INT_MAX and -1 without one
};
constexpr int kTargetRange = 512;     // entries to a workgroup, which looks at all rows
// 64 columns of the bias gradient to a workgroup, its four wavefronts on every fourth block of rows; or a range of entries.  (One launch: of 777 rows each is mostly start.)
__global__ __launch_bounds__(256) void after_slopes_kernel(const AfterSlopesArgs a) {
    if ((int)blockIdx.x < a.biasGroups) {
        __shared__ float sums[4][64];
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = (int)blockIdx.x * 64 + lane;
        float sum = 0.f;
        if (n < a.columns)
#pragma unroll 4
            for (long long b = wave; b < a.blocks; b += 4) sum += a.sums[b * a.stride + n];
        sums[wave][lane] = sum;
        __syncthreads();
        if (wave == 0 && n < a.columns) {
            float v = (sums[0][lane] + sums[1][lane]) + (sums[2][lane] + sums[3][lane]);
            if (a.beta != 0.f) v += a.beta * a.out[n];
            a.out[n] = v;
        }
        return;
    }
    __shared__ int first_of[kTargetRange], last_of[kTargetRange];
    const int v0 = ((int)blockIdx.x - a.biasGroups) * kTargetRange;
    for (int i = threadIdx.x; i < kTargetRange; i += 256) first_of[i] = 0x7FFFFFFF, last_of[i] = -1;
    __syncthreads();
#pragma unroll 8
    for (int m = threadIdx.x; m < a.M; m += 256) {
        const uint32_t v = (uint32_t)a.targets[m] - (uint32_t)a.first - (uint32_t)v0;
        if (v >= kTargetRange) continue;
        atomicMin(&first_of[v], m);
        atomicMax(&last_of[v], m);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < kTargetRange && v0 + i < a.columns; i += 256) {
        a.firstOf[v0 + i] = first_of[i];
        a.lastOf[v0 + i] = last_of[i];
    }
}

struct RestRowsArgs {
    const int *targets;
    int M, first, columns, C;
    const int *firstOf, *lastOf;
    const float *rests;
    const uint16_t *x;
    long long stride, toRow;
    uint16_t *to;               // [M][toRow]: of a target's first row
};
constexpr int kRestColumns = 2048, kRestRows = 2048;     // rows looked at at once, eight to a thread
// (4096 x 4096 -> 8000 in all: 671 us with targets at random, 1404 with all of them the same, which one workgroup's rows add four at a time; eight at a time 697 and 1254.)
__global__ __launch_bounds__(256, 5) void rest_rows_kernel(const RestRowsArgs a) {
    __shared__ int list[kRestRows], counts[4];
    __shared__ float sums[256][8];
    // a row by as many threads as it has eighths, rows in turns by the others
    int across = 256;
    while (across > 1 && across / 2 * 8 >= a.toRow) across /= 2;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, turns = 256 / across, turn = (int)threadIdx.x / across;
    const int c = (int)blockIdx.y * kRestColumns + ((int)threadIdx.x % across) * 8;
    for (int m0 = blockIdx.x; m0 < a.M; m0 += (int)gridDim.x) {
        const int t = a.targets[m0];
        const uint32_t v = (uint32_t)t - (uint32_t)a.first;
        if (v >= (uint32_t)a.columns || a.firstOf[v] != m0) continue;
        const int last = a.lastOf[v];
        float sum[8] = {};
        // up to AT_ONCE rows at once, added one after the other (beyond the last: the first again, not added; no branches between the loads)
        auto add = [&](auto at_once, const int *rows, int n) __attribute__((always_inline)) {
            constexpr int AT_ONCE = decltype(at_once)::value;
            Adjacent<uint16_t, 8> q[AT_ONCE];
            float rest[AT_ONCE];
            int m[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) m[k] = rows[k * turns < n ? k * turns : 0];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) rest[k] = a.rests[m[k]];
            if (c + 8 <= a.C)
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k) q[k] = *reinterpret_cast<const Adjacent<uint16_t, 8> *>(a.x + m[k] * a.stride + c);
            else
#pragma unroll
                for (int k = 0; k < AT_ONCE; ++k)
#pragma unroll
                    for (int e = 0; e < 8; ++e) q[k].v[e] = c + e < a.C ? a.x[m[k] * a.stride + c + e] : (uint16_t)0;
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k)
                if (k * turns < n)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[e] += rest[k] * bf16_bits_to_float(q[k].v[e]);
        };
        if (last == m0) {
            if (turn == 0) add(std::integral_constant<int, 1>(), &m0, 1);
        } else {
            for (long long from = m0; from <= last; from += kRestRows) {
                const long long m = from + (int)threadIdx.x * 8;
                uint32_t same = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (m + e <= last && a.targets[m + e] == t) same |= 1u << e;
                int place = __builtin_popcount(same);
#pragma unroll
                for (int d = 1; d < 64; d *= 2) {
                    const int before = __shfl_up(place, d);
                    if (lane >= d) place += before;
                }
                __syncthreads();
                if (lane == 63) counts[wave] = place;
                __syncthreads();
                place -= __builtin_popcount(same);
                for (int w = 0; w < wave; ++w) place += counts[w];
                for (; same; same &= same - 1) list[place++] = (int)m + __builtin_ctz(same);
                const int n = counts[0] + counts[1] + counts[2] + counts[3];
                __syncthreads();
                for (int k = turn; k < n; k += 4 * turns) add(std::integral_constant<int, 4>(), list + k, n - k);
            }
            if (turns > 1) {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < 8; ++e) sums[threadIdx.x][e] = sum[e];
                __syncthreads();
                for (int w = 1; w < turns && turn == 0; ++w)
#pragma unroll
                    for (int e = 0; e < 8; ++e) sum[e] += sums[threadIdx.x + w * across][e];
            }
        }
        if (c >= a.toRow || turn > 0) continue;
        uint16_t *to = a.to + m0 * a.toRow + c;
        *reinterpret_cast<uint4 *>(to) = uint4{to_bf16_pair(sum[0], sum[1]), to_bf16_pair(sum[2], sum[3]), to_bf16_pair(sum[4], sum[5]), to_bf16_pair(sum[6], sum[7])};
    }
}

// ---- host ---------------------------------------------------------------------------------------------------------------
constexpr long long kMostGroups = 1ll << 20;   // workgroups of a launch; more is taken in turns

long long round_up(long long v, long long to) { return (v + to - 1) / to * to; }
bool off(const void *p, size_t to) { return (uintptr_t)p % to != 0; }
unsigned grid_of(long long groups) { return (unsigned)std::min(std::max(groups, 1ll), kMostGroups); }

// The vocabulary in pieces of `size` entries, a multiple of 256 unless it is the whole; `bytes` to an entry of a row.  (Tiles take rows of less than 2^22
// elements.)
constexpr long long kMostEntries = 1ll << 20;
struct Pieces {
    int size, count;
    long long stride;      // of the rows of a piece, elements
};
Pieces pieces_of(long long M, int V, size_t bytes, long long limit = kMostEntries) {
    const long long most = std::min(std::max((long long)(kPieceBytes / bytes) / M / 256 * 256, 256ll), limit);
    Pieces p;
    if (V <= most) {
        p.size = V;
    } else {
        const long long count = (V + most - 1) / most;
        p.size = (int)round_up((V + count - 1) / count, 256);
    }
    p.count = (V + p.size - 1) / p.size;
    p.stride = round_up(p.size, 64);
    return p;
}

struct Room {
    size_t total = 0;
    size_t take(size_t bytes) {
        const size_t at = total;
        total += (bytes + 255) / 256 * 256;
        return at;
    }
};

// Where the operands lie, as far as plans go by it: on 4-byte boundaries (null), x off them, or w, with which x may be.  The queries take the most that any place needs; calls have the room of
// their own place asked of them.
struct Places {
    const void *x = nullptr, *w = nullptr;
};
constexpr uintptr_t kOff = 2;
Places places_of(const void *x, const void *w) {
    const void *off = reinterpret_cast<const void *>(kOff);
    return (uintptr_t)w % 4 != 0 ? Places{off, off} : ((uintptr_t)x % 4 != 0 ? Places{off, nullptr} : Places());
}
// Rows from which on operands off the boundaries are copied for the tiles; fewer have tiles that take them through registers, in the room of those on boundaries.  (w off, x 4096 wide,
// 32768 entries, loss and gradient: 256 rows copied 218 and 626 us, through registers 183 and 542, 1024 rows 382 and 1134, 663 and 1605; 777 x 1000 -> 10007 49 and 129, 71 and 200.)
constexpr int kPlaceRows = 512;
Places copied_places(const Matrix &x, const Places &at) { return x.rows < kPlaceRows ? Places() : at; }

template <class F>
size_t most_of_places(igcDataType t, const Matrix &x, F total) {
    const void *off = reinterpret_cast<const void *>(kOff);
    size_t most = total(Places());
    if (t == IGC_DATA_BFLOAT16) most = std::max(most, total(places_of(off, nullptr)));
    if (t == IGC_DATA_BFLOAT16 && x.rows >= kPlaceRows) most = std::max(most, total(places_of(off, off)));
    return most;
}

// Where w is copied first, it goes by pieces of so many entries: kPieceBytes of copies, less of a w that needs them for its place alone, for which every call's room is asked.
constexpr size_t kPlaceBytes = (size_t)64 << 20;
size_t copied_bytes(igcDataType t, int C) { return t == IGC_DATA_FLOAT || C % 8 != 0 ? kPieceBytes : kPlaceBytes; }
long long copied_entries(igcDataType t, int C) {
    const long long entry = t == IGC_DATA_FLOAT ? round_up(C, 32) * 6 : round_up(C, 8) * 2;
    return std::max((long long)copied_bytes(t, C) / entry / 256 * 256, 256ll);
}

LinearArgs logits_product(const Matrix &x, int C, const Pieces &p, int columns, const Places &at = Places()) {
    LinearArgs a{};
    a.a = at.x;
    a.b = at.w;
    a.am = x.stride; a.ak = 1; a.bn = C; a.bk = 1;
    a.M = (int)x.rows; a.N = columns; a.K = C;
    a.alpha = 1.f;
    a.act = IGC_ACTIVATION_IDENTITY;
    a.ys = p.stride;
    return a;
}

// Logits in memory are written and read once more, at bytes per us, by a second launch.
constexpr double kLogitsBytes = 4.5e6, kLaunch = 3.0;
double through_memory_us(igcHandle_t h, igcDataType t, const Matrix &x, int C, int V, const Pieces &p, double bytes, size_t room, const Places &at) {
    return p.count * (product_us(h, t, IGC_DATA_FLOAT, logits_product(x, C, p, p.size, at), room) + kLaunch) + (double)x.rows * V * bytes / kLogitsBytes;
}
constexpr size_t kNoLimit = ~(size_t)0;
constexpr int kLeastColumns = 128, kLeastRows = 32;     // of a wavefront's or a tile's entry in the statistics and the column sums

// Few enough tokens and vocabulary entries for the kernel of igconv_cross_entropy_few.hip (figures there).
bool few_tokens(igcHandle_t h, igcDataType t, const Matrix &x, int V) { return t == IGC_DATA_BFLOAT16 && x.rows <= kFewTokens && V <= 128 * h->computeUnits; }
// Rows up to which dz is held in two bfloat16 parts, as rows of their own of the matrix that the products take: a tile's 64 rows have room for both.  More rows pay for the second part
// in full (4096 x 4096 -> 65536 8290 us for 5180, 777 x 1000 -> 10007 143 for 112): by the handle's choice; else what is left at the targets is put back instead.
constexpr int kPartsRows = 32;
// Of a few entries' gradients what is left at the targets is a long sum for each entry, which one workgroup makes in order (a row of 1024 features 0.1 us, of 4096 0.2): with both parts
// of dz there is none, for about 24 bytes a feature of x (16384 x 1024 -> 2, 8, 16 and 32 rounded 903, 294, 195 and 142 us, in two parts 145, 158, 158 and 154; 16384 x 4096 -> 4, 8 and 16
// 1030, 626 and 425 us, in two parts 632 each; 2048 x 1024 -> 2 134 and 58).  Up to kFewEntriesFeatures of x: the parts of dx and x take 12 bytes each of room.
constexpr int kFewEntriesRows = 512;
constexpr long long kFewEntriesFeatures = 1ll << 26;
bool few_entries(const Matrix &x, int C, int V) { return x.rows >= kFewEntriesRows && x.rows * C <= kFewEntriesFeatures && (long long)V * std::max(C, 2048) <= 16 * 2048; }
bool in_parts(igcHandle_t h, igcDataType t, const Matrix &x, int C, int V) {
    return t == IGC_DATA_BFLOAT16 && (x.rows <= kPartsRows || h->crossEntropySlopes == IGC_DATA_FLOAT || few_entries(x, C, V));
}
struct ForwardPlan {
    bool few, whole;     // few tokens; else whether the tiles leave the statistics, no logits in memory
    Pieces pieces;
    int ranges;          // of all columns
    size_t logits, parts, picked, room, total, room_bytes;
};
ForwardPlan plan_forward(igcHandle_t h, igcDataType t, const Matrix &x, int C, int V, const Places &places) {
    const Places at = copied_places(x, places);
    ForwardPlan p;
    p.pieces = pieces_of(x.rows, V, 4);
    p.few = few_tokens(h, t, x, V);
    if (p.few) {
        p.whole = true;
        p.pieces = Pieces{V, 1, 0};
        p.ranges = (V + cross_few_columns(h, V) - 1) / cross_few_columns(h, V);
        p.logits = p.room = p.room_bytes = 0;
        Room r;
        p.parts = r.take((size_t)x.rows * p.ranges * sizeof(RowPart));
        p.picked = r.take((size_t)x.rows * 4);
        p.total = r.total;
        return p;
    }
    // (the last piece may be smaller, and then take other tiles)
    auto most_room = [&](const Pieces &q, auto room) {
        return q.count > 1 ? std::max(room(logits_product(x, C, q, q.size, at)), room(logits_product(x, C, q, V - (q.count - 1) * q.size, at))) : room(logits_product(x, C, q, V, at));
    };
    auto cross = [&](int columns) { return plan_cross_product(h, kRowStatistics, t, logits_product(x, C, p.pieces, columns, at), kNoLimit); };
    auto in_memory = [&](const LinearArgs &a) { return product_room(h, t, IGC_DATA_FLOAT, a); };
    Pieces whole{V, 1, 0};
    CrossPlan all = cross(V);
    if (all.us < 0.0 || all.copiesB) whole = pieces_of(1, V, 4, copied_entries(t, C));
    if (all.us < 0.0) {
        all = cross(whole.size);
        all.us *= whole.count;
    }
    p.room_bytes = most_room(p.pieces, in_memory);
    p.whole = all.us >= 0.0 && all.us <= through_memory_us(h, t, x, C, V, p.pieces, 8.0, p.room_bytes, at);
    if (p.whole) {
        p.pieces = whole;
        p.room_bytes = most_room(whole, [&](const LinearArgs &a) { return plan_cross_product(h, kRowStatistics, t, a, kNoLimit).room; });
    } else if ((t == IGC_DATA_FLOAT || C % 8 != 0 || at.w) && p.room_bytes > copied_bytes(t, C)) {
        p.pieces = pieces_of(x.rows, V, 4, copied_entries(t, C));
        p.room_bytes = most_room(p.pieces, in_memory);
    }
    p.ranges = p.whole ? (V + kLeastColumns - 1) / kLeastColumns : (p.pieces.size + kRange - 1) / kRange * p.pieces.count;
    Room r;
    p.logits = r.take(p.whole ? 0 : (size_t)x.rows * p.pieces.stride * 4);
    p.parts = r.take((size_t)x.rows * p.ranges * sizeof(RowPart));
    p.picked = r.take((size_t)x.rows * 4);
    p.room = r.take(p.room_bytes);
    p.total = r.total;
    return p;
}

LinearArgs data_product(long long rows, int C, const Pieces &p, int columns, const Places &at) {
    LinearArgs a{};
    a.b = at.w;
    a.am = p.stride; a.ak = 1; a.bn = 1; a.bk = C; a.strided_b = true; a.padded_a = true;
    a.M = (int)rows; a.N = C; a.K = columns;
    a.alpha = 1.f;
    a.act = IGC_ACTIVATION_IDENTITY;
    return a;
}
// (parts: x as it was copied, once for each part of dz)
LinearArgs filter_product(const Matrix &x, bool parts, int C, const Pieces &p, int columns, const Places &at) {
    LinearArgs a{};
    a.b = parts ? nullptr : at.x;
    a.am = 1; a.ak = p.stride; a.bn = 1; a.bk = parts ? round_up(C, 8) : x.stride; a.padded_b = parts; a.strided_a = a.strided_b = true; a.padded_a = true;
    a.M = columns; a.N = C; a.K = (int)(parts ? 2 * x.rows : x.rows);
    a.alpha = 1.f;
    a.act = IGC_ACTIVATION_IDENTITY;
    return a;
}
struct BackwardPlan {
    bool few, direct;    // few tokens; else whether the tiles leave dz, no logits in memory
    bool parts;          // dz is in two parts
    Pieces pieces;
    bool sum;            // dx is summed in floats first
    bool rests;          // what rounding dz leaves at the targets goes back in
    long long rows;      // of dz: its parts'
    int slopeRows;       // rows to a workgroup of slope_kernel
    size_t logits, dz, dx, x, sums, restsAt, firstOf, lastOf, restRows, room, total, room_bytes;
};
// dx, dw: null where that gradient is not asked for
BackwardPlan plan_backward(igcHandle_t h, igcDataType t, igcTensorDescriptor_t dx, igcFilterDescriptor_t dw, const Matrix &x, int C, int V, const Places &places) {
    const Places at = copied_places(x, places);
    BackwardPlan p;
    const size_t elem = t == IGC_DATA_FLOAT ? 4 : 2;
    p.few = few_tokens(h, t, x, V);
    p.parts = in_parts(h, t, x, C, V);
    p.rows = p.parts ? 2 * x.rows : x.rows;
    auto in_pieces = [&](long long limit) {
        p.pieces = pieces_of(p.rows, V, elem, limit);
        p.direct = p.few;
        if (p.few) return;
        const CrossPlan cross = plan_cross_product(h, kSlopes, t, logits_product(x, C, p.pieces, p.pieces.size, at), kNoLimit);
        const Pieces wide = pieces_of(p.rows, V, 4, limit);
        p.direct = cross.us >= 0.0 && cross.us * p.pieces.count <= through_memory_us(h, t, x, C, V, wide, 8.0 + elem, kNoLimit, at);
        if (!p.direct) p.pieces = wide;
    };
    in_pieces(kMostEntries);
    // (w copied for its place alone: in smaller pieces)
    if (at.w && C % 8 == 0 && p.pieces.size > copied_entries(t, C) &&
        (plan_cross_product(h, kSlopes, t, logits_product(x, C, p.pieces, p.pieces.size, at), kNoLimit).copiesB ||
         plan_cross_product(h, kDataWithRows, t, data_product(p.rows, C, p.pieces, p.pieces.size, at), kNoLimit).copiesB))
        in_pieces(copied_entries(t, C));
    p.sum = dx && (p.parts || (p.pieces.count > 1 && dx->dtype == IGC_DATA_BFLOAT16));
    Room r;
    p.dz = r.take((size_t)p.rows * p.pieces.stride * elem);
    p.logits = p.direct || elem == 4 ? p.dz : r.take((size_t)x.rows * p.pieces.stride * 4);
    p.dx = r.take(p.sum ? (size_t)p.rows * C * 4 : 0);
    p.x = r.take(p.parts && dw ? (size_t)p.rows * round_up(C, 8) * 2 : 0);
    p.slopeRows = (p.pieces.stride + 1023) / 1024 * ((x.rows + kSlopeRows - 1) / kSlopeRows) < h->computeUnits ? kSlopeRowsFew : kSlopeRows;
    p.sums = r.take((size_t)std::max((x.rows + 255) / 256 * 256 / kLeastRows, p.direct ? 0ll : (x.rows + p.slopeRows - 1) / p.slopeRows) * p.pieces.stride * 4);
    p.rests = t == IGC_DATA_BFLOAT16 && !p.parts && (dx || dw);
    p.restsAt = r.take(p.rests ? (size_t)x.rows * 4 : 0);
    p.firstOf = r.take(p.rests && dw ? (size_t)p.pieces.size * 4 : 0);
    p.lastOf = r.take(p.rests && dw ? (size_t)p.pieces.size * 4 : 0);
    p.restRows = r.take(p.rests && dw ? (size_t)x.rows * round_up(C, 8) * 2 : 0);
    p.room_bytes = 0;
    for (int piece : {0, p.pieces.count - 1}) {
        // (the last piece may be smaller, and then take other tiles)
        const int columns = std::min(p.pieces.size, V - piece * p.pieces.size);
        const LinearArgs logits = logits_product(x, C, p.pieces, columns, at);
        if (!p.few) p.room_bytes = std::max(p.room_bytes, p.direct ? plan_cross_product(h, kSlopes, t, logits, kNoLimit).room : product_room(h, t, IGC_DATA_FLOAT, logits));
        auto room_of = [&](CrossKind kind, igcDataType out, const LinearArgs &a) {
            p.room_bytes = std::max(p.room_bytes, p.rests ? product_with_rows_room(h, kind, out, a) : product_room(h, t, out, a));
        };
        if (dx) room_of(kDataWithRows, p.sum ? IGC_DATA_FLOAT : dx->dtype, data_product(p.rows, C, p.pieces, columns, at));
        if (dw) room_of(kFilterWithRows, dw->dtype, filter_product(x, p.parts, C, p.pieces, columns, places));      // (x off a boundary: copied, else it would go element by element)
        if (p.pieces.count == 1) break;
    }
    p.room = r.take(p.room_bytes);
    p.total = r.total;
    return p;
}

igcStatus check_sizes(igcTensorDescriptor_t x, igcFilterDescriptor_t w, Matrix *mx) {
    if (!x || !w) return IGC_STATUS_BAD_PARAM;
    if (!x->set || !w->set) return IGC_STATUS_NOT_INITIALIZED;
    if (w->r != 1 || w->s != 1 || x->dim[1] != w->c) return IGC_STATUS_BAD_PARAM;
    if ((x->dtype != IGC_DATA_FLOAT && x->dtype != IGC_DATA_BFLOAT16) || w->dtype != x->dtype || !matrix_of(*x, mx) || w->k > kMostColumns) return IGC_STATUS_NOT_SUPPORTED;
    return IGC_STATUS_SUCCESS;
}
// (two parts: their rows are counted as a product's)
igcStatus check_rows(igcHandle_t h, igcDataType t, const Matrix &x) { return t == IGC_DATA_BFLOAT16 && h->crossEntropySlopes == IGC_DATA_FLOAT && x.rows > kMostRows / 2 ? IGC_STATUS_NOT_SUPPORTED : IGC_STATUS_SUCCESS; }
igcStatus check_gradients(igcTensorDescriptor_t x, igcFilterDescriptor_t w, igcTensorDescriptor_t dx, igcFilterDescriptor_t dw, Matrix *mdx) {
    const auto type = [&](igcDataType t) { return t == IGC_DATA_FLOAT || (t == IGC_DATA_BFLOAT16 && x->dtype == IGC_DATA_BFLOAT16); };
    if ((dx && !dx->set) || (dw && !dw->set)) return IGC_STATUS_NOT_INITIALIZED;
    if (dx && (!same_positions(*x, *dx) || dx->dim[1] != x->dim[1] || !non_aliasing(dx->dim, dx->stride))) return IGC_STATUS_BAD_PARAM;
    if (dw && (dw->k != w->k || dw->c != w->c || dw->r != 1 || dw->s != 1)) return IGC_STATUS_BAD_PARAM;
    if ((dx && (!type(dx->dtype) || !matrix_of(*dx, mdx))) || (dw && !type(dw->dtype))) return IGC_STATUS_NOT_SUPPORTED;
    return IGC_STATUS_SUCCESS;
}

}  // namespace
}  // namespace igc

using namespace igc;

extern "C" {

igcStatus igcGetLinearCrossEntropyForwardWorkspaceSize(igcHandle_t handle, igcTensorDescriptor_t xDesc, igcFilterDescriptor_t wDesc, size_t *sizeInBytes) {
    if (!handle || !sizeInBytes) return IGC_STATUS_BAD_PARAM;
    Matrix x;
    const igcStatus st = check_sizes(xDesc, wDesc, &x);
    if (st != IGC_STATUS_SUCCESS) return st;
    *sizeInBytes = most_of_places(xDesc->dtype, x, [&](const Places &at) { return plan_forward(handle, xDesc->dtype, x, wDesc->c, wDesc->k, at).total; });
    return IGC_STATUS_SUCCESS;
}

igcStatus igcLinearCrossEntropyForward(igcHandle_t handle, igcTensorDescriptor_t xDesc, const void *x, igcFilterDescriptor_t wDesc, const void *w, const void *bias,
                                       const int *targets, void *workSpace, size_t workSpaceSizeInBytes, void *loss, void *logSum) {
    if (!handle || !x || !w || !targets || !loss || !workSpace) return IGC_STATUS_BAD_PARAM;
    Matrix mx;
    igcStatus st = check_sizes(xDesc, wDesc, &mx);
    if (st != IGC_STATUS_SUCCESS) return st;
    const igcDataType t = xDesc->dtype;
    if (off(x, elem_size(t)) || off(w, elem_size(t)) || off(bias, 4) || off(targets, 4) || off(loss, 4) || off(logSum, 4) || off(workSpace, 16)) return IGC_STATUS_BAD_PARAM;
    const int C = wDesc->c, V = wDesc->k, M = (int)mx.rows;
    const ForwardPlan p = plan_forward(handle, t, mx, C, V, places_of(x, w));
    if (workSpaceSizeInBytes < p.total) return IGC_STATUS_BAD_PARAM;
    uint8_t *ws = static_cast<uint8_t *>(workSpace);
    RowPart *parts = reinterpret_cast<RowPart *>(ws + p.parts);
    float *picked = reinterpret_cast<float *>(ws + p.picked);
    int ranges = 0;
    for (int first = 0; first < V; first += p.pieces.size) {
        const int columns = std::min(p.pieces.size, V - first);
        LinearArgs a = logits_product(mx, C, p.pieces, columns);
        a.a = x;
        a.b = static_cast<const uint8_t *>(w) + (size_t)first * C * elem_size(t);
        a.bias = bias ? static_cast<const float *>(bias) + first : nullptr;
        if (p.whole) {
            CrossEnd end{};
            end.targets = targets;
            end.first = first;
            end.V = V;
            end.parts = parts + (long long)ranges * M;
            end.picked = picked;
            CrossPlan taken;
            taken.tileColumns = cross_few_columns(handle, V);
            st = p.few ? cross_few(handle, kRowStatistics, a, end) : cross_product(handle, kRowStatistics, t, a, end, ws + p.room, p.room_bytes, &taken);
            if (st != IGC_STATUS_SUCCESS) return st;
            ranges += (columns + taken.tileColumns - 1) / taken.tileColumns;
            continue;
        }
        a.y = ws + p.logits;
        if ((st = product(handle, t, IGC_DATA_FLOAT, a, ws + p.room, p.room_bytes)) != IGC_STATUS_SUCCESS) return st;
        const int here = (columns + kRange - 1) / kRange;
        RowPartsArgs q{reinterpret_cast<const float *>(ws + p.logits), p.pieces.stride, M, columns, here, first, targets, parts + (long long)ranges * M, picked};
        st = launch_kernel(reinterpret_cast<const void *>(&row_parts_kernel), q, dim3(grid_of(((long long)M * here + 3) / 4)), 256, handle->stream);
        if (st != IGC_STATUS_SUCCESS) return st;
        ranges += here;
    }
    LossArgs q{parts, M, V, ranges, targets, picked, static_cast<float *>(loss), static_cast<float *>(logSum)};
    if (M <= kRowLosses && (M <= kFewRowLosses || ranges >= kManyRanges)) return launch_kernel(reinterpret_cast<const void *>(&loss_row_kernel), q, dim3((unsigned)M), 1024, handle->stream);
    return launch_kernel(reinterpret_cast<const void *>(&loss_kernel), q, dim3(grid_of((M + 63) / 64)), 1024, handle->stream);
}

igcStatus igcSetCrossEntropySlopes(igcHandle_t handle, igcDataType type) {
    if (!handle || (type != IGC_DATA_BFLOAT16 && type != IGC_DATA_FLOAT)) return IGC_STATUS_BAD_PARAM;
    handle->crossEntropySlopes = type;
    return IGC_STATUS_SUCCESS;
}

igcStatus igcGetCrossEntropySlopes(igcHandle_t handle, igcDataType *type) {
    if (!handle || !type) return IGC_STATUS_BAD_PARAM;
    *type = handle->crossEntropySlopes;
    return IGC_STATUS_SUCCESS;
}

igcStatus igcGetLinearCrossEntropyBackwardWorkspaceSize(igcHandle_t handle, igcTensorDescriptor_t xDesc, igcFilterDescriptor_t wDesc, igcTensorDescriptor_t dxDesc,
                                                        igcFilterDescriptor_t dwDesc, size_t *sizeInBytes) {
    if (!handle || !sizeInBytes) return IGC_STATUS_BAD_PARAM;
    Matrix x, dx;
    igcStatus st = check_sizes(xDesc, wDesc, &x);
    if (st != IGC_STATUS_SUCCESS || (st = check_gradients(xDesc, wDesc, dxDesc, dwDesc, &dx)) != IGC_STATUS_SUCCESS ||
        (st = check_rows(handle, xDesc->dtype, x)) != IGC_STATUS_SUCCESS)
        return st;
    *sizeInBytes = most_of_places(xDesc->dtype, x, [&](const Places &at) { return plan_backward(handle, xDesc->dtype, dxDesc, dwDesc, x, wDesc->c, wDesc->k, at).total; });
    return IGC_STATUS_SUCCESS;
}

igcStatus igcLinearCrossEntropyBackward(igcHandle_t handle, const void *alpha, igcTensorDescriptor_t xDesc, const void *x, igcFilterDescriptor_t wDesc, const void *w,
                                        const void *bias, const int *targets, const void *logSum, const void *dloss, void *workSpace, size_t workSpaceSizeInBytes,
                                        const void *beta, igcTensorDescriptor_t dxDesc, void *dx, const void *paramBeta, igcFilterDescriptor_t dwDesc, void *dw, void *dbias) {
    if (!dx) dxDesc = nullptr;
    if (!dw) dwDesc = nullptr;
    if (!handle || !alpha || !beta || !paramBeta || !x || !w || !targets || !logSum || !workSpace || (!dx && !dw && !dbias) || (dx && !dxDesc) || (dw && !dwDesc)) return IGC_STATUS_BAD_PARAM;
    Matrix mx, mdx;
    igcStatus st = check_sizes(xDesc, wDesc, &mx);
    if (st != IGC_STATUS_SUCCESS || (st = check_gradients(xDesc, wDesc, dxDesc, dwDesc, &mdx)) != IGC_STATUS_SUCCESS ||
        (st = check_rows(handle, xDesc->dtype, mx)) != IGC_STATUS_SUCCESS)
        return st;
    const igcDataType t = xDesc->dtype;
    if (off(x, elem_size(t)) || off(w, elem_size(t)) || off(bias, 4) || off(targets, 4) || off(logSum, 4) || off(dloss, 4) || off(workSpace, 16) ||
        (dx && off(dx, elem_size(dxDesc->dtype))) || (dw && off(dw, elem_size(dwDesc->dtype))) || off(dbias, 4))
        return IGC_STATUS_BAD_PARAM;
    const int C = wDesc->c, V = wDesc->k, M = (int)mx.rows;
    const Places at = places_of(x, w);
    const BackwardPlan p = plan_backward(handle, t, dxDesc, dwDesc, mx, C, V, at);
    if (workSpaceSizeInBytes < p.total) return IGC_STATUS_BAD_PARAM;
    const float dx_beta = *static_cast<const float *>(beta), w_beta = *static_cast<const float *>(paramBeta);
    uint8_t *ws = static_cast<uint8_t *>(workSpace);
    const long long row_blocks = (M + p.slopeRows - 1) / p.slopeRows;
    float *rests = p.rests ? reinterpret_cast<float *>(ws + p.restsAt) : nullptr;
    if (p.parts && !p.few && dw) {
        TwiceArgs q{static_cast<const uint16_t *>(x), reinterpret_cast<uint16_t *>(ws + p.x), mx.stride, round_up(C, 8), M, C};
        st = launch_kernel(reinterpret_cast<const void *>(&twice_kernel), q, dim3(grid_of((M * q.toRow + 255) / 256)), 256, handle->stream);
        if (st != IGC_STATUS_SUCCESS) return st;
    }
    for (int first = 0; first < V; first += p.pieces.size) {
        const int columns = std::min(p.pieces.size, V - first);
        const void *piece = static_cast<const uint8_t *>(w) + (size_t)first * C * elem_size(t);
        LinearArgs a = logits_product(mx, C, p.pieces, columns);
        a.a = x;
        a.b = piece;
        a.bias = bias ? static_cast<const float *>(bias) + first : nullptr;
        float *sums = dbias ? reinterpret_cast<float *>(ws + p.sums) : nullptr;
        long long sum_blocks = row_blocks;
        if (p.direct) {
            a.y = ws + p.dz;
            CrossEnd end{};
            end.targets = targets;
            end.first = first;
            end.V = V;
            end.alpha = *static_cast<const float *>(alpha);
            end.logSum = static_cast<const float *>(logSum);
            end.dloss = static_cast<const float *>(dloss);
            end.sums = sums;
            end.sumStride = p.pieces.stride;
            end.twoParts = p.parts;
            end.rests = rests;
            CrossPlan taken;
            taken.sumBlocks = 1;
            if (p.few) {
                a.z = dw && first == 0 ? ws + p.x : nullptr;
                a.zs = round_up(C, 8);
                st = cross_few(handle, kSlopes, a, end);
            } else {
                st = cross_product(handle, kSlopes, t, a, end, ws + p.room, p.room_bytes, &taken);
            }
            if (st != IGC_STATUS_SUCCESS) return st;
            sum_blocks = taken.sumBlocks;
        } else {
            a.y = ws + p.logits;
            if ((st = product(handle, t, IGC_DATA_FLOAT, a, ws + p.room, p.room_bytes)) != IGC_STATUS_SUCCESS) return st;
            SlopeArgs q{reinterpret_cast<const float *>(ws + p.logits), ws + p.dz, p.pieces.stride, M, columns, first, *static_cast<const float *>(alpha), targets, V,
                        static_cast<const float *>(logSum), static_cast<const float *>(dloss), sums, p.slopeRows, p.parts ? 1 : 0, rests};
            st = launch_kernel(t == IGC_DATA_FLOAT ? reinterpret_cast<const void *>(&slope_kernel<float>) : reinterpret_cast<const void *>(&slope_kernel<bf16_t>), q,
                               dim3(grid_of((p.pieces.stride + 1023) / 1024 * row_blocks)), 256, handle->stream);
            if (st != IGC_STATUS_SUCCESS) return st;
        }
        int *first_of = reinterpret_cast<int *>(ws + p.firstOf), *last_of = reinterpret_cast<int *>(ws + p.lastOf);
        if (dbias || (dw && p.rests)) {
            AfterSlopesArgs b{sums, p.pieces.stride, sum_blocks, w_beta, dbias ? static_cast<float *>(dbias) + first : nullptr, dbias ? (columns + 63) / 64 : 0,
                              targets, M, first, columns, first_of, last_of};
            const int ranges = dw && p.rests ? (columns + kTargetRange - 1) / kTargetRange : 0;
            st = launch_kernel(reinterpret_cast<const void *>(&after_slopes_kernel), b, dim3((unsigned)(b.biasGroups + ranges)), 256, handle->stream);
            if (st != IGC_STATUS_SUCCESS) return st;
        }
        if (dx) {
            LinearArgs d = data_product(p.rows, C, p.pieces, columns, at);
            d.a = ws + p.dz;
            d.b = piece;
            d.y = p.sum ? ws + p.dx : dx;
            d.ys = p.sum ? C : mdx.stride;
            d.r = d.y;
            d.rs = d.ys;
            d.beta = first > 0 ? 1.f : (p.sum ? 0.f : dx_beta);
            const igcDataType out = p.sum ? IGC_DATA_FLOAT : dxDesc->dtype;
            const RowAddend add{targets, rests, static_cast<const uint16_t *>(piece), C, first, columns};
            st = p.rests ? product_with_rows(handle, kDataWithRows, out, d, add, ws + p.room, p.room_bytes) : product(handle, t, out, d, ws + p.room, p.room_bytes);
            if (st != IGC_STATUS_SUCCESS) return st;
        }
        if (dw) {
            LinearArgs f = filter_product(mx, p.parts, C, p.pieces, columns, at);
            f.a = ws + p.dz;
            f.b = p.parts ? ws + p.x : x;
            f.y = static_cast<uint8_t *>(dw) + (size_t)first * C * elem_size(dwDesc->dtype);
            f.ys = C;
            f.r = f.y;
            f.rs = C;
            f.beta = w_beta;
            if (!p.rests) {
                if ((st = product(handle, t, dwDesc->dtype, f, ws + p.room, p.room_bytes)) != IGC_STATUS_SUCCESS) return st;
                continue;
            }
            uint16_t *rest_rows = reinterpret_cast<uint16_t *>(ws + p.restRows);
            const RestRowsArgs s{targets, M, first, columns, C, first_of, last_of, rests, static_cast<const uint16_t *>(x), mx.stride, round_up(C, 8), rest_rows};
            const long long across = (C + kRestColumns - 1) / kRestColumns;
            st = launch_kernel(reinterpret_cast<const void *>(&rest_rows_kernel), s, dim3((unsigned)std::min<long long>(M, std::max(kMostGroups / across, 1ll)), (unsigned)across), 256, handle->stream);
            if (st != IGC_STATUS_SUCCESS) return st;
            const RowAddend add{first_of, nullptr, rest_rows, s.toRow, 0, M};
            if ((st = product_with_rows(handle, kFilterWithRows, dwDesc->dtype, f, add, ws + p.room, p.room_bytes)) != IGC_STATUS_SUCCESS) return st;
        }
    }
    if (dx && p.sum) {
        const float *from = reinterpret_cast<const float *>(ws + p.dx);
        JoinArgs j{from, p.parts ? from + (long long)M * C : nullptr, dx, mdx.stride, M, C, dx_beta};
        return launch_kernel(dxDesc->dtype == IGC_DATA_FLOAT ? reinterpret_cast<const void *>(&join_kernel<float>) : reinterpret_cast<const void *>(&join_kernel<bf16_t>), j,
                             dim3(grid_of(((long long)M * ((C + 3) / 4) + 255) / 256)), 256, handle->stream);
    }
    return IGC_STATUS_SUCCESS;
}

}  // extern "C"
