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
#include <type_traits>

#include "igconv_rows.h"

namespace igc {
namespace {

template <class W>
struct NormArgs {
    const void *x, *scale, *shift;
    void *y;
    W *mean, *invstd;
    long long xs, ys;   // elements between rows
    int M, C;
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

// sum over a workgroup of 256 threads, given to all; `slots`: four entries that nothing else uses until the next barrier
template <class W>
__device__ __forceinline__ W group_sum(W v, W *slots) {
    v = lanes_sum<64>(v);
    if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = v;
    __syncthreads();
    return (slots[0] + slots[1]) + (slots[2] + slots[3]);
}

// ---- any row length: a workgroup per row at a time, the row read once per pass ------------------------------------------
constexpr int kMostRowGroups = 1 << 20;   // (workgroups times threads is a 32-bit number)
template <class TX, class TY>
__global__ __launch_bounds__(256) void layer_norm_rows_kernel(const NormArgs<typename Stored<TX>::wide_t> a) {
    typedef typename Stored<TX>::wide_t W;
    __shared__ W slots[8];
    for (int i = blockIdx.x; i < a.M; i += (int)gridDim.x) {
        const TX *x = static_cast<const TX *>(a.x) + i * a.xs;
        TY *y = static_cast<TY *>(a.y) + i * a.ys;
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
            if (a.mean) a.mean[i] = mean;
            if (a.invstd) a.invstd[i] = s;
        }
    }
}

template <class TX, class TY>
__global__ __launch_bounds__(256) void layer_norm_backward_rows_kernel(const NormBackwardArgs<typename Stored<TX>::wide_t> a) {
    typedef typename Stored<TX>::wide_t W;
    __shared__ W slots[8];
    for (int i = blockIdx.x; i < a.M; i += (int)gridDim.x) {
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

// Adds the ranges' sums in order; without ranges takes the sums over all rows itself: lanes along 32 feature maps, 32 rows at a time (a range per
// line and round: with eight lines the 188 ranges of 3001 x 777 were six rounds of waits, 14.2 us in all, so 13.7).
template <class TX, class TY>
__global__ __launch_bounds__(1024) void layer_norm_params_sum_kernel(const NormBackwardArgs<typename Stored<TX>::wide_t> a) {
    typedef typename Stored<TX>::wide_t W;
    constexpr int LINES = 32;
    __shared__ W sums[2][LINES][32];
    const int lane = threadIdx.x & 31, line = threadIdx.x >> 5, c = (int)blockIdx.x * 32 + lane;
    W scale = W(0), shift = W(0);
    if (c < a.C) {
        if (a.parts) {
#pragma unroll 4
            for (int r = line; r < a.ranges; r += LINES) {
                scale += a.parts[(size_t)r * 2 * a.C + c];
                shift += a.parts[((size_t)r * 2 + 1) * a.C + c];
            }
        } else {
            for (int i = line; i < a.M; i += LINES) {
                const W dy = Stored<TY>::widen(static_cast<const TY *>(a.dy)[i * a.dys + c]);
                const W h = (Stored<TX>::widen(static_cast<const TX *>(a.x)[i * a.xs + c]) - a.mean[i]) * a.invstd[i];
                shift += dy;
                scale += dy * h;
            }
        }
    }
    sums[0][line][lane] = scale;
    sums[1][line][lane] = shift;
    __syncthreads();
    W *out = line == 0 ? a.dscale : a.dshift;
    if (line < 2 && c < a.C && out) {
        W v = W(0);
#pragma unroll
        for (int i = 0; i < LINES; ++i) v += sums[line][i][lane];
        v *= a.alpha;
        if (a.paramBeta != W(0)) v += a.paramBeta * out[c];
        out[c] = v;
    }
}

// ---- rows that fit into registers ---------------------------------------------------------------------------------------
// LANES threads (a wavefront or a workgroup) share a row: thread t holds the chunks t, t + LANES, ... of E neighbours, CHUNKS of them at
// most, so that a row is read once and its deviations are taken in registers.  Workgroups walk down the rows (every gridDim-th group
// of rows), the loads of the next row under way while the present one is summed; scale and shift stay in registers as well.
// WHOLE: C is a number of whole chunks.  Else the last chunk is moved back to end with the row; the elements it shares with the chunk
// before (`skip` of them) are computed, and stored, twice, but counted once.  (Tested and moved element by element that chunk cost as much
// as the rest of the row: 40000 x 1001 float forward 89 us, 40000 x 1000 61.  Rows off 16-byte boundaries cost next to nothing.)
//
// Bound by memory, each element being read once and written once; a copy of 2 GiB reaches 4.9 TB/s here (what lies in the last-level cache is faster).
// Forward: 16384 x 4096 float into bfloat16 74 us, 5.5 TB/s; 8192 x 8192 bfloat16 42 us, 6.4; 5003 x 1001 float 8.8 us, 4.6; 2048 x 32768 float
// 117 us, 4.6 (one row at a time per compute unit); 4 x 4096 3 us, the latency of two trips to memory and two barriers.  Gradient with dscale, dshift
// and r: 8192 x 8192 bfloat16 104 us, 5.2 TB/s; 65536 x 512 47 us, 5.8; 4096 x 16384 float 222 us, 4.8; 3001 x 777 float without r 13.6 us, 10 of
// them this kernel and 4 the sum over the workgroups.  A wavefront, or part of one, per row as far as its registers go: there are no barriers then;
// more threads beyond, so that two workgroups share a compute unit and one loads while the other sums.
template <class T> constexpr int kChunk = sizeof(T) == 8 ? 4 : 8;

// E neighbours as they are stored; rows need not begin on 16-byte boundaries (the wide loads of this machine do not ask for it)
template <class T, int E>
struct __attribute__((packed, aligned(sizeof(T)))) Chunk {
    T v[E];
};
template <class T, int E>
__device__ __forceinline__ void load_chunk(Chunk<T, E> &r, const T *p) {
    r = *reinterpret_cast<const Chunk<T, E> *>(p);
}
template <class T, class W, int E>
__device__ __forceinline__ void store_chunk(T *p, const W (&v)[E]) {
    Chunk<T, E> r;
    if constexpr (sizeof(T) == 2) {
        uint32_t pair[E / 2];
#pragma unroll
        for (int e = 0; e < E / 2; ++e) pair[e] = to_bf16_pair(v[2 * e], v[2 * e + 1]);
        __builtin_memcpy(&r, pair, sizeof(r));
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e) r.v[e] = v[e];
    }
    *reinterpret_cast<Chunk<T, E> *>(p) = r;
}

// The chunk has arrived from here on.  (A row may be written in place, and a chunk that was moved back shares elements with another thread's: all of a
// row is read before the barrier after which any of it is written.)
template <class T, int E>
__device__ __forceinline__ void arrive(Chunk<T, E> &r) {
    uint32_t words[sizeof(r) / 4];
    __builtin_memcpy(words, &r, sizeof(r));
#pragma unroll
    for (int i = 0; i < (int)(sizeof(r) / 4); ++i) asm volatile("" : "+v"(words[i]));
    __builtin_memcpy(&r, words, sizeof(r));
}

// where a thread's chunks begin
template <int LANES, int CHUNKS, int E, bool WHOLE>
struct Place {
    int c[CHUNKS], skip_[CHUNKS];
    bool live[CHUNKS];
    __device__ __forceinline__ Place(int t, int C) {
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            const int at = (t + j * LANES) * E;
            live[j] = at < C;
            c[j] = WHOLE ? at : min(at, C - E);
            skip_[j] = at - c[j];
        }
    }
    __device__ __forceinline__ int skip(int j) const { return WHOLE ? 0 : skip_[j]; }
    __device__ __forceinline__ bool counts(int j, int e) const { return WHOLE || e >= skip_[j]; }
};

// the sum over the LANES threads of a row; `slots`: LANES / 64 entries that nothing else uses until the next barrier but one
template <int LANES, class W>
__device__ __forceinline__ W row_sum(W a, W *slots) {
    a = lanes_sum<(LANES < 64 ? LANES : 64)>(a);
    if constexpr (LANES > 64) {
        if ((threadIdx.x & 63) == 0) slots[threadIdx.x >> 6] = a;
        __syncthreads();
        a = W(0);
#pragma unroll
        for (int i = 0; i < LANES / 64; ++i) a += slots[i];
    }
    return a;
}
template <int LANES, class W>
__device__ __forceinline__ void row_sums(W &a, W &b, W *slots) {   // (two at once: twice the entries, one barrier)
    a = lanes_sum<(LANES < 64 ? LANES : 64)>(a);
    b = lanes_sum<(LANES < 64 ? LANES : 64)>(b);
    if constexpr (LANES > 64) {
        constexpr int N = LANES / 64;
        if ((threadIdx.x & 63) == 0) {
            slots[threadIdx.x >> 6] = a;
            slots[N + (threadIdx.x >> 6)] = b;
        }
        __syncthreads();
        a = b = W(0);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            a += slots[i];
            b += slots[N + i];
        }
    }
}

constexpr int norm_threads(int lanes) { return lanes < 256 ? 256 : lanes; }

template <class TX, class TY, int LANES, int CHUNKS, bool WHOLE>
__global__ __launch_bounds__(norm_threads(LANES)) void layer_norm_held_kernel(const NormArgs<typename Stored<TX>::wide_t> a) {
    typedef typename Stored<TX>::wide_t W;
    constexpr int E = kChunk<TX>, ROWS = norm_threads(LANES) / LANES;
    __shared__ W slots[2][2][norm_threads(LANES) / 64];
    const int t = threadIdx.x % LANES, sub = threadIdx.x / LANES;
    const W *scale_p = static_cast<const W *>(a.scale), *shift_p = static_cast<const W *>(a.shift);
    constexpr bool ROOM = LANES < 1024;     // (1024 threads of 128 registers hold this row and the next only)
    W scale[CHUNKS][E], shift[CHUNKS][E];   // alpha times
    const Place<LANES, CHUNKS, E, WHOLE> at(t, a.C);
    auto load_params = [&](int j) __attribute__((always_inline)) {
        Chunk<W, E> sc, sh;
        int c = at.c[j];
        if (!ROOM) asm volatile("" : "+v"(c));   // (row by row, not all of them from before the rows on)
#pragma unroll
        for (int e = 0; e < E; ++e) sc.v[e] = W(1), sh.v[e] = W(0);
        if (scale_p && at.live[j]) load_chunk(sc, scale_p + c);
        if (shift_p && at.live[j]) load_chunk(sh, shift_p + c);
#pragma unroll
        for (int e = 0; e < E; ++e) scale[j][e] = a.alpha * sc.v[e], shift[j][e] = a.alpha * sh.v[e];
    };
    if (ROOM)
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) load_params(j);
    const int stride = (int)gridDim.x * ROWS;
    int row = (int)blockIdx.x * ROWS + sub;
    Chunk<TX, E> raw[CHUNKS];
    auto load = [&](int r) __attribute__((always_inline)) {
        const TX *x = static_cast<const TX *>(a.x) + r * a.xs;
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j)
            if (at.live[j]) load_chunk(raw[j], x + at.c[j]);
    };
    if (row < a.M) load(row);
    // (the rows of a workgroup's wavefronts end together but for the last round: with LANES = 64 there is no barrier in the loop)
    for (int parity = 0; row < a.M; row += stride, parity ^= 1) {
        W x[CHUNKS][E];
        W sum = W(0);
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            if (!at.live[j]) continue;
            if (!WHOLE) arrive(raw[j]);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                x[j][e] = Stored<TX>::widen(raw[j].v[e]);
                if (at.counts(j, e)) sum += x[j][e];
            }
        }
        TY *y = static_cast<TY *>(a.y) + row * a.ys;
        Chunk<TY, E> old[CHUNKS];
        if ((ROOM || !WHOLE) && a.beta != W(0))   // (all of the row, before any of it is written)
#pragma unroll
            for (int j = 0; j < CHUNKS; ++j)
                if (at.live[j]) load_chunk(old[j], y + at.c[j]);
        if (row + stride < a.M) load(row + stride);
        if (!WHOLE && a.beta != W(0))
#pragma unroll
            for (int j = 0; j < CHUNKS; ++j)
                if (at.live[j]) arrive(old[j]);
        const W mean = row_sum<LANES>(sum, slots[parity][0]) / W(a.C);
        W squares = W(0);
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            if (!at.live[j]) continue;
#pragma unroll
            for (int e = 0; e < E; ++e) {
                x[j][e] -= mean;
                if (at.counts(j, e)) squares += x[j][e] * x[j][e];
            }
        }
        const W s = W(1) / sqrt(row_sum<LANES>(squares, slots[parity][1]) / W(a.C) + a.epsilon);
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            if (!at.live[j]) continue;
            if (!ROOM) {
                __builtin_amdgcn_sched_barrier(0);   // (one chunk's at a time)
                load_params(j);
                if (WHOLE && a.beta != W(0)) load_chunk(old[j], y + at.c[j]);
            }
            W out[E];
#pragma unroll
            for (int e = 0; e < E; ++e) out[e] = x[j][e] * s * scale[j][e] + shift[j][e];
            if (a.beta != W(0))
#pragma unroll
                for (int e = 0; e < E; ++e) out[e] += a.beta * Stored<TY>::widen(old[j].v[e]);
            store_chunk(y + at.c[j], out);
        }
        if (t == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.invstd) a.invstd[row] = s;
        }
    }
}

// dx of every row, and dscale's and dshift's sums over the workgroup's rows in registers (parts[workgroup]).  With 1024 threads to a
// row their 128 registers hold the row as it is stored and the sums only: scale comes from the cache, the next row's loads are not made ahead.
template <class TX, class TY, int LANES, int CHUNKS, bool WHOLE>
__global__ __launch_bounds__(norm_threads(LANES)) void layer_norm_backward_held_kernel(const NormBackwardArgs<typename Stored<TX>::wide_t> a) {
    typedef typename Stored<TX>::wide_t W;
    constexpr int E = kChunk<TX>, THREADS = norm_threads(LANES), ROWS = THREADS / LANES;
    __shared__ W slots[2][2 * THREADS / 64];
    const int t = threadIdx.x % LANES, sub = threadIdx.x / LANES;
    constexpr bool ROOM = LANES < 1024;
    W scale[CHUNKS][E], ds[CHUNKS][E], db[CHUNKS][E];   // (without room one chunk's scale is alive at a time)
    const Place<LANES, CHUNKS, E, WHOLE> at(t, a.C);
    auto load_scale = [&](int j) __attribute__((always_inline)) {
        Chunk<W, E> sc;
#pragma unroll
        for (int e = 0; e < E; ++e) sc.v[e] = W(1);
        int c = at.c[j];
        if (!ROOM) asm volatile("" : "+v"(c));   // (as above)
        if (a.scale && at.live[j]) load_chunk(sc, a.scale + c);
#pragma unroll
        for (int e = 0; e < E; ++e) scale[j][e] = sc.v[e];
    };
#pragma unroll
    for (int j = 0; j < CHUNKS; ++j) {
        if (ROOM) load_scale(j);
#pragma unroll
        for (int e = 0; e < E; ++e) ds[j][e] = db[j][e] = W(0);
    }
    const int stride = (int)gridDim.x * ROWS;
    int row = (int)blockIdx.x * ROWS + sub;
    Chunk<TX, E> rx[CHUNKS], rr[CHUNKS], next_r[CHUNKS];
    Chunk<TY, E> rdy[CHUNKS];
    W mean, s;
    auto load = [&](int r) __attribute__((always_inline)) {
        const TX *x = static_cast<const TX *>(a.x) + r * a.xs;
        const TY *dy = static_cast<const TY *>(a.dy) + r * a.dys;
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            if (!at.live[j]) continue;
            load_chunk(rx[j], x + at.c[j]);
            load_chunk(rdy[j], dy + at.c[j]);
            if (a.beta != W(0)) load_chunk(next_r[j], static_cast<const TX *>(a.r) + r * a.rs + at.c[j]);
        }
        mean = a.mean[r];
        s = a.invstd[r];
    };
    if (ROOM && row < a.M) load(row);
    for (int parity = 0; row < a.M; row += stride, parity ^= 1) {
        if (!ROOM) load(row);
        // h and q of the row's elements; without room for them they are taken from the row again when dx is written
        W h[ROOM ? CHUNKS : 1][E], q[ROOM ? CHUNKS : 1][E];
        W sum = W(0), along = W(0);
        const W inv = s, average = mean;
        if (ROOM && a.beta != W(0))
#pragma unroll
            for (int j = 0; j < CHUNKS; ++j)
                if (at.live[j]) {
                    if (!WHOLE) arrive(next_r[j]);
                    rr[j] = next_r[j];
                }
        auto take = [&](int j, int to) __attribute__((always_inline)) {
            if (!ROOM) load_scale(j);
#pragma unroll
            for (int e = 0; e < E; ++e) {
                h[to][e] = (Stored<TX>::widen(rx[j].v[e]) - average) * inv;
                q[to][e] = Stored<TY>::widen(rdy[j].v[e]) * scale[j][e];
            }
        };
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            if (!at.live[j]) continue;
            const int to = ROOM ? j : 0;
            take(j, to);
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (at.counts(j, e)) {
                    const W dy = Stored<TY>::widen(rdy[j].v[e]);
                    db[j][e] += dy;
                    ds[j][e] += dy * h[to][e];
                    sum += q[to][e];
                    along += q[to][e] * h[to][e];
                }
        }
        if (ROOM && row + stride < a.M) load(row + stride);
        if (!ROOM && !WHOLE && a.beta != W(0))
#pragma unroll
            for (int j = 0; j < CHUNKS; ++j)
                if (at.live[j]) arrive(next_r[j]);
        row_sums<LANES>(sum, along, slots[parity]);
        sum /= W(a.C);
        along /= W(a.C);
        const W f = a.alpha * inv;
        TX *dx = static_cast<TX *>(a.dx) + row * a.dxs;
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            if (!at.live[j]) continue;
            const int to = ROOM ? j : 0;
            if (!ROOM) take(j, 0);
            W out[E];
#pragma unroll
            for (int e = 0; e < E; ++e) out[e] = f * (q[to][e] - sum - h[to][e] * along);
            if (a.beta != W(0))
#pragma unroll
                for (int e = 0; e < E; ++e) out[e] += a.beta * Stored<TX>::widen((ROOM ? rr[j] : next_r[j]).v[e]);
            store_chunk(dx + at.c[j], out);
        }
    }
    if (!a.parts) return;
    W *parts = a.parts + (size_t)blockIdx.x * 2 * a.C;
    if constexpr (ROWS == 1) {
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j) {
            if (!at.live[j]) continue;
            if (at.skip(j) == 0) {
                store_chunk(parts + at.c[j], ds[j]);
                store_chunk(parts + a.C + at.c[j], db[j]);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (at.counts(j, e)) {
                        parts[at.c[j] + e] = ds[j][e];
                        parts[a.C + at.c[j] + e] = db[j][e];
                    }
            }
        }
    } else {   // the wavefronts' sums, added in their order
        __shared__ W sums[ROWS][LANES * E];
#pragma unroll
        for (int j = 0; j < CHUNKS; ++j)
#pragma unroll
            for (int which = 0; which < 2; ++which) {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < E; ++e)
                    if (at.counts(j, e)) sums[sub][(e - at.skip(j)) * LANES + t] = which ? db[j][e] : ds[j][e];
                __syncthreads();
                for (int i = threadIdx.x; i < LANES * E; i += THREADS) {
                    const int c = j * LANES * E + i, at = (i % E) * LANES + i / E;
                    W v = sums[0][at];
#pragma unroll
                    for (int r = 1; r < ROWS; ++r) v += sums[r][at];
                    if (c < a.C) parts[(which ? a.C : 0) + c] = v;
                }
            }
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

// f(LANES, CHUNKS) of the smallest shape that holds a row of C values of `elem` bytes computed with; false: none does
template <int L, int N> struct Shape {
    static constexpr int LANES = L, CHUNKS = N;
};
template <bool BACKWARD, class F>
bool by_shape(int C, bool f64, F f) {
    const int chunks = f64 ? (C + 3) / 4 : (C + 7) / 8;
    if (C < (f64 ? 4 : 8)) return false;
    if (chunks <= 16) return f(Shape<16, 1>()), true;
    if (chunks <= 32) return f(Shape<32, 1>()), true;
    if (chunks <= 64) return f(Shape<64, 1>()), true;
    if (chunks <= 128) return f(Shape<64, 2>()), true;
    if (chunks <= 256) return f(Shape<256, 1>()), true;
    if (chunks <= 512) return f(Shape<256, 2>()), true;
    if (chunks <= 1024) return f(Shape<512, 2>()), true;
    if (chunks <= 2048) return f(typename std::conditional<BACKWARD, Shape<1024, 2>, Shape<512, 4>>::type()), true;
    if constexpr (!BACKWARD)
        if (chunks <= 4096) return f(Shape<1024, 4>()), true;
    return false;
}

// ranges of rows whose sums are taken side by side
int param_ranges(const igcContext *h, const Matrix &x, bool f64) {
    int held = 0;
    if (by_shape<true>(x.cols, f64, [&](auto shape) {
            constexpr int rows = norm_threads(decltype(shape)::LANES) / decltype(shape)::LANES;
            const long long wanted = (long long)h->computeUnits * (decltype(shape)::LANES >= 512 ? 1 : 2);
            held = (int)std::max(1ll, std::min(wanted, (x.rows + 2 * rows - 1) / (2 * rows)));
        }))
        return held;
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
        a.xs = p.x.stride; a.ys = p.y.stride; a.M = (int)p.x.rows; a.C = p.x.cols;
        a.alpha = (W)host_scalar(alpha, f64); a.beta = (W)host_scalar(beta, f64); a.epsilon = (W)epsilon;
        igcStatus rc = IGC_STATUS_SUCCESS;
        if (by_shape<false>(a.C, f64, [&](auto shape) {
                constexpr int LANES = decltype(shape)::LANES, THREADS = norm_threads(LANES), ROWS = THREADS / LANES;
                const long long groups = (p.x.rows + ROWS - 1) / ROWS, most = (long long)handle->computeUnits * (LANES >= 512 ? 4 : 8);
                rc = launch_kernel(a.C % kChunk<TX> == 0 ? reinterpret_cast<const void *>(&layer_norm_held_kernel<TX, TY, LANES, decltype(shape)::CHUNKS, true>)
                                                     : reinterpret_cast<const void *>(&layer_norm_held_kernel<TX, TY, LANES, decltype(shape)::CHUNKS, false>), a,
                                   dim3((unsigned)std::min(groups, most)), THREADS, handle->stream);
            }))
            return rc;
        return launch_kernel(reinterpret_cast<const void *>(&layer_norm_rows_kernel<TX, TY>), a, dim3((unsigned)std::min(a.M, kMostRowGroups)), 256, handle->stream);
    });
}

igcStatus igcGetLayerNormBackwardWorkspaceSize(igcHandle_t handle, igcTensorDescriptor_t xDesc, igcTensorDescriptor_t dyDesc,
                                               igcTensorDescriptor_t dxDesc, size_t *sizeInBytes) {
    if (!handle || !sizeInBytes) return IGC_STATUS_BAD_PARAM;
    NormProblem p;
    const igcStatus st = check_norm_backward(xDesc, dyDesc, dxDesc, &p);
    if (st != IGC_STATUS_SUCCESS) return st;
    const int ranges = param_ranges(handle, p.x, xDesc->dtype == IGC_DATA_DOUBLE);
    *sizeInBytes = (size_t)ranges * 2 * p.x.cols * (xDesc->dtype == IGC_DATA_DOUBLE ? 8 : 4);
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
        a.ranges = param_ranges(handle, p.x, f64);
        const bool params = dscale || dshift;
        const size_t need = (size_t)a.ranges * 2 * (size_t)a.C * sizeof(W);
        if (params && workSpace && workSpaceSizeInBytes >= need && (uintptr_t)workSpace % sizeof(W) == 0) a.parts = static_cast<W *>(workSpace);
        igcStatus rc = IGC_STATUS_SUCCESS;
        if (by_shape<true>(a.C, f64, [&](auto shape) {
                constexpr int LANES = decltype(shape)::LANES, THREADS = norm_threads(LANES);
                rc = launch_kernel(a.C % kChunk<TX> == 0 ? reinterpret_cast<const void *>(&layer_norm_backward_held_kernel<TX, TY, LANES, decltype(shape)::CHUNKS, true>)
                                                     : reinterpret_cast<const void *>(&layer_norm_backward_held_kernel<TX, TY, LANES, decltype(shape)::CHUNKS, false>), a,
                                   dim3((unsigned)a.ranges), THREADS, handle->stream);
            })) {
            if (rc != IGC_STATUS_SUCCESS || !params) return rc;
        } else {
            rc = launch_kernel(reinterpret_cast<const void *>(&layer_norm_backward_rows_kernel<TX, TY>), a, dim3((unsigned)std::min(a.M, kMostRowGroups)), 256, handle->stream);
            if (rc != IGC_STATUS_SUCCESS || !params) return rc;
            if (a.parts) {
                a.per = (a.M + a.ranges - 1) / a.ranges;
                a.ranges = (a.M + a.per - 1) / a.per;
                rc = launch_kernel(reinterpret_cast<const void *>(&layer_norm_params_kernel<TX, TY>), a, dim3((unsigned)(a.C + 63) / 64u, (unsigned)a.ranges), 256,
                                   handle->stream);
                if (rc != IGC_STATUS_SUCCESS) return rc;
            }
        }
        return launch_kernel(reinterpret_cast<const void *>(&layer_norm_params_sum_kernel<TX, TY>), a, dim3((unsigned)(a.C + 31) / 32u), 1024, handle->stream);
    });
}

}  // extern "C"
