// One AdamW step over many tensors:
//
//   g = s grad,  m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
//   p = p (1 - rate decay) - rate (m / (1 - b1^t)) / (sqrt(v / (1 - b2^t)) + epsilon)
//
// Every tensor's elements are cut into units of kUnit, one for each workgroup; the launch's arguments hold the table of up to kPerLaunch tensors, so
// that a list needs one launch for each that many of them and no table in device memory.
//
// States in 8 bits: blocks of 256 elements, which are a wavefront's four to a lane, each with a scale (the block's largest / the format's largest).  m is
// e4m3, v is e5m2, whose range (2^32) a block's squares need.  Both are rounded up or down at random with the probabilities that keep the
// average: the nearest code would swallow the small changes that both averages are made of (b2 = 0.999: a step moves v by a thousandth of what
// it lacks, the codes are an eighth to a quarter apart).  v itself and not its root is kept, because the average of a squared rounded root is not the square:
// it would grow by a fifth of a percent a step.  The random bits are a hash of seed, step and the element's place: a step gives the same bits again.
#include "igconv_rows.h"

namespace igc {
namespace {

constexpr int kUnit = 4096, kThreads = 256, kBlock = 256, kPerLaunch = 48;
constexpr long long kMostUnits = 1ll << 21;      // workgroups of a launch: more units are taken in turns

struct AdamWEntry {
    void *param;
    const void *grad;
    void *copy, *m, *v;
    float *mScale, *vScale;
    long long count;
    long long firstUnit;
    float decay;
    int kind;      // 1: bfloat16 param, 2: bfloat16 gradient, 4: states in 8 bits, 8: read as a stream
};
struct AdamWArgs {
    double beta1, beta2;
    float keep1, keep2, take1, take2, epsilon, rate, scale, correct1, correct2;   // keep: beta, take: 1 - beta, correct: 1 / (1 - beta^step)
    unsigned int seed;
    int step, tensors;
    long long units;
    const float *deviceRate, *deviceScale;
    const int *deviceStep;
    AdamWEntry entry[kPerLaunch];
};
static_assert(sizeof(AdamWArgs) <= 4096, "a launch's arguments");

// A published hash of 32 bits, multiplications and shifted exclusive ors, whose constants and shifts Chris Wellons found by a search for the least bias ("Prospecting for Hash Functions", 2018).
__host__ __device__ inline uint32_t mixed(uint32_t x) {
    x = (x ^ (x >> 16)) * 0x7FEB352Du;
    x = (x ^ (x >> 15)) * 0x846CA68Bu;
    return x ^ (x >> 16);
}

// 1 / (1 - beta^step), in double: 1 - 0.999 has few bits in float
__host__ __device__ inline float correction(double beta, int step) {
    double power = 1.0, square = beta;
    for (unsigned s = step < 1 ? 1u : (unsigned)step; s; s >>= 1) {
        if (s & 1) power *= square;
        square *= square;
    }
    return (float)(1.0 / (1.0 - power));
}

template <class T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Near {
    T v[N];
};

// (STREAM: not kept in caches, as whatever is stored: nothing is read again soon)
template <class T, bool STREAM>
__device__ __forceinline__ void load4(const void *from, long long at, int left, float (&to)[4]) {
    typedef uint32_t Words __attribute__((ext_vector_type(sizeof(T)), aligned(sizeof(T))));
    const T *p = static_cast<const T *>(from) + at;
    if (left >= 4) {
        const Words *words = reinterpret_cast<const Words *>(p);
        const Near<T, 4> q = __builtin_bit_cast(Near<T, 4>, STREAM ? __builtin_nontemporal_load(words) : *words);
#pragma unroll
        for (int e = 0; e < 4; ++e) to[e] = Stored<T>::widen(q.v[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            to[e] = 0.f;
            if (e < left) to[e] = Stored<T>::widen(p[e]);
        }
    }
}
template <class T>
__device__ __forceinline__ void store4(void *to, long long at, int left, const float (&from)[4]) {
    T *p = static_cast<T *>(to) + at;
    if (left >= 4) {
        Near<T, 4> q;
#pragma unroll
        for (int e = 0; e < 4; ++e) q.v[e] = Stored<T>::narrow(from[e]);
        typedef uint32_t Words __attribute__((ext_vector_type(sizeof(T)), aligned(sizeof(T))));
        __builtin_nontemporal_store(__builtin_bit_cast(Words, q), reinterpret_cast<Words *>(p));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) p[e] = Stored<T>::narrow(from[e]);
    }
}
template <bool STREAM>
__device__ __forceinline__ uint32_t load_codes(const void *from, long long at, int left) {
    typedef uint32_t Word __attribute__((aligned(1)));
    const uint8_t *p = static_cast<const uint8_t *>(from) + at;
    if (left >= 4) {
        const Word *word = reinterpret_cast<const Word *>(p);
        return STREAM ? __builtin_nontemporal_load(word) : *word;
    }
    uint32_t r = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e)
        if (e < left) r |= (uint32_t)p[e] << (8 * e);
    return r;
}
__device__ __forceinline__ void store_codes(void *to, long long at, int left, uint32_t codes) {
    uint8_t *p = static_cast<uint8_t *>(to) + at;
    if (left >= 4) {
        typedef uint32_t Word __attribute__((aligned(1)));
        __builtin_nontemporal_store(codes, reinterpret_cast<Word *>(p));
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) p[e] = (uint8_t)(codes >> (8 * e));
    }
}

// largest over all 64 lanes, of numbers that are not negative
__device__ __forceinline__ float lanes_max(float v) {
    auto with = [&](auto control) {
        return fmaxf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(control)::value, 0xF, 0xF, true)));
    };
    v = with(DppControl<0xB1>());
    v = with(DppControl<0x4E>());
    v = with(DppControl<0x141>());
    v = with(DppControl<0x140>());
    const int i = __builtin_bit_cast(int, v);
    return fmaxf(fmaxf(__builtin_bit_cast(float, __builtin_amdgcn_readlane(i, 0)), __builtin_bit_cast(float, __builtin_amdgcn_readlane(i, 16))),
                 fmaxf(__builtin_bit_cast(float, __builtin_amdgcn_readlane(i, 32)), __builtin_bit_cast(float, __builtin_amdgcn_readlane(i, 48))));
}

__device__ __forceinline__ bool is_finite(float v) { return (__builtin_bit_cast(uint32_t, v) & 0x7F800000u) != 0x7F800000u; }

template <bool SQUARES> struct Eight;   // the formats: bits behind the leading one, largest number
template <> struct Eight<false> {
    static constexpr int KEPT = 3;
    static constexpr float MOST = 448.f;
    static __device__ __forceinline__ uint32_t narrow(const float (&y)[4]) {
        const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
    }
    static __device__ __forceinline__ void widen(uint32_t c, float (&y)[4]) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c, true);
        y[0] = lo[0]; y[1] = lo[1]; y[2] = hi[0]; y[3] = hi[1];
    }
};
template <> struct Eight<true> {
    static constexpr int KEPT = 2;
    static constexpr float MOST = 57344.f, LEAST = 0x1p-16f;   // (a square that is not zero stays so: m over the root of zero would be no step but a leap)
    static __device__ __forceinline__ uint32_t narrow(const float (&y)[4]) {
        const int lo = __builtin_amdgcn_cvt_pk_bf8_f32(y[0], y[1], 0, false);
        return (uint32_t)__builtin_amdgcn_cvt_pk_bf8_f32(y[2], y[3], lo, true);
    }
    static __device__ __forceinline__ void widen(uint32_t c, float (&y)[4]) {
        const auto lo = __builtin_amdgcn_cvt_pk_f32_bf8((int)c, false), hi = __builtin_amdgcn_cvt_pk_f32_bf8((int)c, true);
        y[0] = lo[0]; y[1] = lo[1]; y[2] = hi[0]; y[3] = hi[1];
    }
};

// A block's scale and codes.  An element that is infinite or undefined becomes an undefined code and does not reach its block's scale.  random: 16 bits
// for each element, above (UPPER) or below 16 others.
template <bool SQUARES, bool UPPER>
__device__ __forceinline__ uint32_t encode(const float (&x)[4], const uint32_t (&random)[4], float *scale) {
    typedef Eight<SQUARES> F;
    constexpr int DROP = 23 - F::KEPT;
    // (the largest magnitude as a whole number: above all others where something is not finite)
    uint32_t most = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) most = max(most, __builtin_bit_cast(uint32_t, x[e]) & 0x7FFFFFFFu);
    const bool all_finite = __ballot(most >= 0x7F800000u) == 0;
    if (!all_finite) {
        most = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) most = max(most, is_finite(x[e]) ? __builtin_bit_cast(uint32_t, x[e]) & 0x7FFFFFFFu : 0u);
    }
    float s = lanes_max(__builtin_bit_cast(float, most)) * (1.f / F::MOST);
    float inverse = 1.f / s;
    if (s < 0x1p-100f) s = inverse = 0.f;     // (the inverse would be infinite)
    *scale = s;
    float y[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t part = UPPER ? random[e] >> (32 - DROP) & ~((1u << (DROP - 16)) - 1u) : (random[e] & 0xFFFFu) << (DROP - 16);
        const uint32_t bits = __builtin_bit_cast(uint32_t, x[e] * inverse) + part;
        float r = __builtin_bit_cast(float, bits & ~((1u << DROP) - 1u));
        if constexpr (SQUARES) {
            r = fminf(r, F::MOST);
            if (x[e] > 0.f && s > 0.f) r = fmaxf(r, F::LEAST);
        } else {
            r = __builtin_amdgcn_fmed3f(r, -F::MOST, F::MOST);
        }
        y[e] = r;
    }
    if (!all_finite)
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (!is_finite(x[e])) y[e] = __builtin_nanf("");
    return F::narrow(y);
}

// The instruction's root (like the inverse of the sum with epsilon, off by a last digit: with 8 bits the vector instructions come near to bounding the kernel, 108 of them
// an element with the exact ones, 96 % of its time, 78 with these), which takes numbers below the smallest normal one for zero.
__device__ __forceinline__ float root(float v) {
    const bool small = v < 0x1p-100f;
    const float r = __builtin_amdgcn_sqrtf(small ? v * 0x1p64f : v);
    return small ? r * 0x1p-32f : r;
}

struct Constants {
    float keep1, keep2, take1, take2, epsilon, rate, scale, correct1, correct2;
    uint32_t key;
};

// A wavefront's part of a unit: kUnit / 4 elements from `begin` on, in blocks of 256, all loads in front.
template <class TP, class TG, bool EIGHT, bool STREAM>
__device__ __forceinline__ void update(const AdamWEntry &t, const Constants &c, long long begin, int lane) {
#pragma clang fp contract(off)   // (m and v as written: each operation rounded once)
    constexpr int BLOCKS = kUnit / (kThreads / 64) / kBlock;
    float p[BLOCKS][4], g[BLOCKS][4], m[BLOCKS][4], v[BLOCKS][4], ms[BLOCKS], vs[BLOCKS];
    uint32_t mc[BLOCKS], vc[BLOCKS];
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
        const long long block = begin + b * kBlock, at = block + lane * 4, rest = t.count - at;
        const int left = rest >= 4 ? 4 : (rest < 0 ? 0 : (int)rest);
        load4<TP, STREAM>(t.param, at, left, p[b]);
        load4<TG, STREAM>(t.grad, at, left, g[b]);
        if constexpr (EIGHT) {
            mc[b] = load_codes<STREAM>(t.m, at, left);
            vc[b] = load_codes<STREAM>(t.v, at, left);
            ms[b] = vs[b] = 0.f;
            if (block < t.count) ms[b] = t.mScale[block / kBlock], vs[b] = t.vScale[block / kBlock];
        } else {
            load4<float, STREAM>(t.m, at, left, m[b]);
            load4<float, STREAM>(t.v, at, left, v[b]);
        }
    }
    // (subtracted as it is: 1 - rate decay has steps of 2^-24, a fifth of a decay of 1e-7 and all of one of 2e-8.  An infinite weight stays one.)
    const float decay = c.rate * t.decay, largest = 0x1.fffffep127f;
#pragma unroll
    for (int b = 0; b < BLOCKS; ++b) {
        const long long block = begin + b * kBlock, at = block + lane * 4, rest = t.count - at;
        const int left = rest >= 4 ? 4 : (rest < 0 ? 0 : (int)rest);
        if (block >= t.count) break;
        if constexpr (EIGHT) {
            Eight<false>::widen(mc[b], m[b]);
            Eight<true>::widen(vc[b], v[b]);
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float gs = g[b][e] * c.scale;
            if constexpr (EIGHT) m[b][e] *= ms[b], v[b][e] *= vs[b];
            m[b][e] = m[b][e] * c.keep1 + gs * c.take1;
            v[b][e] = v[b][e] * c.keep2 + gs * gs * c.take2;
            const float change = c.rate * (m[b][e] * c.correct1 * __builtin_amdgcn_rcpf(root(v[b][e] * c.correct2) + c.epsilon));
            p[b][e] -= __builtin_fmaf(decay, __builtin_amdgcn_fmed3f(p[b][e], -largest, largest), change);
        }
        store4<TP>(t.param, at, left, p[b]);
        if (t.copy) store4<bf16_t>(t.copy, at, left, p[b]);
        if constexpr (EIGHT) {
            // (four elements from a multiple of four on)
            uint32_t random[4];
            const uint32_t from = (uint32_t)at ^ c.key ^ ((uint32_t)(at >> 32) * 0x9E3779B9u);      // (2^32 over the golden ratio)
#pragma unroll
            for (int e = 0; e < 4; ++e) random[e] = mixed(from ^ (uint32_t)e);
            float sm, sv;
            const uint32_t cm = encode<false, false>(m[b], random, &sm), cv = encode<true, true>(v[b], random, &sv);
            store_codes(t.m, at, left, cm);
            store_codes(t.v, at, left, cv);
            if (lane == 0) t.mScale[block / kBlock] = sm, t.vScale[block / kBlock] = sv;
        } else {
            store4<float>(t.m, at, left, m[b]);
            store4<float>(t.v, at, left, v[b]);
        }
    }
}

__global__ __launch_bounds__(kThreads) void adamw_kernel(const AdamWArgs a) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    Constants c{a.keep1, a.keep2, a.take1, a.take2, a.epsilon, a.rate, a.scale, a.correct1, a.correct2, 0};
    int step = a.step;
    if (a.deviceRate) c.rate = *a.deviceRate;
    if (a.deviceScale) c.scale *= *a.deviceScale;
    if (a.deviceStep) {
        step = max(1, *a.deviceStep);
        c.correct1 = correction(a.beta1, step);
        c.correct2 = correction(a.beta2, step);
    }
    c.key = mixed(a.seed ^ mixed((uint32_t)step));
    const long long mine = lane < a.tensors ? a.entry[lane].firstUnit : a.units;
    for (long long unit = blockIdx.x; unit < a.units; unit += gridDim.x) {
        const int i = __builtin_popcountll(__ballot(mine <= unit)) - 1;    // (first units never fall along the table)
        const AdamWEntry &t = a.entry[i];
        const long long begin = (unit - t.firstUnit) * kUnit + wave * (kUnit / (kThreads / 64));
        switch (t.kind) {
        case 0: update<float, float, false, false>(t, c, begin, lane); break;
        case 1: update<bf16_t, float, false, false>(t, c, begin, lane); break;
        case 2: update<float, bf16_t, false, false>(t, c, begin, lane); break;
        case 3: update<bf16_t, bf16_t, false, false>(t, c, begin, lane); break;
        case 4: update<float, float, true, false>(t, c, begin, lane); break;
        case 5: update<bf16_t, float, true, false>(t, c, begin, lane); break;
        case 6: update<float, bf16_t, true, false>(t, c, begin, lane); break;
        case 7: update<bf16_t, bf16_t, true, false>(t, c, begin, lane); break;
        case 8: update<float, float, false, true>(t, c, begin, lane); break;
        case 9: update<bf16_t, float, false, true>(t, c, begin, lane); break;
        case 10: update<float, bf16_t, false, true>(t, c, begin, lane); break;
        case 11: update<bf16_t, bf16_t, false, true>(t, c, begin, lane); break;
        case 12: update<float, float, true, true>(t, c, begin, lane); break;
        case 13: update<bf16_t, float, true, true>(t, c, begin, lane); break;
        case 14: update<float, bf16_t, true, true>(t, c, begin, lane); break;
        default: update<bf16_t, bf16_t, true, true>(t, c, begin, lane); break;
        }
    }
}

// Elements of a call from which on what lies on 128-byte boundaries is read past the caches too (that of the step before has left them; off the boundaries a line's two halves are
// read by two wavefronts).  5.4e8 float elements 3030 us, with it 2810, before stores went past the caches 3130; 4e8 with 8 bits 1250, 1169, 1276; at odd places 1265, 1444,
// 1363; 1e6 float elements 8.6, 9.1, 10.4.
constexpr long long kStreamed = 1ll << 24;

bool off(const void *p, size_t to) { return (uintptr_t)p % to != 0; }
bool is_number(double v) { return (float)v - (float)v == 0.f; }    // (as a float)

igcStatus check_tensor(const igcAdamWTensor &t) {
    if (t.count < 0 || !is_number(t.weightDecay)) return IGC_STATUS_BAD_PARAM;
    if (t.stateBits != 32 && t.stateBits != 8) return IGC_STATUS_NOT_SUPPORTED;
    if ((t.paramType != IGC_DATA_FLOAT && t.paramType != IGC_DATA_BFLOAT16) || (t.gradType != IGC_DATA_FLOAT && t.gradType != IGC_DATA_BFLOAT16) ||
        t.count > (1ll << 40))
        return IGC_STATUS_NOT_SUPPORTED;
    if (t.copy && t.paramType != IGC_DATA_FLOAT) return IGC_STATUS_BAD_PARAM;
    if (t.count == 0) return IGC_STATUS_SUCCESS;
    if (!t.param || !t.grad || !t.m || !t.v || off(t.param, elem_size(t.paramType)) || off(t.grad, elem_size(t.gradType)) || off(t.copy, 2)) return IGC_STATUS_BAD_PARAM;
    if (t.stateBits == 8 ? !t.mScale || !t.vScale || off(t.mScale, 4) || off(t.vScale, 4) : off(t.m, 4) || off(t.v, 4)) return IGC_STATUS_BAD_PARAM;
    return IGC_STATUS_SUCCESS;
}

}  // namespace
}  // namespace igc

using namespace igc;

extern "C" igcStatus igcAdamWStep(igcHandle_t handle, const igcAdamWParameters *parameters, int tensors, const igcAdamWTensor *list) {
    if (!handle || !parameters || tensors < 0 || (tensors > 0 && !list)) return IGC_STATUS_BAD_PARAM;
    const igcAdamWParameters &q = *parameters;
    if (!(q.beta1 >= 0.0 && q.beta1 < 1.0 && q.beta2 >= 0.0 && q.beta2 < 1.0 && q.epsilon > 0.0) || !is_number(q.epsilon) || !is_number(q.gradientScale) ||
        (!q.deviceLearningRate && !is_number(q.learningRate)) || (!q.deviceStep && q.step < 1) || (float)q.epsilon < 0x1p-126f || off(q.deviceLearningRate, 4) ||
        off(q.deviceGradientScale, 4) || off(q.deviceStep, 4))
        return IGC_STATUS_BAD_PARAM;
    long long elements = 0;
    for (int i = 0; i < tensors; ++i) {
        const igcStatus st = check_tensor(list[i]);
        if (st != IGC_STATUS_SUCCESS) return st;
        elements += std::min(list[i].count, kStreamed);
    }
    AdamWArgs a{};
    a.beta1 = q.beta1; a.beta2 = q.beta2;
    a.keep1 = (float)q.beta1; a.keep2 = (float)q.beta2;
    a.take1 = (float)(1.0 - q.beta1); a.take2 = (float)(1.0 - q.beta2);
    a.epsilon = (float)q.epsilon; a.rate = (float)q.learningRate; a.scale = (float)q.gradientScale;
    a.correct1 = correction(q.beta1, q.step); a.correct2 = correction(q.beta2, q.step);
    a.seed = q.seed; a.step = q.step;
    a.deviceRate = q.deviceLearningRate; a.deviceScale = q.deviceGradientScale; a.deviceStep = q.deviceStep;
    for (int i = 0; i < tensors;) {
        a.tensors = 0;
        a.units = 0;
        for (; i < tensors && a.tensors < kPerLaunch; ++i) {
            const igcAdamWTensor &t = list[i];
            if (t.count == 0) continue;
            AdamWEntry &e = a.entry[a.tensors++];
            e.param = t.param; e.grad = t.grad; e.copy = t.copy; e.m = t.m; e.v = t.v; e.mScale = t.mScale; e.vScale = t.vScale;
            e.count = t.count;
            e.firstUnit = a.units;
            e.decay = (float)t.weightDecay;
            e.kind = (t.paramType == IGC_DATA_BFLOAT16 ? 1 : 0) | (t.gradType == IGC_DATA_BFLOAT16 ? 2 : 0) | (t.stateBits == 8 ? 4 : 0) |
                     (elements < kStreamed || off(t.param, 128) || off(t.grad, 128) || off(t.m, 128) || off(t.v, 128) ? 0 : 8);
            a.units += (t.count + kUnit - 1) / kUnit;
        }
        if (a.tensors == 0) continue;
        const igcStatus st = launch_kernel(reinterpret_cast<const void *>(&adamw_kernel), a, dim3((unsigned)std::min(a.units, kMostUnits)), kThreads, handle->stream);
        if (st != IGC_STATUS_SUCCESS) return st;
    }
    return IGC_STATUS_SUCCESS;
}
