// What the operators on device tensors share: types, matrix products and running softmax weights of the attention kernels, and rows of
// logits with their exponentials in 64 bits.
#pragma once
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>

#include "ps_internal.h"

namespace ps {

namespace {

typedef _Float16 f16_t;
typedef __bf16 bf16_t;
typedef uint32_t u4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u2_t __attribute__((ext_vector_type(2)));

constexpr float kFloatMax = 3.402823466e38f;
constexpr uint64_t kMostGroups = (1u << 24) - 1;       // of 256 threads: a launch holds less than 2^32

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return min(max(v, lo), hi); }

template <typename T> __device__ __forceinline__ float to_f(T v) { return (float)v; }

// ------------------------------------------------------------------------------------ attention on the matrix cores
typedef float f4_t __attribute__((ext_vector_type(4)));
typedef f16_t f16x8_t __attribute__((ext_vector_type(8)));
typedef bf16_t bf16x8_t __attribute__((ext_vector_type(8)));

template <typename T> struct Mfma;
template <> struct Mfma<f16_t> {
    typedef f16x8_t v8;
    static constexpr uint32_t kInf = 0x7C007C00u;
    static __device__ __forceinline__ f4_t mul(v8 a, v8 b, f4_t c) {
#if defined(__HIP_DEVICE_COMPILE__)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
#else
        return c;
#endif
    }
};
template <> struct Mfma<bf16_t> {
    typedef bf16x8_t v8;
    static constexpr uint32_t kInf = 0x7F807F80u;
    static __device__ __forceinline__ f4_t mul(v8 a, v8 b, f4_t c) {
#if defined(__HIP_DEVICE_COMPILE__)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
#else
        return c;
#endif
    }
};

// A operand of 16 dims x 32 positions from rows staged in LDS: two transpose reads, four rows (hi bytes) apart
__device__ __forceinline__ u4_t transposed(const unsigned char *p, uint32_t hi) {
#if defined(__HIP_DEVICE_COMPILE__)
    typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s4_t;
    typedef __attribute__((address_space(3))) s4_t lds_s4_t;
    const u2_t a = __builtin_bit_cast(u2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_t *)(p)));
    const u2_t b = __builtin_bit_cast(u2_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4_t *)(p + hi)));
    return u4_t{a.x, a.y, b.x, b.y};
#else
    return u4_t{};
#endif
}
// largest value of the four lanes that share a row (lane, lane ^ 16, ^ 32, ^ 48)
__device__ __forceinline__ float row_max(float v) {
    v = fmaxf(v, __shfl_xor(v, 16, 64));
    return fmaxf(v, __shfl_xor(v, 32, 64));
}
// An infinite value or one that is no number must not meet the zero weight of a row that does not see it: the product takes
// zero in its place (and rows that do see it get it at the end); whether there was one
template <typename T>
__device__ __forceinline__ bool made_finite(u4_t &v) {
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const uint32_t d = v[e];
        const bool l16 = (d & Mfma<T>::kInf & 0xFFFFu) == (Mfma<T>::kInf & 0xFFFFu), h16 = (d & Mfma<T>::kInf & 0xFFFF0000u) == (Mfma<T>::kInf & 0xFFFF0000u);
        odd |= l16 || h16;
        v[e] = (l16 ? 0u : d & 0xFFFFu) | (h16 ? 0u : d & 0xFFFF0000u);
    }
    return odd;
}

// Weights in the tensors' type are held as 2^kLift times exp(score - running maximum), and a row's maximum is raised only where one would
// pass 2^(kLift + kSlack).  fp16 ends at 2^-24 below and 2^16 above: lifted by 2^10 its steps end at 2^-34 of the maximum, and the roundings of 2^17 keys
// there are 2^-18 of it together (without the lift, 4000 keys 18 nats behind one whose value is zero vanished, where they are the whole result).
// bf16 has the range of fp32: its weights stay at or below 1, so that they add up with large values no further than unscaled ones do.
// A larger lift leaves less slack and more rows to raise: 64 tokens over 131072 positions 185 us with 7 and 8, 186 with 10 and 5.9, 189 with 12 and 3.
template <typename T> struct WeightRange;
template <> struct WeightRange<f16_t> { static constexpr float kLift = 10.f, kSlack = 5.9f; };
template <> struct WeightRange<bf16_t> { static constexpr float kLift = -8.f, kSlack = 8.f; };

// Scores of a tile (S, hidden positions -inf) to weights P relative to the running maximum: each row by its own scores alone, so
// its result does not depend on its neighbours
template <typename T, int NT, int DT>
__device__ __forceinline__ void weigh(const f4_t (&S)[NT][2], float (&m_run)[NT], f4_t (&L)[NT], f4_t (&O)[NT][DT], typename Mfma<T>::v8 (&P)[NT], float c2, float slack) {
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        float mx = fmaxf(fmaxf(fmaxf(S[t][0][0], S[t][0][1]), fmaxf(S[t][0][2], S[t][0][3])), fmaxf(fmaxf(S[t][1][0], S[t][1][1]), fmaxf(S[t][1][2], S[t][1][3])));
        // (the difference is exact where it is close to the slack; a sum rounds, from 2^24 on past what fp16 holds)
        if (__any(mx - m_run[t] > slack)) {
            mx = row_max(mx);
            mx = mx - m_run[t] > slack ? mx : m_run[t];
            const float resc = m_run[t] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f((m_run[t] - mx) * c2);
            m_run[t] = mx;
            L[t] = L[t] * resc;
#pragma unroll
            for (int dt = 0; dt < DT; ++dt) O[t][dt] = O[t][dt] * resc;
        }
        // the difference first: 0 at the maximum, however large (s c2 - m c2 in one operation is off by half a step of m c2, 2^4 at 2^28; 3 % of the
        // time of 64 tokens over 131072 positions, nothing where the cache's bytes bound)
        const float ms = m_run[t] == -INFINITY ? 0.f : m_run[t];
#pragma unroll
        for (int e = 0; e < 8; ++e) P[t][e] = (T)__builtin_amdgcn_exp2f(fmaf(S[t][e >> 2][e & 3] - ms, c2, WeightRange<T>::kLift));
    }
}

// ------------------------------------------------------------------------------------ rows of logits
// no number: -inf (the larger of the two that is one); +inf: the largest finite number
__device__ __forceinline__ float sane(float v) { return fminf(fmaxf(v, -INFINITY), kFloatMax); }

// exp((x - m) / T) with k = log2(e) / T, for N values in step (one after the other they are a chain of 15 operations each, which few
// waves cannot hide): 2^t, t = n + f, |f| <= 1/2, and the polynomial of degree 7 whose largest relative error on that range is least (4e-11
// where fp32 has 6e-8 beside the same exponent's; its nine extrema found by exchange; degree 8, 8e-13, takes 125 us where this takes 121).  n is
// what remains of t beside 1.5 2^52, and then its low word.  t below 1000; -inf gives 0, where m is finite.  (x k - m k in one operation
// would lose everything where m is the largest finite number)
template <int N>
__device__ __forceinline__ void weights(const float (&x)[N], float m, double k, double (&w)[N]) {
    constexpr double c[8] = {1.520192159459773e-05, 0.00015469291141683518, 0.001333392256353862, 0.00961802725366847, 0.0555041035344798,
                             0.24022651198157585, 0.693147180728447, 0.9999999999616819};
    constexpr double kWhole = 6755399441055744.0;
    const double least = -1100.0 / k;
    double f[N];
    int n[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const double d = fmax((double)x[e] - (double)m, least), t = fma(d, k, kWhole);
        f[e] = fma(d, k, kWhole - t);
        n[e] = (int)(uint32_t)__builtin_bit_cast(uint64_t, t);
        w[e] = c[0];
    }
#pragma unroll
    for (int j = 1; j < 8; ++j)
#pragma unroll
        for (int e = 0; e < N; ++e) w[e] = fma(w[e], f[e], c[j]);
#pragma unroll
    for (int e = 0; e < N; ++e) w[e] = ldexp(w[e], n[e]);
}
__device__ __forceinline__ double weight(float x, float m, double k) {
    const float v[1] = {x};
    double w[1];
    weights(v, m, k, w);
    return w[0];
}
__device__ __forceinline__ double rate_of(float temp) { return 1.4426950408889634 / (double)fminf(temp, 1e30f); }

// Eight logits of a row, which may start anywhere, as they lie in memory (past the end -inf), taken out two at a time
template <typename T>
struct Oct {
    static constexpr int N = sizeof(T) * 2;
    uint32_t d[N];
    __device__ __forceinline__ void fill(const T *x, uint32_t i) { __builtin_memcpy(d, x + i, sizeof(d)); }
    __device__ __forceinline__ void fill(const T *x, uint32_t i, uint32_t end) {
        if (i + 8 <= end) { fill(x, i); return; }
#pragma unroll 1
        for (uint32_t e = i; e < i + 8; ++e) {
            const T v = e < end ? x[e] : (T)-INFINITY;
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const uint32_t from = j + 1 < N ? d[j + 1] : sizeof(T) == 2 ? (uint32_t)__builtin_bit_cast(uint16_t, (uint16_t)bits(v)) : bits(v);
                d[j] = sizeof(T) == 2 ? d[j] >> 16 | from << 16 : from;
            }
        }
    }
    static __device__ __forceinline__ uint32_t bits(T v) {
        if constexpr (sizeof(T) == 2) return __builtin_bit_cast(uint16_t, v);
        else return __builtin_bit_cast(uint32_t, v);
    }
    __device__ __forceinline__ void take(float &a, float &b) {
        if constexpr (sizeof(T) == 2) {
            a = sane(to_f(__builtin_bit_cast(T, (uint16_t)d[0])));
            b = sane(to_f(__builtin_bit_cast(T, (uint16_t)(d[0] >> 16))));
#pragma unroll
            for (int j = 0; j + 1 < N; ++j) d[j] = d[j + 1];
        } else {
            a = sane(__builtin_bit_cast(float, d[0]));
            b = sane(__builtin_bit_cast(float, d[1]));
#pragma unroll
            for (int j = 0; j + 2 < N; ++j) d[j] = d[j + 2];
        }
    }
};

}  // namespace

// ------------------------------------------------------------------------------------ entry points
#define PS_TRY(call)                                                                                    \
    do {                                                                                                \
        const hipError_t e_ = (call);                                                                   \
        if (e_ != hipSuccess) { set_error("%s failed: %s", #call, hipGetErrorString(e_)); return PS_E_HIP; } \
    } while (0)
#define PS_WANT(cond, ...)                                        \
    do {                                                          \
        if (!(cond)) { set_error(__VA_ARGS__); return PS_E_ARG; } \
    } while (0)

inline uint32_t type_bytes(uint32_t type) { return type == PS_TYPE_F32 ? 4 : 2; }
inline bool aligned(const void *p, uint64_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

}  // namespace ps
