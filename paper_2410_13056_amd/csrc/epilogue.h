// What follows a product: bias, activation, second factor and residual, in fp32.  One form for the integer products,
// which have it behind their sums, and for the call that runs it by itself.
#pragma once

#include "serving.h"

// N elements from p + i on, of which `n` are there (the others read 0).
template <int N>
__device__ __forceinline__ void load_some(const void *p, int dtype, int64_t i, int n, float (&x)[N]) {
    with_dtype(dtype, [&](auto like) {
        typedef decltype(like) T;
        const T *at = static_cast<const T *>(p) + i;
        if (n >= N) {
            load_f32<T, N>(at, x);
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k) x[k] = k < n ? (float)at[k] : 0.f;
        }
    });
}

// The first `n` of N values, each rounded once, to p + i on.
template <int N>
__device__ __forceinline__ void store_some(void *p, int dtype, int64_t i, int n, const float (&x)[N]) {
    with_dtype(dtype, [&](auto like) {
        typedef decltype(like) T;
        typedef T V __attribute__((ext_vector_type(N)));
        typedef V Any __attribute__((aligned(sizeof(T))));
        T *at = static_cast<T *>(p) + i;
        V v;
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = (T)x[k];
        if (n >= N) {
            *reinterpret_cast<Any *>(at) = v;
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k)
                if (k < n) at[k] = v[k];
        }
    });
}

// Eight values as they lie in memory, on their way before anything is done with them.
struct Raw8 {
    typedef uint32_t U4 __attribute__((ext_vector_type(4)));
    U4 w[2];
    __device__ __forceinline__ void load(const void *from, int dtype, int64_t i, int n) {
        typedef U4 Any __attribute__((aligned(2)));
        const int size = dtype == CMPQ_F32 ? 4 : 2;
        const char *p = static_cast<const char *>(from) + i * size;
        if (n >= 8) {
            w[0] = *reinterpret_cast<const Any *>(p);
            if (size == 4) w[1] = *reinterpret_cast<const Any *>(p + 16);
        } else {
            float x[8];
            load_some<8>(from, dtype, i, n, x);
            with_dtype(dtype, [&](auto like) {
                typedef decltype(like) T;
                typedef T V __attribute__((ext_vector_type(8)));
                V v;
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = (T)x[k];
                __builtin_memcpy(w, &v, sizeof(V));
            });
        }
    }
    __device__ __forceinline__ void values(int dtype, float (&x)[8]) const {
        with_dtype(dtype, [&](auto like) {
            typedef decltype(like) T;
            typedef T V __attribute__((ext_vector_type(8)));
            V v;
            __builtin_memcpy(&v, w, sizeof(V));
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = (float)v[k];
        });
    }
};

// e^x 2^-shift, |x| <= 1000, to about 2 steps of fp32: 2^(x log2 e - shift), with what the product's rounding and the constant's left
// out put back as a factor 1 + d ln 2.
__device__ __forceinline__ float exp_near(float x, float shift) {
#pragma clang fp contract(off)
    constexpr float kLog2e = 0x1.715476p+0f, kRest = 0x1.4ae0cp-26f, kLn2 = 0x1.62e43p-1f;  // log2 e = the first two's sum
    const float t = x * kLog2e, d = fmaf(x, kLog2e, -t) + x * kRest;
    return __builtin_amdgcn_exp2f(t - shift) * fmaf(d, kLn2, 1.f);
}

// v / (1 + e^z).  Beyond z = 80, where the 1 counts for nothing and 64 leaves no bit of z log2 e behind, e^z is taken 2^-64-fold and
// the quotient with it, or both would leave fp32 before the result does (-v / (1 + e^-v) is 2^-121 there); below -80 e^z counts for
// nothing.  Asked of all values of a wavefront at once, since few are so far out: 2048 rows of 28672 with a factor in bfloat16
// 77.4 us; 82 where each value chooses for itself, 76.8 without the tails.
template <int N>
__device__ __forceinline__ void over_one_plus_exp(float (&v)[N], const float (&z)[N]) {
#pragma clang fp contract(off)
    constexpr float kFar = 80.f;
    float most = fabsf(z[0]), q[N];
#pragma unroll
    for (int i = 1; i < N; ++i) most = fmaxf(most, fabsf(z[i]));
#pragma unroll
    for (int i = 0; i < N; ++i) q[i] = v[i] * __builtin_amdgcn_rcpf(1.f + exp_near(z[i], 0.f));
    if (__ballot(most > kFar)) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            if (z[i] > kFar) q[i] = v[i] * __builtin_amdgcn_rcpf(exp_near(fminf(z[i], 1000.f), 64.f)) * 0x1p-64f;
            if (z[i] < -kFar) q[i] = v[i];
        }
    }
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = q[i];
}

// `act` is the same in all lanes.  A NaN stays one; the limits at minus infinity are not taken (0 times infinity: NaN).
template <int N>
__device__ __forceinline__ void activate(int act, float (&v)[N]) {
#pragma clang fp contract(off)
    if (act == CMPQ_ACT_SILU) {
        float z[N];
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = -v[i];
        over_one_plus_exp(v, z);
    } else if (act == CMPQ_ACT_GELU) {  // v Phi(v), Phi(v) = erfc(-v / sqrt 2) / 2: no difference of near numbers
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = v[i] * (0.5f * erfcf(v[i] * -0.707106781f));
    } else if (act == CMPQ_ACT_GELU_TANH) {  // v (1 + tanh u) / 2 = v / (1 + e^-2u), u = sqrt(2 / pi) (v + 0.044715 v^3)
        float z[N];
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = -1.59576912f * (v[i] + 0.044715f * v[i] * v[i] * v[i]);
        over_one_plus_exp(v, z);
    } else if (act == CMPQ_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = v[i] < 0.f ? 0.f : v[i];
    }
}

static inline bool known_activation(int act) { return act >= CMPQ_ACT_NONE && act <= CMPQ_ACT_RELU; }
