// What the kernels of a worker's local step share: element types, 16-byte access, activations.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <type_traits>

#include "common.cuh"

namespace slimdp {

inline size_t type_bytes(int32_t type) { return type == SLIMDP_F32 ? 4 : 2; }
inline bool type_ok(int32_t type) { return type >= SLIMDP_F32 && type <= SLIMDP_F16; }

// Calls f with a value of the element type that `type` names.
template <typename F>
inline slimdp_status with_type(int32_t type, F&& f) {
    switch (type) {
        case SLIMDP_F32: return f(float());
        case SLIMDP_BF16: return f(__nv_bfloat16());
        case SLIMDP_F16: return f(__half());
    }
    return SLIMDP_ERR_INVALID_ARG;
}

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }

template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// N adjacent elements as one access; N sizeof(T) is 16 for a vector access and sizeof(T) for a scalar one.
template <typename T, int N>
struct alignas(N * sizeof(T)) Pack {
    T v[N];
};

template <typename T, int N>
__device__ __forceinline__ Pack<T, N> load_pack(const T* p) {
    return *reinterpret_cast<const Pack<T, N>*>(p);
}

template <typename T, int N>
__device__ __forceinline__ void unpack(const Pack<T, N>& p, float* f) {
#pragma unroll
    for (int i = 0; i < N; ++i) f[i] = to_f32(p.v[i]);
}

// Two values rounded and packed by one instruction.
template <typename T>
__device__ __forceinline__ uint32_t pack_two(float lo, float hi) {
    if constexpr (std::is_same<T, __half>::value) {
        const __half2 r = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&r);
    } else {
        const __nv_bfloat162 r = __floats2bfloat162_rn(lo, hi);
        return *reinterpret_cast<const uint32_t*>(&r);
    }
}

template <typename T, int N>
__device__ __forceinline__ void store_pack(T* p, const float* f) {
    if constexpr (sizeof(T) == 2 && N == 8) {
        *reinterpret_cast<uint4*>(p) = make_uint4(pack_two<T>(f[0], f[1]), pack_two<T>(f[2], f[3]), pack_two<T>(f[4], f[5]), pack_two<T>(f[6], f[7]));
    } else {
        Pack<T, N> r;
#pragma unroll
        for (int i = 0; i < N; ++i) r.v[i] = from_f32<T>(f[i]);
        *reinterpret_cast<Pack<T, N>*>(p) = r;
    }
}

// Elements of a 16-byte access.
template <typename T>
constexpr int kVec = 16 / (int)sizeof(T);

// Whether every row of a matrix can be read in 16-byte pieces from its start to its end.
inline bool rows_vectorise(const void* p, uint64_t ld, uint64_t cols, int32_t type) {
    const uint64_t b = type_bytes(type);
    return aligned16(p) && (ld * b) % 16 == 0 && (cols * b) % 16 == 0;
}

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) v += __shfl_xor_sync(0xFFFFFFFFu, v, d);
    return v;
}
__device__ __forceinline__ float warp_max(float v) {
    float r;
    asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}

// 2^x; the hardware's approximation (2 ulp, subnormal results to 0) is below the rounding of what is made of it.
__device__ __forceinline__ float exp2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// The normal distribution's Phi(z) and phi(z) from one exponential: erfc(x) = p(t) exp(-x^2), t = 1 / (1 + 0.3275911 x), p of
// degree 5, within 1.5e-7 (Abramowitz and Stegun, Handbook of Mathematical Functions, 7.1.26).  The lower tail is p(t) exp(-x^2) / 2
// itself, without a difference from 1.
__device__ __forceinline__ void normal(float z, float& cdf, float& pdf) {
    const float x = fabsf(z) * 0.70710678118654752f;
    const float t = rcp_approx(fmaf(0.3275911f, x, 1.0f));
    const float e = exp2_approx(x * x * -kLog2e);
    float p = fmaf(1.061405429f, t, -1.453152027f);
    p = fmaf(p, t, 1.421413741f);
    p = fmaf(p, t, -0.284496736f);
    p = fmaf(p, t, 0.254829592f);
    const float tail = 0.5f * p * t * e;
    cdf = z < 0.0f ? tail : 1.0f - tail;
    pdf = 0.39894228040143268f * e;
}

__device__ __forceinline__ float logistic(float z) { return rcp_approx(1.0f + exp2_approx(z * -kLog2e)); }

// z -> act(z).  0.5 (1 + tanh u) is logistic(2 u).
template <int ACT>
__device__ __forceinline__ float act_value(float z) {
    if constexpr (ACT == SLIMDP_ACT_RELU) return z != z ? z : fmaxf(z, 0.0f);
    if constexpr (ACT == SLIMDP_ACT_GELU) {
        float cdf, pdf;
        normal(z, cdf, pdf);
        return z * cdf;
    }
    if constexpr (ACT == SLIMDP_ACT_GELU_TANH) return z * logistic(1.5957691216057308f * (z + 0.044715f * z * z * z));
    if constexpr (ACT == SLIMDP_ACT_SILU) return z * logistic(z);
    return z;
}

// z -> d act(z) / dz.
template <int ACT>
__device__ __forceinline__ float act_slope(float z) {
    if constexpr (ACT == SLIMDP_ACT_RELU) return z > 0.0f ? 1.0f : 0.0f;
    if constexpr (ACT == SLIMDP_ACT_GELU) {
        float cdf, pdf;
        normal(z, cdf, pdf);
        return fmaf(z, pdf, cdf);
    }
    if constexpr (ACT == SLIMDP_ACT_GELU_TANH) {
        const float z2 = z * z, s = logistic(1.5957691216057308f * z * fmaf(0.044715f, z2, 1.0f));
        return fmaf(s * (1.0f - s) * 1.5957691216057308f * z, fmaf(0.134145f, z2, 1.0f), s);
    }
    if constexpr (ACT == SLIMDP_ACT_SILU) {
        const float s = logistic(z);
        return fmaf(z * s, 1.0f - s, s);
    }
    return 1.0f;
}

// Calls f with the activation that `act` names as a constant; not for none.
template <typename F>
__device__ __forceinline__ void with_act(int act, F&& f) {
    switch (act) {
        case SLIMDP_ACT_RELU: f(std::integral_constant<int, SLIMDP_ACT_RELU>()); break;
        case SLIMDP_ACT_GELU: f(std::integral_constant<int, SLIMDP_ACT_GELU>()); break;
        case SLIMDP_ACT_GELU_TANH: f(std::integral_constant<int, SLIMDP_ACT_GELU_TANH>()); break;
        case SLIMDP_ACT_SILU: f(std::integral_constant<int, SLIMDP_ACT_SILU>()); break;
    }
}

}  // namespace slimdp
