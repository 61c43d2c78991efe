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

// z -> act(z).
__device__ __forceinline__ float act_value(float z, int act) {
    switch (act) {
        case SLIMDP_ACT_RELU: return z != z ? z : fmaxf(z, 0.0f);
        case SLIMDP_ACT_GELU: return 0.5f * z * (1.0f + erff(z * 0.70710678118654752f));
        case SLIMDP_ACT_GELU_TANH: {
            const float u = 0.79788456080286536f * (z + 0.044715f * z * z * z);
            return 0.5f * z * (1.0f + tanhf(u));
        }
        case SLIMDP_ACT_SILU: return z / (1.0f + expf(-z));
        default: return z;
    }
}

// z -> d act(z) / dz.
__device__ __forceinline__ float act_slope(float z, int act) {
    switch (act) {
        case SLIMDP_ACT_RELU: return z > 0.0f ? 1.0f : 0.0f;
        case SLIMDP_ACT_GELU:
            return 0.5f * (1.0f + erff(z * 0.70710678118654752f)) + z * 0.39894228040143268f * expf(-0.5f * z * z);
        case SLIMDP_ACT_GELU_TANH: {
            const float u = 0.79788456080286536f * (z + 0.044715f * z * z * z);
            const float t = tanhf(u);
            return 0.5f * (1.0f + t) + 0.5f * z * (1.0f - t * t) * 0.79788456080286536f * (1.0f + 0.134145f * z * z);
        }
        case SLIMDP_ACT_SILU: {
            const float s = 1.0f / (1.0f + expf(-z));
            return s * (1.0f + z * (1.0f - s));
        }
        default: return 1.0f;
    }
}

}  // namespace slimdp
