// Matrix products of a layer, forward and backward, with what follows them in the same kernel.
//
//   forward          z = x w^T + bias, y = act(z) + residual
//   backward_input   dx = (dy w) * act'(z) + add
//   backward_weight  dw (+)= dy^T x, db (+)= sum over rows of dy
//
// All three are one product  C[i, j] = sum_l A(i, l) B(j, l)  over operands with two strides each.
#include <algorithm>

#include "train.cuh"

namespace slimdp {

namespace {

// What is done with C[i, j] before it is stored; NULL members are left out.
struct Epilogue {
    const float* bias;                 // + bias[j]
    void* z;  uint64_t ldz;            // pre-activation: written by forward, read by backward_input
    const void* add;  uint64_t ldadd;  // residual or its gradient
    void* out;  uint64_t ldo;
    int act;
    bool accumulate;                   // out is fp32 and keeps what it holds
};

enum Product { kForward, kInput, kWeight };

template <typename T, Product P>
__device__ __forceinline__ void finish(const Epilogue& e, uint64_t i, uint64_t j, float v) {
    if constexpr (P == kForward) {
        if (e.bias) v += __ldg(e.bias + j);
        if (e.z) ((T*)e.z)[i * e.ldz + j] = from_f32<T>(v);
        v = act_value(v, e.act);
        if (e.add) v += to_f32(((const T*)e.add)[i * e.ldadd + j]);
        ((T*)e.out)[i * e.ldo + j] = from_f32<T>(v);
    } else if constexpr (P == kInput) {
        if (e.act != SLIMDP_ACT_NONE) v *= act_slope(to_f32(((const T*)e.z)[i * e.ldz + j]), e.act);
        if (e.add) v += to_f32(((const T*)e.add)[i * e.ldadd + j]);
        ((T*)e.out)[i * e.ldo + j] = from_f32<T>(v);
    } else {
        float* o = (float*)e.out + i * e.ldo + j;
        *o = e.accumulate ? *o + v : v;
    }
}

template <typename T>
struct Operand {
    const T* p;
    uint64_t row, col;   // strides of the kept and of the summed index
};

// 64 x 64 results a CTA, 4 x 4 a thread, 16 summed indices a step.
template <typename T, Product P>
__global__ void __launch_bounds__(256) product_kernel(Operand<T> a, Operand<T> b, uint64_t m, uint64_t n, uint64_t k,
                                                      Epilogue e) {
    __shared__ float sa[16][65], sb[16][65];
    const uint64_t i0 = (uint64_t)blockIdx.y * 64, j0 = (uint64_t)blockIdx.x * 64;
    const uint32_t ti = threadIdx.x / 16, tj = threadIdx.x % 16;
    float acc[4][4] = {};
    for (uint64_t l0 = 0; l0 < k; l0 += 16) {
        for (uint32_t s = threadIdx.x; s < 64 * 16; s += 256) {
            const uint32_t r = a.col == 1 ? s / 16 : s % 64, c = a.col == 1 ? s % 16 : s / 64;
            sa[c][r] = (i0 + r < m && l0 + c < k) ? to_f32(a.p[(i0 + r) * a.row + (l0 + c) * a.col]) : 0.0f;
        }
        for (uint32_t s = threadIdx.x; s < 64 * 16; s += 256) {
            const uint32_t r = b.col == 1 ? s / 16 : s % 64, c = b.col == 1 ? s % 16 : s / 64;
            sb[c][r] = (j0 + r < n && l0 + c < k) ? to_f32(b.p[(j0 + r) * b.row + (l0 + c) * b.col]) : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int c = 0; c < 16; ++c)
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[u][v] = fmaf(sa[c][ti * 4 + u], sb[c][tj * 4 + v], acc[u][v]);
        __syncthreads();
    }
    for (int u = 0; u < 4; ++u)
        for (int v = 0; v < 4; ++v) {
            const uint64_t i = i0 + ti * 4 + u, j = j0 + tj * 4 + v;
            if (i < m && j < n) finish<T, P>(e, i, j, acc[u][v]);
        }
}

// db (+)= sum over rows of dy: a CTA takes 32 columns, its 32 warps every 32nd row each.
template <typename T>
__global__ void __launch_bounds__(1024) column_sum_kernel(const T* __restrict__ dy, uint64_t lddy, uint64_t m,
                                                          uint64_t n, float* __restrict__ db, bool accumulate) {
    __shared__ float smem[32][33];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint64_t j = (uint64_t)blockIdx.x * 32 + lane;
    float s = 0.0f;
    if (j < n)
        for (uint64_t i = warp; i < m; i += 32) s += to_f32(dy[i * lddy + j]);
    smem[warp][lane] = s;
    __syncthreads();
    s = warp_sum(smem[lane][warp]);
    const uint64_t c = (uint64_t)blockIdx.x * 32 + warp;
    if (lane == 0 && c < n) db[c] = accumulate ? db[c] + s : s;
}

template <typename T>
__global__ void __launch_bounds__(256) activation_backward_kernel(const T* __restrict__ dy, uint64_t lddy,
                                                                  const T* __restrict__ z, uint64_t ldz, uint64_t m,
                                                                  uint64_t n, int act, T* __restrict__ dz,
                                                                  uint64_t lddz) {
    for (uint64_t i = blockIdx.y; i < m; i += gridDim.y)
        for (uint64_t j = (uint64_t)blockIdx.x * 256 + threadIdx.x; j < n; j += (uint64_t)gridDim.x * 256) {
            const float d = to_f32(dy[i * lddy + j]);
            dz[i * lddz + j] = from_f32<T>(act == SLIMDP_ACT_NONE ? d : d * act_slope(to_f32(z[i * ldz + j]), act));
        }
}

template <typename T, Product P>
slimdp_status launch_product(Operand<T> a, Operand<T> b, uint64_t m, uint64_t n, uint64_t k, const Epilogue& e,
                             cudaStream_t st) {
    const dim3 grid((unsigned)((n + 63) / 64), (unsigned)((m + 63) / 64));
    if (grid.y > 65535) return SLIMDP_ERR_UNSUPPORTED;
    product_kernel<T, P><<<grid, 256, 0, st>>>(a, b, m, n, k, e);
    SLIMDP_LAUNCHED(1);
    return SLIMDP_OK;
}

}  // namespace

size_t linear_ws_bytes(uint64_t, uint64_t, uint64_t, int32_t) { return 256; }

slimdp_status launch_linear_forward(const void* x, uint64_t ldx, const void* w, uint64_t ldw, const float* bias,
                                    const void* residual, uint64_t ldr, uint64_t m, uint64_t n, uint64_t k,
                                    int32_t type, int32_t act, void* y, uint64_t ldy, void* z, uint64_t ldz, void* ws,
                                    cudaStream_t st) {
    if (m == 0) return SLIMDP_OK;
    const Epilogue e = {bias, z, ldz, residual, ldr, y, ldy, act, false};
    return with_type(type, [&](auto v) {
        using T = decltype(v);
        return launch_product<T, kForward>({(const T*)x, ldx, 1}, {(const T*)w, ldw, 1}, m, n, k, e, st);
    });
}

slimdp_status launch_linear_backward_input(const void* dy, uint64_t lddy, const void* w, uint64_t ldw, const void* z,
                                           uint64_t ldz, const void* add, uint64_t ldadd, uint64_t m, uint64_t n,
                                           uint64_t k, int32_t type, int32_t act, void* dx, uint64_t lddx, void* ws,
                                           cudaStream_t st) {
    if (m == 0) return SLIMDP_OK;
    const Epilogue e = {nullptr, const_cast<void*>(z), ldz, add, ldadd, dx, lddx, act, false};
    return with_type(type, [&](auto v) {
        using T = decltype(v);
        return launch_product<T, kInput>({(const T*)dy, lddy, 1}, {(const T*)w, 1, ldw}, m, k, n, e, st);
    });
}

slimdp_status launch_linear_backward_weight(const void* dy, uint64_t lddy, const void* x, uint64_t ldx, uint64_t m,
                                            uint64_t n, uint64_t k, int32_t type, float* dw, uint64_t lddw, float* db,
                                            bool accumulate, void* ws, cudaStream_t st) {
    if (m == 0 && accumulate) return SLIMDP_OK;
    const Epilogue e = {nullptr, nullptr, 0, nullptr, 0, dw, lddw, SLIMDP_ACT_NONE, accumulate};
    return with_type(type, [&](auto v) -> slimdp_status {
        using T = decltype(v);
        if (db) {
            column_sum_kernel<T><<<(unsigned)((n + 31) / 32), 1024, 0, st>>>((const T*)dy, lddy, m, n, db, accumulate);
            SLIMDP_LAUNCHED(1);
        }
        return launch_product<T, kWeight>({(const T*)dy, 1, lddy}, {(const T*)x, 1, ldx}, n, k, m, e, st);
    });
}

slimdp_status launch_activation_backward(const void* dy, uint64_t lddy, const void* z, uint64_t ldz, uint64_t m,
                                         uint64_t n, int32_t type, int32_t act, void* dz, uint64_t lddz,
                                         cudaStream_t st) {
    if (m == 0) return SLIMDP_OK;
    const dim3 grid((unsigned)std::min<uint64_t>((n + 255) / 256, 64), (unsigned)std::min<uint64_t>(m, 16384));
    return with_type(type, [&](auto v) -> slimdp_status {
        using T = decltype(v);
        activation_backward_kernel<T><<<grid, 256, 0, st>>>((const T*)dy, lddy, (const T*)z, ldz, m, n, act, (T*)dz, lddz);
        SLIMDP_LAUNCHED(1);
        return SLIMDP_OK;
    });
}

}  // namespace slimdp
