// Layer norm of a worker's local step, forward and backward.
//
// Forward, row by row:  mean = sum x / dim,  rstd = 1 / sqrt(sum (x - mean)^2 / dim + eps),
// y = (x - mean) rstd gamma + beta.  Backward with h = (x - mean) rstd and g = dy gamma:
// dx = rstd (g - avg(g) - h avg(g h)), dgamma = sum over rows of dy h, dbeta = sum over rows of dy.
//
// Both directions are bound by memory: each element is read once and written once, so a row stays in
// registers between its reductions and its result.  A group of threads (a warp for rows of up to 1024 elements, a
// CTA beyond) owns fixed columns and walks over rows; gamma, beta and the column sums of the gradients stay in
// registers all the while.  The variance is summed about the mean (a second reduction over registers, no
// second pass over memory), so that rows with a large mean or a single huge element keep their precision.
// The column sums leave a CTA as one row of partial sums in the workspace; a second kernel adds these rows in
// a fixed order, which keeps the result independent of scheduling.
#include <algorithm>

#include "train.cuh"

namespace slimdp {

namespace {

constexpr uint32_t kLnMaxParts = 592;      // rows of partial column sums; four CTAs on each of 148 SMs
constexpr uint64_t kLnRegisterDim = 16384; // longest row that stays in registers (1024 threads x 16 elements)

// Sum over the THREADS threads of a group, in every thread; `slot` alternates between calls that no barrier separates.
template <int N, bool WARP, int THREADS>
__device__ __forceinline__ void group_sum(float (&v)[N], float (&smem)[2][N][32], int slot) {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = warp_sum(v[i]);
    if constexpr (!WARP) {
        constexpr int kWarps = THREADS / 32;
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
        if (lane == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) smem[slot][i][warp] = v[i];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float s = lane < kWarps ? smem[slot][i][lane] : 0.0f;
            v[i] = warp_sum(s);
        }
    }
}

template <typename T, int VEC, int ELEMS, int THREADS, bool WARP>
__global__ void __launch_bounds__(THREADS) ln_forward_kernel(const T* __restrict__ x, uint64_t ldx, uint32_t rows,
                                                             uint32_t dim, const float* __restrict__ gamma,
                                                             const float* __restrict__ beta, float eps,
                                                             T* __restrict__ y, uint64_t ldy, float* __restrict__ mean,
                                                             float* __restrict__ rstd) {
    constexpr int kGroup = WARP ? 32 : THREADS, kItems = ELEMS / VEC;
    __shared__ float smem[2][1][32];
    const uint32_t t = WARP ? (threadIdx.x & 31) : threadIdx.x;
    const uint32_t group = WARP ? (threadIdx.x >> 5) : 0, groups = THREADS / kGroup;
    const float inv_dim = 1.0f / (float)dim;
    float ga[ELEMS], be[ELEMS];
#pragma unroll
    for (int i = 0; i < kItems; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const uint32_t c = (i * kGroup + t) * VEC + j;
            ga[i * VEC + j] = (gamma && c < dim) ? __ldg(gamma + c) : 1.0f;
            be[i * VEC + j] = (beta && c < dim) ? __ldg(beta + c) : 0.0f;
        }
    for (uint64_t row = (uint64_t)blockIdx.x * groups + group; row < rows; row += (uint64_t)gridDim.x * groups) {
        const T* xr = x + row * ldx;
        float v[ELEMS], s[1] = {0.0f};
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const uint32_t c = (i * kGroup + t) * VEC;
            if (c < dim) {
                unpack<T, VEC>(load_pack<T, VEC>(xr + c), v + i * VEC);
#pragma unroll
                for (int j = 0; j < VEC; ++j) s[0] += v[i * VEC + j];
            }
        }
        group_sum<1, WARP, THREADS>(s, smem, 0);
        const float mu = s[0] * inv_dim;
        s[0] = 0.0f;
#pragma unroll
        for (int i = 0; i < kItems; ++i)
            if ((i * kGroup + t) * VEC < dim) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    v[i * VEC + j] -= mu;
                    s[0] = fmaf(v[i * VEC + j], v[i * VEC + j], s[0]);
                }
            }
        group_sum<1, WARP, THREADS>(s, smem, 1);
        const float r = 1.0f / sqrtf(s[0] * inv_dim + eps);
        if (t == 0) {
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = r;
        }
        T* yr = y + row * ldy;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const uint32_t c = (i * kGroup + t) * VEC;
            if (c < dim) {
#pragma unroll
                for (int j = 0; j < VEC; ++j)
                    v[i * VEC + j] = fmaf(v[i * VEC + j] * r, ga[i * VEC + j], be[i * VEC + j]);
                store_pack<T, VEC>(yr + c, v + i * VEC);
            }
        }
    }
}

// Rows too long for registers: the CTA walks over the row three times; the second and third walk find it in L2.
template <typename T>
__global__ void __launch_bounds__(1024) ln_forward_long_kernel(const T* __restrict__ x, uint64_t ldx, uint32_t rows,
                                                               uint32_t dim, const float* __restrict__ gamma,
                                                               const float* __restrict__ beta, float eps,
                                                               T* __restrict__ y, uint64_t ldy,
                                                               float* __restrict__ mean, float* __restrict__ rstd) {
    __shared__ float smem[2][1][32];
    for (uint64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T* xr = x + row * ldx;
        float s[1] = {0.0f};
        for (uint32_t c = threadIdx.x; c < dim; c += 1024) s[0] += to_f32(xr[c]);
        group_sum<1, false, 1024>(s, smem, 0);
        const float mu = s[0] / (float)dim;
        s[0] = 0.0f;
        for (uint32_t c = threadIdx.x; c < dim; c += 1024) {
            const float d = to_f32(xr[c]) - mu;
            s[0] = fmaf(d, d, s[0]);
        }
        group_sum<1, false, 1024>(s, smem, 1);
        const float r = 1.0f / sqrtf(s[0] / (float)dim + eps);
        if (threadIdx.x == 0) {
            if (mean) mean[row] = mu;
            if (rstd) rstd[row] = r;
        }
        for (uint32_t c = threadIdx.x; c < dim; c += 1024) {
            const float h = (to_f32(xr[c]) - mu) * r;
            y[row * ldy + c] = from_f32<T>(fmaf(h, gamma ? __ldg(gamma + c) : 1.0f, beta ? __ldg(beta + c) : 0.0f));
        }
    }
}

// parts: [gridDim.x][2][dim] partial column sums of dy h and dy, or NULL.
template <typename T, int VEC, int ELEMS, int THREADS, bool WARP>
__global__ void __launch_bounds__(THREADS) ln_backward_kernel(const T* __restrict__ dy, uint64_t lddy,
                                                              const T* __restrict__ x, uint64_t ldx, uint32_t rows,
                                                              uint32_t dim, const float* __restrict__ gamma,
                                                              const float* __restrict__ mean,
                                                              const float* __restrict__ rstd, T* __restrict__ dx,
                                                              uint64_t lddx, float* __restrict__ parts) {
    constexpr int kGroup = WARP ? 32 : THREADS, kItems = ELEMS / VEC;
    __shared__ float smem[2][2][32];
    const uint32_t t = WARP ? (threadIdx.x & 31) : threadIdx.x;
    const uint32_t group = WARP ? (threadIdx.x >> 5) : 0, groups = THREADS / kGroup;
    const float inv_dim = 1.0f / (float)dim;
    float ga[ELEMS], sum_h[ELEMS], sum_1[ELEMS];
#pragma unroll
    for (int i = 0; i < kItems; ++i)
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const uint32_t c = (i * kGroup + t) * VEC + j;
            ga[i * VEC + j] = (gamma && c < dim) ? __ldg(gamma + c) : 1.0f;
            sum_h[i * VEC + j] = sum_1[i * VEC + j] = 0.0f;
        }
    int slot = 0;
    for (uint64_t row = (uint64_t)blockIdx.x * groups + group; row < rows; row += (uint64_t)gridDim.x * groups) {
        const T *xr = x + row * ldx, *dyr = dy + row * lddy;
        const float mu = __ldg(mean + row), r = __ldg(rstd + row);
        float h[ELEMS], g[ELEMS], s[2] = {0.0f, 0.0f};
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const uint32_t c = (i * kGroup + t) * VEC;
            if (c < dim) {
                unpack<T, VEC>(load_pack<T, VEC>(xr + c), h + i * VEC);
                unpack<T, VEC>(load_pack<T, VEC>(dyr + c), g + i * VEC);
            }
        }
#pragma unroll
        for (int i = 0; i < kItems; ++i)
            if ((i * kGroup + t) * VEC < dim) {
#pragma unroll
                for (int e = i * VEC; e < (i + 1) * VEC; ++e) {
                    h[e] = (h[e] - mu) * r;
                    sum_h[e] = fmaf(g[e], h[e], sum_h[e]);
                    sum_1[e] += g[e];
                    g[e] *= ga[e];
                    s[0] += g[e];
                    s[1] = fmaf(g[e], h[e], s[1]);
                }
            }
        group_sum<2, WARP, THREADS>(s, smem, slot);
        slot ^= 1;
        const float a = s[0] * inv_dim, b = s[1] * inv_dim;
        T* dxr = dx + row * lddx;
#pragma unroll
        for (int i = 0; i < kItems; ++i) {
            const uint32_t c = (i * kGroup + t) * VEC;
            if (c < dim) {
#pragma unroll
                for (int e = i * VEC; e < (i + 1) * VEC; ++e) g[e] = r * (g[e] - fmaf(h[e], b, a));
                store_pack<T, VEC>(dxr + c, g + i * VEC);
            }
        }
    }
    if (!parts) return;
    float* part = parts + (uint64_t)blockIdx.x * 2 * dim;
    if constexpr (WARP) {
        // the warps add their column sums one after the other: a fixed order
        __shared__ float column[2][32 * ELEMS];
        for (uint32_t w = 0; w < groups; ++w) {
            if (w == group) {
#pragma unroll
                for (int i = 0; i < kItems; ++i)
#pragma unroll
                    for (int j = 0; j < VEC; ++j) {
                        const uint32_t c = (i * 32 + t) * VEC + j;
                        column[0][c] = (w ? column[0][c] : 0.0f) + sum_h[i * VEC + j];
                        column[1][c] = (w ? column[1][c] : 0.0f) + sum_1[i * VEC + j];
                    }
            }
            __syncthreads();
        }
        for (uint32_t c = threadIdx.x; c < dim; c += THREADS) {
            part[c] = column[0][c];
            part[dim + c] = column[1][c];
        }
    } else {
#pragma unroll
        for (int i = 0; i < kItems; ++i)
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const uint32_t c = (i * kGroup + t) * VEC + j;
                if (c < dim) {
                    part[c] = sum_h[i * VEC + j];
                    part[dim + c] = sum_1[i * VEC + j];
                }
            }
    }
}

template <typename T>
__global__ void __launch_bounds__(1024) ln_backward_long_kernel(const T* __restrict__ dy, uint64_t lddy,
                                                                const T* __restrict__ x, uint64_t ldx, uint32_t rows,
                                                                uint32_t dim, const float* __restrict__ gamma,
                                                                const float* __restrict__ mean,
                                                                const float* __restrict__ rstd, T* __restrict__ dx,
                                                                uint64_t lddx) {
    __shared__ float smem[2][2][32];
    int slot = 0;
    for (uint64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const T *xr = x + row * ldx, *dyr = dy + row * lddy;
        const float mu = __ldg(mean + row), r = __ldg(rstd + row);
        float s[2] = {0.0f, 0.0f};
        for (uint32_t c = threadIdx.x; c < dim; c += 1024) {
            const float g = to_f32(dyr[c]) * (gamma ? __ldg(gamma + c) : 1.0f);
            s[0] += g;
            s[1] = fmaf(g, (to_f32(xr[c]) - mu) * r, s[1]);
        }
        group_sum<2, false, 1024>(s, smem, slot);
        slot ^= 1;
        const float a = s[0] / (float)dim, b = s[1] / (float)dim;
        for (uint32_t c = threadIdx.x; c < dim; c += 1024) {
            const float g = to_f32(dyr[c]) * (gamma ? __ldg(gamma + c) : 1.0f), h = (to_f32(xr[c]) - mu) * r;
            dx[row * lddx + c] = from_f32<T>(r * (g - fmaf(h, b, a)));
        }
    }
}

// Partial column sums of rows too long for registers: CTA (x, y) takes 256 columns and every gridDim.y-th row.
template <typename T>
__global__ void __launch_bounds__(256) ln_columns_long_kernel(const T* __restrict__ dy, uint64_t lddy,
                                                              const T* __restrict__ x, uint64_t ldx, uint32_t rows,
                                                              uint32_t dim, const float* __restrict__ mean,
                                                              const float* __restrict__ rstd,
                                                              float* __restrict__ parts) {
    const uint32_t c = blockIdx.x * 256 + threadIdx.x;
    if (c >= dim) return;
    float sh = 0.0f, s1 = 0.0f;
    for (uint64_t row = blockIdx.y; row < rows; row += gridDim.y) {
        const float g = to_f32(dy[row * lddy + c]);
        sh = fmaf(g, (to_f32(x[row * ldx + c]) - __ldg(mean + row)) * __ldg(rstd + row), sh);
        s1 += g;
    }
    float* part = parts + (uint64_t)blockIdx.y * 2 * dim;
    part[c] = sh;
    part[dim + c] = s1;
}

// Adds the rows of partial sums: 32 columns a CTA, 8 warps take every eighth row each.
__global__ void __launch_bounds__(256) ln_reduce_kernel(const float* __restrict__ parts, uint32_t count, uint32_t dim,
                                                        float* __restrict__ dgamma, float* __restrict__ dbeta,
                                                        bool accumulate) {
    __shared__ float smem[8][32];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t c = blockIdx.x * 32 + lane;       // of the 2 dim columns of a row of parts
    const uint32_t width = 2 * dim;
    float s = 0.0f;
    if (c < width)
        for (uint32_t p = warp; p < count; p += 8) s += parts[(uint64_t)p * width + c];
    smem[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && c < width) {
        s = smem[0][lane];
#pragma unroll
        for (int w = 1; w < 8; ++w) s += smem[w][lane];
        float* out = c < dim ? dgamma : dbeta;
        const uint32_t i = c < dim ? c : c - dim;
        if (out) out[i] = accumulate ? out[i] + s : s;
    }
}

// Calls f.template operator()<ELEMS, THREADS, WARP>() for the shortest group that holds a row of dim elements.
template <typename F>
slimdp_status with_shape(uint64_t dim, F&& f) {
    if (dim <= 256) return f.template operator()<8, 256, true>();
    if (dim <= 512) return f.template operator()<16, 256, true>();
    if (dim <= 1024) return f.template operator()<32, 256, true>();
    if (dim <= 2048) return f.template operator()<8, 256, false>();
    if (dim <= 4096) return f.template operator()<16, 256, false>();
    if (dim <= 8192) return f.template operator()<16, 512, false>();
    return f.template operator()<16, 1024, false>();
}

template <typename T>
struct LnForward {
    const T* x; uint64_t ldx; uint32_t rows, dim; const float *gamma, *beta; float eps; T* y; uint64_t ldy;
    float *mean, *rstd; bool vec; cudaStream_t st;

    template <int ELEMS, int THREADS, bool WARP>
    slimdp_status operator()() const {
        const uint32_t groups = WARP ? THREADS / 32 : 1;
        const uint32_t ctas = (uint32_t)std::min<uint64_t>(((uint64_t)rows + groups - 1) / groups, (uint64_t)sm_count() * (2048 / THREADS));
        if (vec)
            ln_forward_kernel<T, kVec<T>, ELEMS, THREADS, WARP><<<ctas, THREADS, 0, st>>>(x, ldx, rows, dim, gamma, beta, eps, y, ldy, mean, rstd);
        else
            ln_forward_kernel<T, 1, ELEMS, THREADS, WARP><<<ctas, THREADS, 0, st>>>(x, ldx, rows, dim, gamma, beta, eps, y, ldy, mean, rstd);
        SLIMDP_LAUNCHED(1);
        return SLIMDP_OK;
    }
};

template <typename T>
struct LnBackward {
    const T* dy; uint64_t lddy; const T* x; uint64_t ldx; uint32_t rows, dim; const float *gamma, *mean, *rstd; T* dx;
    uint64_t lddx; float* parts; bool vec; cudaStream_t st; uint32_t* count;

    template <int ELEMS, int THREADS, bool WARP>
    slimdp_status operator()() const {
        const uint32_t groups = WARP ? THREADS / 32 : 1;
        const uint32_t ctas = (uint32_t)std::min<uint64_t>(((uint64_t)rows + groups - 1) / groups, std::min<uint64_t>(kLnMaxParts, (uint64_t)sm_count() * (1024 / THREADS)));
        *count = ctas;
        if (vec)
            ln_backward_kernel<T, kVec<T>, ELEMS, THREADS, WARP><<<ctas, THREADS, 0, st>>>(dy, lddy, x, ldx, rows, dim, gamma, mean, rstd, dx, lddx, parts);
        else
            ln_backward_kernel<T, 1, ELEMS, THREADS, WARP><<<ctas, THREADS, 0, st>>>(dy, lddy, x, ldx, rows, dim, gamma, mean, rstd, dx, lddx, parts);
        SLIMDP_LAUNCHED(1);
        return SLIMDP_OK;
    }
};

}  // namespace

size_t layernorm_ws_bytes(uint64_t rows, uint64_t dim) {
    return align_up(std::max<uint64_t>(1, std::min<uint64_t>(rows, kLnMaxParts)) * 2 * dim * sizeof(float), 16);
}

slimdp_status launch_layernorm_forward(const void* x, uint64_t ldx, uint32_t rows, uint32_t dim, int32_t type,
                                       const float* gamma, const float* beta, float eps, void* y, uint64_t ldy,
                                       float* mean, float* rstd, cudaStream_t st) {
    const bool vec = rows_vectorise(x, ldx, dim, type) && rows_vectorise(y, ldy, dim, type);
    return with_type(type, [&](auto e) -> slimdp_status {
        using T = decltype(e);
        if (dim > kLnRegisterDim) {
            const uint32_t ctas = (uint32_t)std::min<uint64_t>(rows, (uint64_t)sm_count() * 2);
            ln_forward_long_kernel<T><<<ctas, 1024, 0, st>>>((const T*)x, ldx, rows, dim, gamma, beta, eps, (T*)y, ldy, mean, rstd);
            SLIMDP_LAUNCHED(1);
            return SLIMDP_OK;
        }
        return with_shape(dim, LnForward<T>{(const T*)x, ldx, rows, dim, gamma, beta, eps, (T*)y, ldy, mean, rstd, vec, st});
    });
}

slimdp_status launch_layernorm_backward(const void* dy, uint64_t lddy, const void* x, uint64_t ldx, uint32_t rows,
                                        uint32_t dim, int32_t type, const float* gamma, const float* mean,
                                        const float* rstd, void* dx, uint64_t lddx, float* dgamma, float* dbeta,
                                        bool accumulate, void* ws, cudaStream_t st) {
    const bool vec = rows_vectorise(x, ldx, dim, type) && rows_vectorise(dy, lddy, dim, type) && rows_vectorise(dx, lddx, dim, type);
    float* parts = (dgamma || dbeta) ? (float*)ws : nullptr;
    uint32_t count = 0;
    if (rows > 0) {
        const slimdp_status s = with_type(type, [&](auto e) -> slimdp_status {
            using T = decltype(e);
            if (dim > kLnRegisterDim) {
                const uint32_t ctas = (uint32_t)std::min<uint64_t>(rows, (uint64_t)sm_count() * 2);
                ln_backward_long_kernel<T><<<ctas, 1024, 0, st>>>((const T*)dy, lddy, (const T*)x, ldx, rows, dim, gamma, mean, rstd, (T*)dx, lddx);
                SLIMDP_LAUNCHED(1);
                if (parts) {
                    count = std::min<uint32_t>(rows, 32);
                    ln_columns_long_kernel<T><<<dim3((dim + 255) / 256, count), 256, 0, st>>>((const T*)dy, lddy, (const T*)x, ldx, rows, dim, mean, rstd, parts);
                    SLIMDP_LAUNCHED(1);
                }
                return SLIMDP_OK;
            }
            return with_shape(dim, LnBackward<T>{(const T*)dy, lddy, (const T*)x, ldx, rows, dim, gamma, mean, rstd, (T*)dx, lddx, parts, vec, st, &count});
        });
        if (s != SLIMDP_OK) return s;
    }
    if (parts) {
        ln_reduce_kernel<<<(unsigned)((2 * (uint64_t)dim + 31) / 32), 256, 0, st>>>(parts, count, dim, dgamma, dbeta, accumulate);
        SLIMDP_LAUNCHED(1);
    }
    return SLIMDP_OK;
}

}  // namespace slimdp
