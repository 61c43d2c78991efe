// The forward product of up to eight rows, as single tokens make it, on the ordinary cores.
//
// Bound by reading w [n, k] once: warps walk over its rows in 16-byte pieces, the rows of x stay in L1.  fp32 is multiplied as it
// is.  Sums run over the summed axis in a fixed order, so that results do not depend on scheduling.  One row of 16384 x 8192 fp32
// 84 us (6.4 TB/s), bf16 45 us (5.9 TB/s); eight rows 188 and 123 us, bound by what sixteen warps an SM keep on its way.  Five
// rows of 4096 x 1024 fp16 6.6 us.
#include <algorithm>

#include "epilogue.cuh"

namespace slimdp {

namespace {

constexpr int kColumns = 4;            // outputs of a warp, forward

// N sums over a warp, N a power of two: value i ends in every lane l with l % N = i.  Halves are exchanged and added, N - 1
// exchanges and log2(32 / N) more instead of 5 N.
template <int N>
__device__ __forceinline__ float warp_sums(float (&v)[N], uint32_t lane) {
#pragma unroll
    for (int d = N / 2; d >= 1; d >>= 1) {
        const bool upper = lane & d;
#pragma unroll
        for (int i = 0; i < d; ++i) {
            const float keep = upper ? v[i + d] : v[i], send = upper ? v[i] : v[i + d];
            v[i] = keep + __shfl_xor_sync(0xFFFFFFFFu, send, d);
        }
    }
#pragma unroll
    for (int d = N; d < 32; d <<= 1) v[0] += __shfl_xor_sync(0xFFFFFFFFu, v[0], d);
    return v[0];
}

// y = act(x w^T + bias) + residual: a warp makes M x 4 dot products over every (1 << split)-th stretch of 32 pieces; the warps
// of a CTA that share outputs add theirs.  16-byte pieces where the rows allow, else pairs or single elements.
template <typename T, int V, int M>
__global__ void __launch_bounds__(256) few_forward_kernel(const T* __restrict__ x, uint64_t ldx, const T* __restrict__ w,
                                                          uint64_t ldw, uint32_t m, uint64_t n, uint64_t k, uint32_t split,
                                                          const Epilogue e) {
    constexpr int N = M * kColumns;
    // Two and four rows of fp32 ask for the pieces of w two steps ahead: 16384 x 8192 99 and 102 us, 145 and 138 without.  One row (108 to
    // 85) and eight (300 to 188) are better off without, by more loads in flight and by more warps.
    constexpr bool kTwoAhead = sizeof(T) == 4 && V > 1 && (M == 2 || M == 4);
    __shared__ float sums[8][N];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, ways = 1u << split, way = warp & (ways - 1);
    const uint64_t j0 = ((uint64_t)blockIdx.x * (8 >> split) + (warp >> split)) * kColumns;
    const T *wr[kColumns], *xr[M];
#pragma unroll
    for (int c = 0; c < kColumns; ++c) wr[c] = w + min(j0 + c, n - 1) * ldw;       // a row beyond the last is not stored
#pragma unroll
    for (int i = 0; i < M; ++i) xr[i] = x + min((uint32_t)i, m - 1) * ldx;
    // sums of the even and of the odd elements; more of them would not fit the registers of eight rows
    using Acc = Vals<V == 1 ? 1 : 2>;
    Acc acc[M][kColumns];
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
        for (int c = 0; c < kColumns; ++c) acc[i][c] = Acc::splat(0.0f);
    const uint64_t pieces = k / V;
    const uint64_t first = way * 32 + lane, step = ways * 32;
    auto multiply = [&](const Vals<V>(&a)[kColumns], uint64_t p) {
#pragma unroll
        for (int i = 0; i < M; ++i) {
            const Vals<V> b = Vals<V>::of(load_pack<T, V>(xr[i] + p * V));
#pragma unroll
            for (int c = 0; c < kColumns; ++c)
#pragma unroll
                for (int u = 0; u < (V + 1) / 2; ++u) acc[i][c].p[0] = fma_pair(a[c].p[u], b.p[u], acc[i][c].p[0]);
        }
    };
    if constexpr (kTwoAhead) {
        Pack<T, V> next[2][kColumns];
        auto fetch = [&](int slot, uint64_t p) {
#pragma unroll
            for (int c = 0; c < kColumns; ++c)
                if (p < pieces) next[slot][c] = load_pack<T, V>(wr[c] + p * V);
        };
        fetch(0, first);
        fetch(1, first + step);
        for (uint64_t p = first; p < pieces; p += 2 * step)
#pragma unroll
            for (int u = 0; u < 2; ++u)
                if (p + u * step < pieces) {
                    Vals<V> a[kColumns];
#pragma unroll
                    for (int c = 0; c < kColumns; ++c) a[c] = Vals<V>::of(next[u][c]);
                    fetch(u, p + (u + 2) * step);
                    multiply(a, p + u * step);
                }
    } else {
#pragma unroll 2
        for (uint64_t p = first; p < pieces; p += step) {
            Vals<V> a[kColumns];
#pragma unroll
            for (int c = 0; c < kColumns; ++c) a[c] = Vals<V>::of(load_pack<T, V>(wr[c] + p * V));
            multiply(a, p);
        }
    }
    float v[N];
#pragma unroll
    for (int i = 0; i < M; ++i)
#pragma unroll
        for (int c = 0; c < kColumns; ++c) v[i * kColumns + c] = acc[i][c].sum();
    if (V > 1 && way == 0 && pieces * V + lane < k) {
        const uint64_t l = pieces * V + lane;
#pragma unroll
        for (int i = 0; i < M; ++i)
#pragma unroll
            for (int c = 0; c < kColumns; ++c) v[i * kColumns + c] = fmaf(to_f32(xr[i][l]), to_f32(wr[c][l]), v[i * kColumns + c]);
    }
    const float s = warp_sums<N>(v, lane);
    if (lane < N) sums[warp][lane] = s;
    __syncthreads();
    if (way != 0 || lane >= N) return;
    float one[1][1] = {{s}};
    for (uint32_t o = 1; o < ways; ++o) one[0][0] += sums[warp + o][lane];
    const uint64_t i = lane / kColumns, j = j0 + lane % kColumns;
    if (i >= m || j >= n) return;
    const float bias[1] = {e.bias ? __ldg(e.bias + j) : 0.0f};
    Extra<T, kForward, 1> extra[1];
    extra[0].load(e, i, j);
    finish<T, kForward, 1, 1>(e, i, 0, 1, j, one, bias, extra);
}

}  // namespace

template <typename T>
slimdp_status launch_few_forward(const T* x, uint64_t ldx, const T* w, uint64_t ldw, uint64_t m, uint64_t n, uint64_t k,
                                 const Epilogue& e, cudaStream_t st) {
    auto fits = [&](uint64_t v) {        // rows of pieces of v elements
        const uint64_t bytes = v * sizeof(T);
        return (uintptr_t)x % bytes == 0 && (uintptr_t)w % bytes == 0 && (n == 1 || ldw % v == 0) && (m == 1 || ldx % v == 0);
    };
    // Rows of a 16-bit type on 4-byte boundaries go by pairs, up to four of them: two rows of 14665 x 9492 bf16 121 us, 237 by single
    // elements, one of 4096 x 4098 29 and 61; eight of 4096 x 1002 would take 30, 17.5 by single elements.
    const bool wide = fits(kVec<T>), twos = sizeof(T) == 2 && !wide && m <= 4 && fits(2);
    const uint64_t warps = (n + kColumns - 1) / kColumns, stretches = k / (wide ? kVec<T> : twos ? 2 : 1) / 32;
    const int sms = sm_count();
    if (sms <= 0) return SLIMDP_ERR_CUDA;
    // more warps an output only while there are fewer than eight an SM and each has a stretch
    uint32_t split = 0;
    while (split < 3 && (warps << split) < 8ull * sms && (stretches >> (split + 1)) > 0) ++split;
    const unsigned ctas = (unsigned)(((warps << split) + 7) / 8);
    return with_rows(m, [&](auto rows) -> slimdp_status {
        constexpr int M = decltype(rows)::value;
        if (wide)
            few_forward_kernel<T, kVec<T>, M><<<ctas, 256, 0, st>>>(x, ldx, w, ldw, (uint32_t)m, n, k, split, e);
        else if (twos) {
            if constexpr (sizeof(T) == 2 && M <= 4) few_forward_kernel<T, 2, M><<<ctas, 256, 0, st>>>(x, ldx, w, ldw, (uint32_t)m, n, k, split, e);
        } else
            few_forward_kernel<T, 1, M><<<ctas, 256, 0, st>>>(x, ldx, w, ldw, (uint32_t)m, n, k, split, e);
        SLIMDP_LAUNCHED(1);
        return SLIMDP_OK;
    });
}

template slimdp_status launch_few_forward<float>(const float*, uint64_t, const float*, uint64_t, uint64_t, uint64_t, uint64_t,
                                                 const Epilogue&, cudaStream_t);
template slimdp_status launch_few_forward<__nv_bfloat16>(const __nv_bfloat16*, uint64_t, const __nv_bfloat16*, uint64_t,
                                                         uint64_t, uint64_t, uint64_t, const Epilogue&, cudaStream_t);
template slimdp_status launch_few_forward<__half>(const __half*, uint64_t, const __half*, uint64_t, uint64_t, uint64_t, uint64_t,
                                                  const Epilogue&, cudaStream_t);

}  // namespace slimdp
