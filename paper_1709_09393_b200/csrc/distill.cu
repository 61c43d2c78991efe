// Distillation from a teacher's top logits, with hard labels beside them: loss and gradient of each row.
//
// With T the temperature, p^T = softmax(s / T), p = softmax(s) and q the softmax of the teacher's entries / T:
//   loss = w ( kd T^2 sum_j q_j (log q_j - log p^T[i_j]) - ce log p[y] )
//   ds_i = w ( kd T (Q p^T_i - sum over j with i_j = i of q_j) + ce (p_i - [i = y]) ),  Q = sum_j q_j = 1 or 0.
// Everywhere but at the teacher's entries and at the label the gradient is a multiple of the two softmaxes, so one
// walk over the row yields the maximum and the two sums (kept relative to a running maximum, rescaled
// where that rises) and a second walk writes the gradient; the few entries that have a term of their own are computed
// from logits set aside before the second walk and stored after it, so that each result is rounded once.
#include <algorithm>
#include <math.h>

#include "train.cuh"

namespace slimdp {

namespace {

constexpr int kDistillThreads = 512;
constexpr int kDistillWarps = kDistillThreads / 32;

// A softmax in the making: sums of 2^((s - m) c) relative to the maximum m.
struct SoftSums {
    float m, at_t, at_1;
};

__device__ __forceinline__ SoftSums join(SoftSums a, SoftSums b, float c_t, float c_1) {
    SoftSums r;
    r.m = fmaxf(a.m, b.m);
    // a side without a finite logit has sums 0 (or NaN, which stays): its factor is 1 to keep -inf - -inf out
    const float fa = a.m == -INFINITY ? 0.0f : a.m - r.m, fb = b.m == -INFINITY ? 0.0f : b.m - r.m;
    r.at_t = a.at_t * exp2_approx(fa * c_t) + b.at_t * exp2_approx(fb * c_t);
    r.at_1 = a.at_1 * exp2_approx(fa * c_1) + b.at_1 * exp2_approx(fb * c_1);
    return r;
}

__device__ __forceinline__ float load_teacher(const void* p, int32_t type, uint64_t i) {
    if (type == SLIMDP_F32) return ((const float*)p)[i];
    if (type == SLIMDP_BF16) return to_f32(((const __nv_bfloat16*)p)[i]);
    return to_f32(((const __half*)p)[i]);
}

__device__ __forceinline__ float block_sum(float v, float* smem) {
    v = warp_sum(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < kDistillWarps; ++w) s += smem[w];
    return s;
}

__device__ __forceinline__ float block_max(float v, float* smem) {
    v = warp_max(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = -INFINITY;
#pragma unroll
    for (int w = 0; w < kDistillWarps; ++w) s = fmaxf(s, smem[w]);
    return s;
}

struct DistillArgs {
    uint64_t ldl, ldd;
    uint32_t rows, vocab, top;
    const int32_t* idx;
    const void* teacher;
    int32_t teacher_type;
    const int32_t* label;
    const float* weight;
    float temperature, kd, ce;
    float* loss;
};

// Calls f(c, count) for the elements of a row of n that thread t owns: a head and a tail of single elements, and
// 16-byte pieces from the first 16-byte boundary of p on.
template <typename T, typename Scalar, typename Vector>
__device__ __forceinline__ void walk_row(const T* p, uint32_t n, Scalar&& scalar, Vector&& vector) {
    constexpr uint32_t V = kVec<T>;
    const uint32_t off = (uint32_t)((reinterpret_cast<uintptr_t>(p) & 15u) / sizeof(T));
    const uint32_t head = min(n, off ? V - off : 0u), pieces = (n - head) / V, tail = head + pieces * V;
    for (uint32_t i = threadIdx.x; i < pieces; i += kDistillThreads) vector(head + i * V);
    if (threadIdx.x < head) scalar(threadIdx.x);
    if (threadIdx.x < n - tail) scalar(tail + threadIdx.x);
}

template <typename T>
__global__ void __launch_bounds__(kDistillThreads) distill_kernel(const T* logits, T* dlogits, DistillArgs a) {
    constexpr int V = kVec<T>;
    __shared__ float red[kDistillWarps];
    __shared__ SoftSums red_soft[kDistillWarps];
    __shared__ int32_t s_idx[SLIMDP_MAX_TOP];
    __shared__ float s_q[SLIMDP_MAX_TOP], s_fix[SLIMDP_MAX_TOP];
    const uint32_t row = blockIdx.x, tid = threadIdx.x;
    const T* z = logits + row * a.ldl;
    T* out = dlogits ? dlogits + row * a.ldd : nullptr;
    const float w = a.weight ? __ldg(a.weight + row) : 1.0f;
    const int32_t y = a.label ? __ldg(a.label + row) : -1;
    const bool has_label = a.ce != 0.0f && y >= 0 && (uint32_t)y < a.vocab;

    // the teacher's softmax over the entries that are there
    float tmax = -INFINITY;
    bool any = false;
    if (a.kd != 0.0f)
        for (uint32_t j = tid; j < a.top; j += kDistillThreads) {
            const int32_t i = a.idx[(uint64_t)row * a.top + j];
            const bool there = i >= 0 && (uint32_t)i < a.vocab;
            const float t = there ? load_teacher(a.teacher, a.teacher_type, (uint64_t)row * a.top + j) : -INFINITY;
            s_idx[j] = there ? i : -1;
            s_q[j] = t;
            any |= t != -INFINITY;
            tmax = fmaxf(tmax, t);
        }
    const bool has_teacher = __syncthreads_or(any);
    const float c_t = kLog2e / a.temperature, c_1 = kLog2e;

    if (w == 0.0f || (!has_teacher && !has_label)) {
        if (out)
            walk_row(out, a.vocab, [&](uint32_t c) { out[c] = from_f32<T>(0.0f); },
                     [&](uint32_t c) {
                         float v[V] = {};
                         store_pack<T, V>(out + c, v);
                     });
        if (tid == 0) a.loss[row] = 0.0f;
        return;
    }

    // first walk
    SoftSums s = {-INFINITY, 0.0f, 0.0f};
    auto take = [&](const float* v, int count) {
        float top = v[0];
        for (int i = 1; i < count; ++i) top = fmaxf(top, v[i]);
        if (top > s.m) {
            const float f = s.m - top;      // -inf on the first logit: the sums are 0 then, or NaN
            s.at_t *= exp2_approx(f * c_t);
            s.at_1 *= exp2_approx(f * c_1);
            s.m = top;
        }
        const float m = s.m == -INFINITY ? 0.0f : s.m;
        for (int i = 0; i < count; ++i) {
            if (has_teacher) s.at_t += exp2_approx((v[i] - m) * c_t);
            if (has_label) s.at_1 += exp2_approx((v[i] - m) * c_1);
        }
    };
    walk_row(z, a.vocab,
             [&](uint32_t c) {
                 const float v = to_f32(z[c]);
                 take(&v, 1);
             },
             [&](uint32_t c) {
                 float v[V];
                 unpack<T, V>(load_pack<T, V>(z + c), v);
                 take(v, V);
             });
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1) {
        SoftSums o = {__shfl_xor_sync(0xFFFFFFFFu, s.m, d), __shfl_xor_sync(0xFFFFFFFFu, s.at_t, d),
                      __shfl_xor_sync(0xFFFFFFFFu, s.at_1, d)};
        s = join(s, o, c_t, c_1);
    }
    if ((tid & 31) == 0) red_soft[tid >> 5] = s;
    __syncthreads();
    s = red_soft[0];
#pragma unroll
    for (int i = 1; i < kDistillWarps; ++i) s = join(s, red_soft[i], c_t, c_1);

    const float m = s.m == -INFINITY ? 0.0f : s.m;
    const bool empty = has_teacher ? s.at_t == 0.0f : s.at_1 == 0.0f;   // nothing but -inf
    const float log_t = logf(s.at_t), log_1 = logf(s.at_1);
    const float scale = empty ? 0.0f : w;
    // gradient = g_t 2^((s - m) c_t) + g_1 2^((s - m) c_1), less the terms of single entries
    const float g_t = has_teacher && !empty ? scale * a.kd * a.temperature / s.at_t : 0.0f;
    const float g_1 = has_label && !empty ? scale * a.ce / s.at_1 : 0.0f;
    auto dense = [&](float v) {
        float g = 0.0f;
        if (has_teacher) g = g_t * exp2_approx((v - m) * c_t);
        if (has_label) g = fmaf(g_1, exp2_approx((v - m) * c_1), g);
        return empty ? 0.0f : g;
    };

    // the teacher's term of the loss, and the gradient where it has an entry
    float loss = 0.0f;
    if (has_teacher) {
        tmax = block_max(tmax, red);
        float sum = 0.0f;
        for (uint32_t j = tid; j < a.top; j += kDistillThreads) sum += exp2_approx((s_q[j] - tmax) * c_t);
        const float total = block_sum(sum, red);
        // T (log q_j - log p^T) with the temperature multiplied out: (s - m) / T would overflow for the lowest
        // values that masks put in place of logits
        const float shift = a.temperature * (log_t - logf(total));
        for (uint32_t j = tid; j < a.top; j += kDistillThreads) {
            const float t = s_q[j] - tmax, q = exp2_approx(t * c_t) / total;
            s_q[j] = q;
            if (s_idx[j] >= 0) {
                const float v = to_f32(z[s_idx[j]]);
                s_fix[j] = dense(v);
                if (q != 0.0f) loss += q * (t - (v - m) + shift);
            }
        }
        loss = block_sum(loss, red) * a.kd * a.temperature;
    }
    float label_fix = 0.0f;
    if (has_label) {
        const float v = to_f32(z[y]);
        label_fix = dense(v) - scale * a.ce;
        loss += a.ce * (log_1 - (v - m));
    }
    if (tid == 0) a.loss[row] = empty ? 0.0f : w * loss;
    if (!out) return;
    __syncthreads();

    // second walk, then the entries of their own
    walk_row(z, a.vocab, [&](uint32_t c) { out[c] = from_f32<T>(dense(to_f32(z[c]))); },
             [&](uint32_t c) {
                 float v[V];
                 unpack<T, V>(load_pack<T, V>(z + c), v);
#pragma unroll
                 for (int i = 0; i < V; ++i) v[i] = dense(v[i]);
                 if ((reinterpret_cast<uintptr_t>(out + c) & 15u) == 0) {
                     store_pack<T, V>(out + c, v);
                 } else {
#pragma unroll
                     for (int i = 0; i < V; ++i) out[c + i] = from_f32<T>(v[i]);
                 }
             });
    __syncthreads();
    bool label_done = !has_label;
    if (has_teacher)
        for (uint32_t j = tid; j < a.top; j += kDistillThreads) {
            const int32_t i = s_idx[j];
            if (i < 0) continue;
            float q = 0.0f;
            bool first = true;
            for (uint32_t k = 0; k < a.top; ++k)
                if (s_idx[k] == i) {
                    q += s_q[k];
                    first = first && k >= j;
                }
            if (!first) continue;     // the first of the entries that share an index stores their sum
            float g = s_fix[j] - scale * a.kd * a.temperature * q;
            if (has_label && i == y) g -= scale * a.ce;
            out[i] = from_f32<T>(g);
        }
    if (has_label && has_teacher)
        for (uint32_t k = tid; k < a.top; k += kDistillThreads) label_done |= s_idx[k] == y;
    label_done = has_label ? __syncthreads_or(label_done) : true;
    if (tid == 0 && !label_done) out[y] = from_f32<T>(label_fix);
}

}  // namespace

slimdp_status launch_distill(const void* logits, uint64_t ldl, uint32_t rows, uint32_t vocab, int32_t type,
                             const int32_t* idx, const void* teacher, int32_t teacher_type, uint32_t top,
                             const int32_t* label, const float* weight, float temperature, float kd, float ce,
                             float* loss, void* dlogits, uint64_t ldd, cudaStream_t st) {
    if (rows == 0) return SLIMDP_OK;
    const DistillArgs a = {ldl, ldd, rows, vocab, top, idx, teacher, teacher_type, label, weight, temperature, kd, ce, loss};
    return with_type(type, [&](auto e) -> slimdp_status {
        using T = decltype(e);
        distill_kernel<T><<<rows, kDistillThreads, 0, st>>>((const T*)logits, (T*)dlogits, a);
        SLIMDP_LAUNCHED(1);
        return SLIMDP_OK;
    });
}

}  // namespace slimdp
