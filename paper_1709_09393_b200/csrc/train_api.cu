// The exported calls of a worker's local step: argument validation and workspace sizing; the launches are
// in layernorm.cu, linear.cu and distill.cu.
#include <math.h>

#include "train.cuh"

namespace slimdp {

size_t layernorm_ws_bytes(uint64_t rows, uint64_t dim);
slimdp_status launch_layernorm_forward(const void* x, uint64_t ldx, uint32_t rows, uint32_t dim, int32_t type,
                                       const float* gamma, const float* beta, float eps, void* y, uint64_t ldy,
                                       float* mean, float* rstd, cudaStream_t st);
slimdp_status launch_layernorm_backward(const void* dy, uint64_t lddy, const void* x, uint64_t ldx, uint32_t rows,
                                        uint32_t dim, int32_t type, const float* gamma, const float* mean,
                                        const float* rstd, void* dx, uint64_t lddx, float* dgamma, float* dbeta,
                                        bool accumulate, void* ws, cudaStream_t st);
size_t linear_ws_bytes(uint64_t m, uint64_t n, uint64_t k, int32_t type);
slimdp_status launch_linear_forward(const void* x, uint64_t ldx, const void* w, uint64_t ldw, const float* bias,
                                    const void* residual, uint64_t ldr, uint64_t m, uint64_t n, uint64_t k,
                                    int32_t type, int32_t act, void* y, uint64_t ldy, void* z, uint64_t ldz, void* ws,
                                    cudaStream_t st);
slimdp_status launch_linear_backward_input(const void* dy, uint64_t lddy, const void* w, uint64_t ldw, const void* z,
                                           uint64_t ldz, const void* add, uint64_t ldadd, uint64_t m, uint64_t n,
                                           uint64_t k, int32_t type, int32_t act, void* dx, uint64_t lddx, void* ws,
                                           cudaStream_t st);
slimdp_status launch_linear_backward_weight(const void* dy, uint64_t lddy, const void* x, uint64_t ldx, uint64_t m,
                                            uint64_t n, uint64_t k, int32_t type, float* dw, uint64_t lddw, float* db,
                                            bool accumulate, void* ws, cudaStream_t st);
slimdp_status launch_activation_backward(const void* dy, uint64_t lddy, const void* z, uint64_t ldz, uint64_t m,
                                         uint64_t n, int32_t type, int32_t act, void* dz, uint64_t lddz,
                                         cudaStream_t st);
slimdp_status read_product_status();
slimdp_status read_distill_status();
slimdp_status read_layernorm_status();
slimdp_status launch_distill(const void* logits, uint64_t ldl, uint32_t rows, uint32_t vocab, int32_t type,
                             const int32_t* idx, const void* teacher, int32_t teacher_type, uint32_t top,
                             const int32_t* label, const float* weight, float temperature, float kd, float ce,
                             float* loss, void* dlogits, uint64_t ldd, cudaStream_t st);

namespace {

constexpr uint64_t kMaxDim = 0x7FFFFFFFull;
constexpr uint64_t kMaxLd = 1ull << 40;      // rows of a matrix start below 2^40 elements apart

bool aligned_to(const void* p, size_t b) { return (reinterpret_cast<uintptr_t>(p) & (b - 1)) == 0; }

bool dims_ok(uint64_t rows, uint64_t cols) { return rows <= kMaxDim && cols >= 1 && cols <= kMaxDim; }

// A matrix that has to be there (unless it has no rows).
bool matrix_ok(const void* p, uint64_t ld, uint64_t rows, uint64_t cols, int32_t type) {
    if (ld < cols || ld > kMaxLd) return false;
    return rows == 0 || (p && aligned_to(p, type_bytes(type)));
}

bool matrix_or_null(const void* p, uint64_t ld, uint64_t rows, uint64_t cols, int32_t type) {
    return !p || matrix_ok(p, ld, rows, cols, type);
}

bool vector_or_null(const void* p) { return !p || aligned4(p); }

bool act_ok(int32_t act) { return act >= SLIMDP_ACT_NONE && act <= SLIMDP_ACT_SILU; }

slimdp_status workspace_ok(const void* ws, size_t have, size_t need, size_t align) {
    if (!ws || !aligned_to(ws, align)) return SLIMDP_ERR_INVALID_ARG;
    return have < need ? SLIMDP_ERR_WORKSPACE : SLIMDP_OK;
}

}  // namespace
}  // namespace slimdp

using namespace slimdp;

extern "C" {

size_t slimdp_layernorm_workspace_bytes(uint64_t rows, uint64_t dim) {
    return dims_ok(rows, dim) ? layernorm_ws_bytes(rows, dim) : 0;
}

slimdp_status slimdp_layernorm_forward(const void* x, uint64_t ldx, uint64_t rows, uint64_t dim, int32_t type,
                                       const float* gamma, const float* beta, float eps, void* y, uint64_t ldy,
                                       float* mean, float* rstd, void* stream) {
    if (!type_ok(type) || !dims_ok(rows, dim) || !isfinite(eps) || eps < 0.0f) return SLIMDP_ERR_INVALID_ARG;
    if (!matrix_ok(x, ldx, rows, dim, type) || !matrix_ok(y, ldy, rows, dim, type)) return SLIMDP_ERR_INVALID_ARG;
    if (!vector_or_null(gamma) || !vector_or_null(beta) || !vector_or_null(mean) || !vector_or_null(rstd))
        return SLIMDP_ERR_INVALID_ARG;
    if (rows == 0) return SLIMDP_OK;
    return launch_layernorm_forward(x, ldx, (uint32_t)rows, (uint32_t)dim, type, gamma, beta, eps, y, ldy, mean, rstd,
                                    (cudaStream_t)stream);
}

slimdp_status slimdp_layernorm_backward(const void* dy, uint64_t lddy, const void* x, uint64_t ldx, uint64_t rows,
                                        uint64_t dim, int32_t type, const float* gamma, const float* mean,
                                        const float* rstd, void* dx, uint64_t lddx, float* dgamma, float* dbeta,
                                        int32_t accumulate, void* ws, size_t ws_bytes, void* stream) {
    if (!type_ok(type) || !dims_ok(rows, dim)) return SLIMDP_ERR_INVALID_ARG;
    if (!matrix_ok(dy, lddy, rows, dim, type) || !matrix_ok(x, ldx, rows, dim, type) ||
        !matrix_ok(dx, lddx, rows, dim, type))
        return SLIMDP_ERR_INVALID_ARG;
    if (rows > 0 && (!mean || !rstd)) return SLIMDP_ERR_INVALID_ARG;
    if (!vector_or_null(gamma) || !vector_or_null(mean) || !vector_or_null(rstd) || !vector_or_null(dgamma) ||
        !vector_or_null(dbeta))
        return SLIMDP_ERR_INVALID_ARG;
    if (dgamma || dbeta) {
        const slimdp_status s = workspace_ok(ws, ws_bytes, layernorm_ws_bytes(rows, dim), 16);
        if (s != SLIMDP_OK) return s;
    }
    return launch_layernorm_backward(dy, lddy, x, ldx, (uint32_t)rows, (uint32_t)dim, type, gamma, mean, rstd, dx, lddx,
                                     dgamma, dbeta, accumulate != 0, ws, (cudaStream_t)stream);
}

size_t slimdp_linear_workspace_bytes(uint64_t m, uint64_t n, uint64_t k, int32_t type) {
    return type_ok(type) && dims_ok(m, n) && dims_ok(m, k) ? linear_ws_bytes(m, n, k, type) : 0;
}

slimdp_status slimdp_linear_forward(const void* x, uint64_t ldx, const void* w, uint64_t ldw, const float* bias,
                                    const void* residual, uint64_t ldr, uint64_t m, uint64_t n, uint64_t k,
                                    int32_t type, int32_t act, void* y, uint64_t ldy, void* z, uint64_t ldz, void* ws,
                                    size_t ws_bytes, void* stream) {
    if (!type_ok(type) || !dims_ok(m, n) || !dims_ok(m, k) || !act_ok(act)) return SLIMDP_ERR_INVALID_ARG;
    if (!matrix_ok(x, ldx, m, k, type) || !matrix_ok(w, ldw, n, k, type) || !matrix_ok(y, ldy, m, n, type) ||
        !matrix_or_null(residual, ldr, m, n, type) || !matrix_or_null(z, ldz, m, n, type) || !vector_or_null(bias))
        return SLIMDP_ERR_INVALID_ARG;
    const slimdp_status s = workspace_ok(ws, ws_bytes, linear_ws_bytes(m, n, k, type), 256);
    if (s != SLIMDP_OK) return s;
    return launch_linear_forward(x, ldx, w, ldw, bias, residual, ldr, m, n, k, type, act, y, ldy, z, ldz, ws,
                                 (cudaStream_t)stream);
}

slimdp_status slimdp_linear_backward_input(const void* dy, uint64_t lddy, const void* w, uint64_t ldw, const void* z,
                                           uint64_t ldz, const void* add, uint64_t ldadd, uint64_t m, uint64_t n,
                                           uint64_t k, int32_t type, int32_t act, void* dx, uint64_t lddx, void* ws,
                                           size_t ws_bytes, void* stream) {
    if (!type_ok(type) || !dims_ok(m, n) || !dims_ok(m, k) || !act_ok(act)) return SLIMDP_ERR_INVALID_ARG;
    if (act != SLIMDP_ACT_NONE && !matrix_ok(z, ldz, m, k, type)) return SLIMDP_ERR_INVALID_ARG;
    if (!matrix_ok(dy, lddy, m, n, type) || !matrix_ok(w, ldw, n, k, type) || !matrix_ok(dx, lddx, m, k, type) ||
        !matrix_or_null(add, ldadd, m, k, type))
        return SLIMDP_ERR_INVALID_ARG;
    const slimdp_status s = workspace_ok(ws, ws_bytes, linear_ws_bytes(m, n, k, type), 256);
    if (s != SLIMDP_OK) return s;
    return launch_linear_backward_input(dy, lddy, w, ldw, z, ldz, add, ldadd, m, n, k, type, act, dx, lddx, ws,
                                        (cudaStream_t)stream);
}

slimdp_status slimdp_linear_backward_weight(const void* dy, uint64_t lddy, const void* x, uint64_t ldx, uint64_t m,
                                            uint64_t n, uint64_t k, int32_t type, float* dw, uint64_t lddw, float* db,
                                            int32_t accumulate, void* ws, size_t ws_bytes, void* stream) {
    if (!type_ok(type) || !dims_ok(m, n) || !dims_ok(m, k)) return SLIMDP_ERR_INVALID_ARG;
    if (!matrix_ok(dy, lddy, m, n, type) || !matrix_ok(x, ldx, m, k, type) ||
        !matrix_ok(dw, lddw, n, k, SLIMDP_F32) || !vector_or_null(db))
        return SLIMDP_ERR_INVALID_ARG;
    const slimdp_status s = workspace_ok(ws, ws_bytes, linear_ws_bytes(m, n, k, type), 256);
    if (s != SLIMDP_OK) return s;
    return launch_linear_backward_weight(dy, lddy, x, ldx, m, n, k, type, dw, lddw, db, accumulate != 0, ws,
                                         (cudaStream_t)stream);
}

slimdp_status slimdp_activation_backward(const void* dy, uint64_t lddy, const void* z, uint64_t ldz, uint64_t m,
                                         uint64_t n, int32_t type, int32_t act, void* dz, uint64_t lddz,
                                         void* stream) {
    if (!type_ok(type) || !dims_ok(m, n) || !act_ok(act)) return SLIMDP_ERR_INVALID_ARG;
    if (act != SLIMDP_ACT_NONE && !matrix_ok(z, ldz, m, n, type)) return SLIMDP_ERR_INVALID_ARG;
    if (!matrix_ok(dy, lddy, m, n, type) || !matrix_ok(dz, lddz, m, n, type)) return SLIMDP_ERR_INVALID_ARG;
    return launch_activation_backward(dy, lddy, z, ldz, m, n, type, act, dz, lddz, (cudaStream_t)stream);
}

slimdp_status slimdp_train_read_status(void* stream) {
    if (cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess) return SLIMDP_ERR_CUDA;
    slimdp_status s = read_product_status();
    if (s == SLIMDP_OK) s = read_distill_status();
    return s == SLIMDP_OK ? read_layernorm_status() : s;
}

slimdp_status slimdp_distill(const void* logits, uint64_t ldl, uint64_t rows, uint64_t vocab, int32_t type,
                             const int32_t* teacher_idx, const void* teacher_logit, int32_t teacher_type, uint32_t top,
                             const int32_t* label, const float* row_weight, float temperature, float kd_weight,
                             float ce_weight, float* loss, void* dlogits, uint64_t ldd, void* stream) {
    if (!type_ok(type) || !type_ok(teacher_type) || !dims_ok(rows, vocab) || top > SLIMDP_MAX_TOP)
        return SLIMDP_ERR_INVALID_ARG;
    if (!isfinite(temperature) || temperature <= 0.0f || !isfinite(kd_weight) || !isfinite(ce_weight))
        return SLIMDP_ERR_INVALID_ARG;
    if (!matrix_ok(logits, ldl, rows, vocab, type) || !matrix_or_null(dlogits, ldd, rows, vocab, type) ||
        (dlogits == logits && dlogits && ldd != ldl))
        return SLIMDP_ERR_INVALID_ARG;
    if (rows > 0 && top > 0 && (!teacher_idx || !teacher_logit)) return SLIMDP_ERR_INVALID_ARG;
    if ((rows > 0 && !loss) || !vector_or_null(teacher_idx) || !vector_or_null(label) || !vector_or_null(row_weight) ||
        !vector_or_null(loss) || (teacher_logit && !aligned_to(teacher_logit, type_bytes(teacher_type))))
        return SLIMDP_ERR_INVALID_ARG;
    return launch_distill(logits, ldl, (uint32_t)rows, (uint32_t)vocab, type, teacher_idx, teacher_logit, teacher_type,
                          top, label, row_weight, temperature, kd_weight, ce_weight, loss, dlogits, ldd,
                          (cudaStream_t)stream);
}

}  // extern "C"
