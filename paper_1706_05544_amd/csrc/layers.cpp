// C entry points of the feature-map operators: argument checks, status codes
// and dispatch.  Every check comes before any device call; the arithmetic is
// in linear.hip, norm.hip, hinge.hip and adamw.hip.
#include <cmath>
#include <cstdint>
#include <string>

#include "checks.hpp"

using namespace msvm;

namespace {

svm_status check_linear_inputs(const svm_array* X, const svm_array* W)
{
    CHECK(check_first(X, "X"));
    CHECK(check_first(W, "W"));
    if (W->rows < 1 || W->rows > msvm::kMaxWidth)
        return fail(SVM_E_INVALID, "W: rows must be in [1, 2^21]");
    return check_array(W, "W", W->rows, X->cols, X->dtype);
}

svm_status check_linear_grad(const svm_array* dY, const svm_array* X,
                             const svm_array* W, int32_t act,
                             const svm_array* dX, const svm_array* dW,
                             const svm_array* dbias)
{
    CHECK(check_act(act));
    CHECK(check_first(dY, "dY"));
    const int64_t m = dY->rows, n = dY->cols;
    const int32_t t = dY->dtype;
    int64_t k = 0;
    if (X) {
        CHECK(check_first(X, "X"));
        k = X->cols;
        CHECK(check_array(X, "X", m, k, t));
    } else if (dW) {
        return fail(SVM_E_INVALID, "X is NULL");
    }
    if (W) {
        CHECK(check_first(W, "W"));
        if (!X) k = W->cols;
        CHECK(check_array(W, "W", n, k, t));
    } else if (dX) {
        return fail(SVM_E_INVALID, "W is NULL");
    }
    if (dX) CHECK(check_array(dX, "dX", m, k, t));
    if (dW) CHECK(check_array(dW, "dW", n, k, t));
    if (dbias) CHECK(check_array(dbias, "dbias", 1, n, t));
    return SVM_OK;
}

}  // namespace

extern "C" {

svm_status svm_linear_workspace(const svm_array* X, const svm_array* W,
                                int64_t* bytes)
{
    ENTRY_BEGIN
    if (!bytes) return fail(SVM_E_INVALID, "bytes is NULL");
    *bytes = 0;
    CHECK(check_linear_inputs(X, W));
    msvm::LinearArgs a{*X, *W, kNone, kNone, kNone, kNone, SVM_ACT_NONE};
    msvm::Pieces count;
    msvm::linear_forward(a, count, nullptr);
    *bytes = count.used;
    return SVM_OK;
    GUARD_END
}

svm_status svm_linear(const svm_array* X, const svm_array* W,
                      const svm_array* bias, const svm_array* residual,
                      int32_t act, const svm_array* Y, const svm_array* Z,
                      void* work, int64_t work_bytes, int32_t device,
                      void* stream)
{
    ENTRY_BEGIN
    CHECK(check_act(act));
    CHECK(check_linear_inputs(X, W));
    const int64_t m = X->rows, n = W->rows;
    const int32_t t = X->dtype;
    if (bias) CHECK(check_array(bias, "bias", 1, n, t));
    if (residual) CHECK(check_array(residual, "residual", m, n, t));
    CHECK(check_array(Y, "Y", m, n, t));
    CHECK(check_apart(Y, "Y", {X, W, bias, Z}));
    if (!same(Y, residual)) CHECK(check_apart(Y, "Y", {residual}));
    if (Z) {
        CHECK(check_array(Z, "Z", m, n, t));
        CHECK(check_apart(Z, "Z", {X, W, bias, residual}));
    }
    msvm::LinearArgs a{*X,           *W, *Y, or_none(Z), or_none(bias),
                       or_none(residual), act};
    msvm::Pieces count;
    msvm::linear_forward(a, count, nullptr);
    CHECK(check_work(work, work_bytes, count.used));
    CHECK(check_ordinal(device));
    if (m == 0) return SVM_OK;
    msvm::OnDevice on(device);
    msvm::Pieces ws{static_cast<unsigned char*>(work), true};
    msvm::linear_forward(a, ws, (hipStream_t)stream);
    HIP_TRY(hipPeekAtLastError());
    return SVM_OK;
    GUARD_END
}

svm_status svm_linear_backward_workspace(const svm_array* dY,
                                         const svm_array* X,
                                         const svm_array* W, int32_t act,
                                         const svm_array* dX,
                                         const svm_array* dW,
                                         const svm_array* dbias,
                                         int64_t* bytes)
{
    ENTRY_BEGIN
    if (!bytes) return fail(SVM_E_INVALID, "bytes is NULL");
    *bytes = 0;
    CHECK(check_linear_grad(dY, X, W, act, dX, dW, dbias));
    msvm::LinearGradArgs a{*dY,         or_none(X),  or_none(W),
                           kNone,       or_none(dX), or_none(dW),
                           or_none(dbias), act};
    msvm::Pieces count;
    msvm::linear_backward(a, count, nullptr);
    *bytes = count.used;
    return SVM_OK;
    GUARD_END
}

svm_status svm_linear_backward(const svm_array* dY, const svm_array* X,
                               const svm_array* W, const svm_array* Z,
                               int32_t act, const svm_array* dX,
                               const svm_array* dW, const svm_array* dbias,
                               void* work, int64_t work_bytes, int32_t device,
                               void* stream)
{
    ENTRY_BEGIN
    CHECK(check_linear_grad(dY, X, W, act, dX, dW, dbias));
    const int64_t m = dY->rows, n = dY->cols;
    if (Z)
        CHECK(check_array(Z, "Z", m, n, dY->dtype));
    else if (act != SVM_ACT_NONE)
        return fail(SVM_E_INVALID, "Z is NULL");
    if (dX) CHECK(check_apart(dX, "dX", {dY, X, W, Z, dW, dbias}));
    if (dW) CHECK(check_apart(dW, "dW", {dY, X, W, Z, dbias}));
    if (dbias) CHECK(check_apart(dbias, "dbias", {dY, X, W, Z}));
    msvm::LinearGradArgs a{*dY,         or_none(X),  or_none(W),
                           or_none(Z),  or_none(dX), or_none(dW),
                           or_none(dbias), act};
    msvm::Pieces count;
    msvm::linear_backward(a, count, nullptr);
    CHECK(check_work(work, work_bytes, count.used));
    CHECK(check_ordinal(device));
    if (!dX && !dW && !dbias) return SVM_OK;
    msvm::OnDevice on(device);
    msvm::Pieces ws{static_cast<unsigned char*>(work), true};
    msvm::linear_backward(a, ws, (hipStream_t)stream);
    HIP_TRY(hipPeekAtLastError());
    return SVM_OK;
    GUARD_END
}

svm_status svm_layer_norm(const svm_array* X, const svm_array* weight,
                          const svm_array* bias, double eps,
                          const svm_array* Y, float* mean, float* rstd,
                          int32_t device, void* stream)
{
    ENTRY_BEGIN
    CHECK(check_first(X, "X"));
    const int64_t m = X->rows, n = X->cols;
    if (weight) CHECK(check_array(weight, "weight", 1, n, X->dtype));
    if (bias) CHECK(check_array(bias, "bias", 1, n, X->dtype));
    if (!std::isfinite(eps) || eps < 0)
        return fail(SVM_E_INVALID, "eps must be finite and >= 0");
    CHECK(check_array(Y, "Y", m, n, X->dtype));
    CHECK(check_apart(Y, "Y", {weight, bias}));
    if (!same(Y, X)) CHECK(check_apart(Y, "Y", {X}));
    CHECK(check_ordinal(device));
    if (m == 0) return SVM_OK;
    msvm::OnDevice on(device);
    msvm::NormArgs a{*X, or_none(weight), or_none(bias), *Y, (float)eps, mean,
                     rstd};
    msvm::norm_forward(a, (hipStream_t)stream);
    HIP_TRY(hipPeekAtLastError());
    return SVM_OK;
    GUARD_END
}

svm_status svm_layer_norm_backward_workspace(int64_t rows, int64_t cols,
                                             int64_t* bytes)
{
    ENTRY_BEGIN
    if (!bytes) return fail(SVM_E_INVALID, "bytes is NULL");
    *bytes = 0;
    if (rows < 0 || rows > ((int64_t)1 << 31) - 1)
        return fail(SVM_E_INVALID, "rows must be in [0, 2^31)");
    if (cols < 1 || cols > msvm::kMaxWidth)
        return fail(SVM_E_INVALID, "cols must be in [1, 2^21]");
    *bytes = msvm::norm_backward_bytes(rows, cols);
    return SVM_OK;
    GUARD_END
}

svm_status svm_layer_norm_backward(const svm_array* dY, const svm_array* X,
                                   const float* mean, const float* rstd,
                                   const svm_array* weight,
                                   const svm_array* residual,
                                   const svm_array* dX,
                                   const svm_array* dweight,
                                   const svm_array* dbias, void* work,
                                   int64_t work_bytes, int32_t device,
                                   void* stream)
{
    ENTRY_BEGIN
    CHECK(check_first(dY, "dY"));
    const int64_t m = dY->rows, n = dY->cols;
    const int32_t t = dY->dtype;
    CHECK(check_array(X, "X", m, n, t));
    if (m > 0 && (!mean || !rstd))
        return fail(SVM_E_INVALID, "mean or rstd is NULL");
    if (weight) CHECK(check_array(weight, "weight", 1, n, t));
    if (residual) CHECK(check_array(residual, "residual", m, n, t));
    if (dX) {
        CHECK(check_array(dX, "dX", m, n, t));
        CHECK(check_apart(dX, "dX", {X, weight, dweight, dbias}));
        if (!same(dX, dY)) CHECK(check_apart(dX, "dX", {dY}));
        if (!same(dX, residual)) CHECK(check_apart(dX, "dX", {residual}));
    }
    if (dweight) {
        CHECK(check_array(dweight, "dweight", 1, n, t));
        CHECK(check_apart(dweight, "dweight",
                          {dY, X, weight, residual, dbias}));
    }
    if (dbias) {
        CHECK(check_array(dbias, "dbias", 1, n, t));
        CHECK(check_apart(dbias, "dbias", {dY, X, weight, residual}));
    }
    if (dweight || dbias)
        CHECK(check_work(work, work_bytes, msvm::norm_backward_bytes(m, n)));
    CHECK(check_ordinal(device));
    msvm::OnDevice on(device);
    msvm::NormGradArgs a{*dY,         *X,
                         or_none(weight),  or_none(residual),
                         or_none(dX),      or_none(dweight),
                         or_none(dbias),   mean,
                         rstd};
    msvm::Pieces ws{static_cast<unsigned char*>(work), true};
    msvm::norm_backward(a, ws, (hipStream_t)stream);
    HIP_TRY(hipPeekAtLastError());
    return SVM_OK;
    GUARD_END
}

svm_status svm_hinge_loss_workspace(int64_t rows, int64_t cols,
                                    int64_t* bytes)
{
    ENTRY_BEGIN
    if (!bytes) return fail(SVM_E_INVALID, "bytes is NULL");
    *bytes = 0;
    if (rows < 0 || rows > ((int64_t)1 << 31) - 1)
        return fail(SVM_E_INVALID, "rows must be in [0, 2^31)");
    if (cols < 1 || cols > msvm::kMaxWidth)
        return fail(SVM_E_INVALID, "cols must be in [1, 2^21]");
    *bytes = msvm::hinge_bytes(rows, cols);
    return SVM_OK;
    GUARD_END
}

svm_status svm_hinge_loss(const svm_array* S, const int32_t* labels,
                          double scale, const svm_array* dS, float* loss,
                          void* work, int64_t work_bytes, int32_t device,
                          void* stream)
{
    ENTRY_BEGIN
    CHECK(check_first(S, "S"));
    if (S->rows > 0 && !labels) return fail(SVM_E_INVALID, "labels is NULL");
    if (!loss) return fail(SVM_E_INVALID, "loss is NULL");
    if (!std::isfinite(2.0f * (float)scale))
        return fail(SVM_E_INVALID, "2 scale must be finite in 32 bits");
    if (dS) {
        CHECK(check_array(dS, "dS", S->rows, S->cols, S->dtype));
        if (!same(dS, S)) CHECK(check_apart(dS, "dS", {S}));
    }
    CHECK(check_work(work, work_bytes,
                     msvm::hinge_bytes(S->rows, S->cols)));
    CHECK(check_ordinal(device));
    msvm::OnDevice on(device);
    msvm::Pieces ws{static_cast<unsigned char*>(work), true};
    msvm::hinge_loss(*S, labels, (float)scale, or_none(dS), loss, ws,
                     (hipStream_t)stream);
    HIP_TRY(hipPeekAtLastError());
    return SVM_OK;
    GUARD_END
}

svm_status svm_adamw_step(const svm_adamw_tensor* tensors, int32_t n_tensors,
                          const svm_adamw_params* p, int32_t device,
                          void* stream)
{
    ENTRY_BEGIN
    CHECK(check_adamw(tensors, n_tensors, p));
    CHECK(check_ordinal(device));
    msvm::OnDevice on(device);
    msvm::adamw_step(tensors, n_tensors, *p, (hipStream_t)stream);
    HIP_TRY(hipPeekAtLastError());
    return SVM_OK;
    GUARD_END
}

svm_status svm_adamw_state(const int8_t* m, const uint8_t* v,
                           const float* m_scale, const float* v_scale,
                           int64_t n, float* m_out, float* v_out,
                           int32_t device, void* stream)
{
    ENTRY_BEGIN
    if (n < 0 || n > (int64_t)1 << 40)
        return fail(SVM_E_INVALID, "n must be in [0, 2^40]");
    if (n > 0 && ((m_out && (!m || !m_scale)) || (v_out && (!v || !v_scale))))
        return fail(SVM_E_INVALID, "codes or scales are NULL");
    CHECK(check_ordinal(device));
    if (n == 0 || (!m_out && !v_out)) return SVM_OK;
    msvm::OnDevice on(device);
    msvm::adamw_state(m, v, m_scale, v_scale, n, m_out, v_out,
                      (hipStream_t)stream);
    HIP_TRY(hipPeekAtLastError());
    return SVM_OK;
    GUARD_END
}

}  // extern "C"
