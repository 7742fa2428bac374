// C entry points of the feature-map operators: argument checks, status codes
// and dispatch.  Every check comes before any device call; the arithmetic is
// in linear.hip, norm.hip, hinge.hip and adamw.hip.
#include <cmath>
#include <cstdint>
#include <string>

#include "entry.hpp"
#include "layers.hpp"

using msvm::check_device;
using msvm::fail;

namespace {

const svm_array kNone = {nullptr, 0, 0, 0, 0, 0};

// One array of a call: there, in device memory, of the given shape and type.
svm_status check_array(const svm_array* a, const char* name, int64_t rows,
                       int64_t cols, int32_t dtype)
{
    const std::string n(name);
    if (!a) return fail(SVM_E_INVALID, n + " is NULL");
    if (a->dtype < SVM_F32 || a->dtype > SVM_F16)
        return fail(SVM_E_INVALID, n + ": unknown type");
    if (a->dtype != dtype)
        return fail(SVM_E_INVALID, n + " has another type than the rest");
    if (a->rows != rows || a->cols != cols)
        return fail(SVM_E_INVALID,
                    n + " must be " + std::to_string(rows) + " x " +
                        std::to_string(cols) + ", is " +
                        std::to_string(a->rows) + " x " +
                        std::to_string(a->cols));
    if (a->ld < a->cols) return fail(SVM_E_INVALID, n + ": ld must be >= cols");
    if (a->ld > (int64_t)1 << 40)
        return fail(SVM_E_INVALID, n + ": ld must be at most 2^40");
    if (!a->on_device)
        return fail(SVM_E_UNSUPPORTED, n + " must be in device memory");
    if (a->rows > 0 && !a->data)
        return fail(SVM_E_INVALID, n + " has no data");
    if ((uintptr_t)a->data % msvm::dtype_bytes(a->dtype))
        return fail(SVM_E_INVALID, n + " is not aligned to its type");
    return SVM_OK;
}

// The first array of a call, which gives the others their sizes and type.
svm_status check_first(const svm_array* a, const char* name)
{
    const std::string n(name);
    if (!a) return fail(SVM_E_INVALID, n + " is NULL");
    if (a->rows < 0 || a->rows > ((int64_t)1 << 31) - 1)
        return fail(SVM_E_INVALID, n + ": rows must be in [0, 2^31)");
    if (a->cols < 1 || a->cols > msvm::kMaxWidth)
        return fail(SVM_E_INVALID, n + ": cols must be in [1, 2^21]");
    return check_array(a, name, a->rows, a->cols, a->dtype);
}

// Whether the two arrays have elements in common (as far as their ranges of
// bytes say; columns side by side in the rows of one buffer have none).
bool overlap(const svm_array* a, const svm_array* b)
{
    if (!a || !b || !a->data || !b->data || !a->rows || !b->rows) return false;
    const uintptr_t ea = msvm::dtype_bytes(a->dtype);
    const uintptr_t eb = msvm::dtype_bytes(b->dtype);
    const uintptr_t pa = (uintptr_t)a->data, pb = (uintptr_t)b->data;
    const uintptr_t na = ((uintptr_t)(a->rows - 1) * a->ld + a->cols) * ea;
    const uintptr_t nb = ((uintptr_t)(b->rows - 1) * b->ld + b->cols) * eb;
    if (pa >= pb + nb || pb >= pa + na) return false;
    const uintptr_t row = (uintptr_t)a->ld * ea;
    if (row != (uintptr_t)b->ld * eb) return true;
    const uintptr_t at = pb >= pa ? (pb - pa) % row
                                  : (row - (pa - pb) % row) % row;
    return at < (uintptr_t)a->cols * ea || at + (uintptr_t)b->cols * eb > row;
}

bool same(const svm_array* a, const svm_array* b)
{
    return a && b && a->data == b->data && a->ld == b->ld;
}

// Output `out` against the arrays it must not overlap.
template <size_t N>
svm_status check_apart(const svm_array* out, const char* name,
                       const svm_array* const (&others)[N])
{
    for (const svm_array* o : others)
        if (overlap(out, o))
            return fail(SVM_E_INVALID,
                        std::string(name) + " overlaps another array");
    return SVM_OK;
}

svm_status check_act(int32_t act)
{
    if (act < SVM_ACT_NONE || act > SVM_ACT_COS)
        return fail(SVM_E_INVALID, "unknown activation");
    return SVM_OK;
}

svm_status check_work(const void* work, int64_t work_bytes, int64_t need)
{
    if (need > 0 && (!work || work_bytes < need))
        return fail(SVM_E_INVALID, "work must have " + std::to_string(need) +
                                       " bytes, has " +
                                       std::to_string(work ? work_bytes : 0));
    if ((uintptr_t)work & 15)
        return fail(SVM_E_INVALID, "work must be aligned to 16 bytes");
    return SVM_OK;
}

svm_status check_ordinal(int32_t device)
{
    if (device < 0) return fail(SVM_E_INVALID, "device must be >= 0");
    msvm::ClearHipError clear;
    return check_device(device);
}

const svm_array& or_none(const svm_array* a) { return a ? *a : kNone; }

#define CHECK(expr)                            \
    do {                                       \
        const svm_status st_ = (expr);         \
        if (st_ != SVM_OK) return st_;         \
    } while (0)

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
    if (!p) return fail(SVM_E_INVALID, "params is NULL");
    if (n_tensors < 0) return fail(SVM_E_INVALID, "n_tensors must be >= 0");
    if (n_tensors > 0 && !tensors)
        return fail(SVM_E_INVALID, "tensors is NULL");
    if (!std::isfinite(p->lr) || !std::isfinite(p->weight_decay) ||
        !std::isfinite(p->grad_scale))
        return fail(SVM_E_INVALID,
                    "lr, weight_decay and grad_scale must be finite");
    if (!(p->beta1 >= 0 && p->beta1 < 1) || !(p->beta2 >= 0 && p->beta2 < 1))
        return fail(SVM_E_INVALID, "beta1 and beta2 must be in [0, 1)");
    if (!std::isfinite(p->eps) || p->eps < 0)
        return fail(SVM_E_INVALID, "eps must be finite and >= 0");
    if (p->step < 1) return fail(SVM_E_INVALID, "step must be >= 1");
    if (p->bits != 32 && p->bits != 8)
        return fail(SVM_E_INVALID, "bits must be 32 or 8");
    for (int32_t i = 0; i < n_tensors; ++i) {
        const svm_adamw_tensor& t = tensors[i];
        const std::string at = "tensor " + std::to_string(i) + ": ";
        if (t.n < 0 || t.n > (int64_t)1 << 40)
            return fail(SVM_E_INVALID, at + "n must be in [0, 2^40]");
        if (t.dtype < SVM_F32 || t.dtype > SVM_F16)
            return fail(SVM_E_INVALID, at + "unknown type");
        if (t.grad_dtype != t.dtype && t.grad_dtype != SVM_F32)
            return fail(SVM_E_INVALID,
                        at + "the gradient must have the parameter's type or "
                             "SVM_F32");
        if (t.master && t.dtype == SVM_F32)
            return fail(SVM_E_INVALID,
                        at + "master copies are for 16-bit parameters");
        if (t.n == 0) continue;
        if (!t.param || !t.grad || !t.m || !t.v)
            return fail(SVM_E_INVALID, at + "param, grad, m or v is NULL");
        if (p->bits == 8 && (!t.m_scale || !t.v_scale))
            return fail(SVM_E_INVALID, at + "m_scale or v_scale is NULL");
        if (p->bits == 32 && (t.m_scale || t.v_scale))
            return fail(SVM_E_INVALID,
                        at + "scales are for states in 8 bits");
        if ((uintptr_t)t.param % msvm::dtype_bytes(t.dtype) ||
            (uintptr_t)t.grad % msvm::dtype_bytes(t.grad_dtype) ||
            (uintptr_t)t.m_scale % 4 || (uintptr_t)t.v_scale % 4)
            return fail(SVM_E_INVALID, at + "not aligned to its type");
        if ((uintptr_t)t.master % 16 || (uintptr_t)t.m % 16 ||
            (uintptr_t)t.v % 16)
            return fail(SVM_E_INVALID,
                        at + "m, v and master must be aligned to 16 bytes");
    }
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
