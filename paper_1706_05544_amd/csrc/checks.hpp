// Argument checks that the entries of the feature-map calls share: every one
// comes before any device call.
#pragma once

#include <cmath>
#include <cstdint>
#include <string>

#include "entry.hpp"
#include "layers.hpp"

namespace msvm {

inline const svm_array kNone = {nullptr, 0, 0, 0, 0, 0};

// One array of a call: there, in device memory, of the given shape and type.
inline svm_status check_array(const svm_array* a, const char* name,
                              int64_t rows, int64_t cols, int32_t dtype)
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
    if ((uintptr_t)a->data % dtype_bytes(a->dtype))
        return fail(SVM_E_INVALID, n + " is not aligned to its type");
    return SVM_OK;
}

// The first array of a call, which gives the others their sizes and type.
inline svm_status check_first(const svm_array* a, const char* name)
{
    const std::string n(name);
    if (!a) return fail(SVM_E_INVALID, n + " is NULL");
    if (a->rows < 0 || a->rows > ((int64_t)1 << 31) - 1)
        return fail(SVM_E_INVALID, n + ": rows must be in [0, 2^31)");
    if (a->cols < 1 || a->cols > kMaxWidth)
        return fail(SVM_E_INVALID, n + ": cols must be in [1, 2^21]");
    return check_array(a, name, a->rows, a->cols, a->dtype);
}

// Whether the two arrays have elements in common (as far as their ranges of
// bytes say; columns side by side in the rows of one buffer have none).
inline bool overlap(const svm_array* a, const svm_array* b)
{
    if (!a || !b || !a->data || !b->data || !a->rows || !b->rows) return false;
    const uintptr_t ea = dtype_bytes(a->dtype);
    const uintptr_t eb = dtype_bytes(b->dtype);
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

inline bool same(const svm_array* a, const svm_array* b)
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

inline svm_status check_act(int32_t act)
{
    if (act < SVM_ACT_NONE || act > SVM_ACT_COS)
        return fail(SVM_E_INVALID, "unknown activation");
    return SVM_OK;
}

inline svm_status check_work(const void* work, int64_t work_bytes, int64_t need)
{
    if (need > 0 && (!work || work_bytes < need))
        return fail(SVM_E_INVALID, "work must have " + std::to_string(need) +
                                       " bytes, has " +
                                       std::to_string(work ? work_bytes : 0));
    if ((uintptr_t)work & 15)
        return fail(SVM_E_INVALID, "work must be aligned to 16 bytes");
    return SVM_OK;
}

inline svm_status check_ordinal(int32_t device)
{
    if (device < 0) return fail(SVM_E_INVALID, "device must be >= 0");
    ClearHipError clear;
    return check_device(device);
}

inline svm_status check_adamw(const svm_adamw_tensor* tensors,
                              int32_t n_tensors, const svm_adamw_params* p)
{
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
        if ((uintptr_t)t.param % dtype_bytes(t.dtype) ||
            (uintptr_t)t.grad % dtype_bytes(t.grad_dtype) ||
            (uintptr_t)t.m_scale % 4 || (uintptr_t)t.v_scale % 4)
            return fail(SVM_E_INVALID, at + "not aligned to its type");
        if ((uintptr_t)t.master % 16 || (uintptr_t)t.m % 16 ||
            (uintptr_t)t.v % 16)
            return fail(SVM_E_INVALID,
                        at + "m, v and master must be aligned to 16 bytes");
    }
    return SVM_OK;
}

inline const svm_array& or_none(const svm_array* a) { return a ? *a : kNone; }

}  // namespace msvm

#define CHECK(expr)                            \
    do {                                       \
        const svm_status st_ = (expr);         \
        if (st_ != SVM_OK) return st_;         \
    } while (0)
