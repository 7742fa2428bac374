// C entry points around a feature network's training step and its serving:
// argument checks, status codes and dispatch.  Every check comes before any
// device call; the arithmetic is in gradnorm.hip and adamw.hip.
#include <cmath>
#include <cstdint>
#include <string>

#include "checks.hpp"

using namespace msvm;

namespace {

svm_status check_grads(const svm_grad* grads, int32_t n)
{
    if (n < 0) return fail(SVM_E_INVALID, "n_grads must be >= 0");
    if (n > 0 && !grads) return fail(SVM_E_INVALID, "grads is NULL");
    for (int32_t i = 0; i < n; ++i) {
        const svm_grad& g = grads[i];
        const std::string at = "gradient " + std::to_string(i) + ": ";
        if (g.n < 0 || g.n > (int64_t)1 << 40)
            return fail(SVM_E_INVALID, at + "n must be in [0, 2^40]");
        if (g.dtype < SVM_F32 || g.dtype > SVM_F16)
            return fail(SVM_E_INVALID, at + "unknown type");
        if (g.n == 0) continue;
        if (!g.data) return fail(SVM_E_INVALID, at + "no data");
        if ((uintptr_t)g.data % dtype_bytes(g.dtype))
            return fail(SVM_E_INVALID, at + "not aligned to its type");
    }
    return SVM_OK;
}

// One float on the device.
svm_status check_float(const void* p, const char* name)
{
    if ((uintptr_t)p % 4)
        return fail(SVM_E_INVALID, std::string(name) + " is not aligned");
    return SVM_OK;
}

}  // namespace

extern "C" {

svm_status svm_grad_norm_workspace(const svm_grad* grads, int32_t n_grads,
                                   int64_t* bytes)
{
    ENTRY_BEGIN
    if (!bytes) return fail(SVM_E_INVALID, "bytes is NULL");
    *bytes = 0;
    CHECK(check_grads(grads, n_grads));
    Pieces count;
    grad_norm(grads, n_grads, 1.0, 1.0, nullptr, nullptr, count, nullptr);
    *bytes = count.used;
    return SVM_OK;
    GUARD_END
}

svm_status svm_grad_norm(const svm_grad* grads, int32_t n_grads,
                         double grad_scale, double max_norm, float* norm,
                         float* factor, void* work, int64_t work_bytes,
                         int32_t device, void* stream)
{
    ENTRY_BEGIN
    CHECK(check_grads(grads, n_grads));
    if (!std::isfinite(grad_scale))
        return fail(SVM_E_INVALID, "grad_scale must be finite");
    if (!(max_norm >= 0)) return fail(SVM_E_INVALID, "max_norm must be >= 0");
    if (!norm) return fail(SVM_E_INVALID, "norm is NULL");
    CHECK(check_float(norm, "norm"));
    CHECK(check_float(factor, "factor"));
    if (norm == factor)
        return fail(SVM_E_INVALID, "norm and factor are the same");
    Pieces count;
    grad_norm(grads, n_grads, grad_scale, max_norm, norm, factor, count,
              nullptr);
    CHECK(check_work(work, work_bytes, count.used));
    CHECK(check_ordinal(device));
    OnDevice on(device);
    Pieces ws{static_cast<unsigned char*>(work), true};
    grad_norm(grads, n_grads, grad_scale, max_norm, norm, factor, ws,
              (hipStream_t)stream);
    HIP_TRY(hipPeekAtLastError());
    return SVM_OK;
    GUARD_END
}

svm_status svm_adamw_step_clipped(const svm_adamw_tensor* tensors,
                                  int32_t n_tensors,
                                  const svm_adamw_params* p,
                                  const float* factor, int32_t device,
                                  void* stream)
{
    ENTRY_BEGIN
    CHECK(check_adamw(tensors, n_tensors, p));
    CHECK(check_float(factor, "factor"));
    CHECK(check_ordinal(device));
    OnDevice on(device);
    adamw_step_clipped(tensors, n_tensors, *p, factor, (hipStream_t)stream);
    HIP_TRY(hipPeekAtLastError());
    return SVM_OK;
    GUARD_END
}

}  // extern "C"
