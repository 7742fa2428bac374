// C entry of the AdamW step that counts the steps left out: argument checks
// and dispatch.  Every check comes before any device call; the arithmetic is
// in adamw.hip.
#include <cstdint>
#include <string>

#include "checks.hpp"

using namespace msvm;

namespace {

bool inside(const void* p, int64_t size, const void* data, int64_t bytes)
{
    const uintptr_t a = (uintptr_t)p, d = (uintptr_t)data;
    return p && data && a < d + (uintptr_t)bytes && d < a + (uintptr_t)size;
}

// Whether `size` bytes at p lie in what a step of the tensor writes.
bool in_tensor(const void* p, int64_t size, const svm_adamw_tensor& t,
               int32_t bits)
{
    const int64_t blocks = (t.n + kAdamBlock - 1) / kAdamBlock;
    const int64_t held = blocks * kAdamBlock, each = bits == 8 ? 1 : 4;
    return inside(p, size, t.param, t.n * dtype_bytes(t.dtype)) ||
           inside(p, size, t.master, held * 4) ||
           inside(p, size, t.m, held * each) ||
           inside(p, size, t.v, held * each) ||
           inside(p, size, t.m_scale, blocks * 4) ||
           inside(p, size, t.v_scale, blocks * 4);
}

}  // namespace

extern "C" svm_status svm_adamw_step_counted(
    const svm_adamw_tensor* tensors, int32_t n_tensors,
    const svm_adamw_params* p, const float* factor, int64_t* left_out,
    int32_t device, void* stream)
{
    ENTRY_BEGIN
    CHECK(check_adamw(tensors, n_tensors, p));
    if ((uintptr_t)factor % 4)
        return fail(SVM_E_INVALID, "factor is not aligned");
    if ((uintptr_t)left_out % 8)
        return fail(SVM_E_INVALID, "left_out is not aligned");
    if (inside(factor, 4, left_out, 8))
        return fail(SVM_E_INVALID, "factor and left_out overlap");
    for (int32_t i = 0; i < n_tensors; ++i)
        if (tensors[i].n > 0 && (in_tensor(factor, 4, tensors[i], p->bits) ||
                                 in_tensor(left_out, 8, tensors[i], p->bits)))
            return fail(SVM_E_INVALID, "factor or left_out lies in tensor " +
                                           std::to_string(i));
    CHECK(check_ordinal(device));
    OnDevice on(device);
    adamw_step_counted(tensors, n_tensors, *p, factor, left_out,
                       (hipStream_t)stream);
    HIP_TRY(hipPeekAtLastError());
    return SVM_OK;
    GUARD_END
}
