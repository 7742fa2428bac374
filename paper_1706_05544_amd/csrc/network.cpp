// C entry points around a feature network's training step and its serving:
// argument checks, status codes and dispatch.  Every check comes before any
// device call; the arithmetic is in gradnorm.hip, adamw.hip,
// linear4.hip and groupnorm.hip.
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

svm_status check_shape4(int64_t rows, int64_t cols, int32_t group,
                        int32_t dtype)
{
    if (rows < 1 || rows > kMaxWidth || cols < 1 || cols > kMaxWidth)
        return fail(SVM_E_INVALID,
                    "packed weights: rows and cols must be in [1, 2^21]");
    if (group != 32 && group != 64 && group != 128)
        return fail(SVM_E_INVALID,
                    "packed weights: group must be 32, 64 or 128");
    if (dtype < SVM_F32 || dtype > SVM_F16)
        return fail(SVM_E_INVALID, "packed weights: unknown type");
    return SVM_OK;
}

svm_status check_packed4(const svm_packed* w)
{
    if (!w) return fail(SVM_E_INVALID, "packed weights are NULL");
    CHECK(check_shape4(w->rows, w->cols, w->group, w->dtype));
    if (!w->data) return fail(SVM_E_INVALID, "packed weights have no data");
    if ((uintptr_t)w->data & 15)
        return fail(SVM_E_INVALID,
                    "packed weights must be aligned to 16 bytes");
    const int64_t need = Shape4(*w).bytes;
    if (w->bytes < need)
        return fail(SVM_E_INVALID, "packed weights must have " +
                                       std::to_string(need) + " bytes, have " +
                                       std::to_string(w->bytes));
    return SVM_OK;
}

// Whether the array has bytes in common with packed weights.
bool overlap4(const svm_array* a, const svm_packed* w)
{
    if (!a || !a->data || !a->rows) return false;
    const uintptr_t pa = (uintptr_t)a->data, pw = (uintptr_t)w->data;
    const uintptr_t na = ((uintptr_t)(a->rows - 1) * a->ld + a->cols) *
                         dtype_bytes(a->dtype);
    return pa < pw + (uintptr_t)Shape4(*w).bytes && pw < pa + na;
}

svm_status check_linear4_inputs(const svm_array* X, const svm_packed* W)
{
    CHECK(check_first(X, "X"));
    CHECK(check_packed4(W));
    return check_array(X, "X", X->rows, W->cols, W->dtype);
}

// rows positions in samples of `positions`, cols channels in groups
svm_status check_groups(int64_t rows, int64_t positions, int64_t cols,
                        int64_t groups)
{
    if (rows < 0 || rows > ((int64_t)1 << 31) - 1)
        return fail(SVM_E_INVALID, "rows must be in [0, 2^31)");
    if (cols < 1 || cols > kMaxWidth)
        return fail(SVM_E_INVALID, "cols must be in [1, 2^21]");
    if (positions < 1 || rows % positions)
        return fail(SVM_E_INVALID, "rows must be whole samples of positions");
    if (groups < 1 || cols % groups)
        return fail(SVM_E_INVALID, "cols must be whole groups");
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

svm_status svm_pack_weights_bytes(int64_t rows, int64_t cols, int32_t group,
                                  int32_t dtype, int64_t* bytes)
{
    ENTRY_BEGIN
    if (!bytes) return fail(SVM_E_INVALID, "bytes is NULL");
    *bytes = 0;
    CHECK(check_shape4(rows, cols, group, dtype));
    *bytes = Shape4(rows, cols, group, dtype).bytes;
    return SVM_OK;
    GUARD_END
}

svm_status svm_pack_weights(const svm_array* W, const svm_packed* to,
                            int32_t device, void* stream)
{
    ENTRY_BEGIN
    CHECK(check_first(W, "W"));
    CHECK(check_packed4(to));
    CHECK(check_array(W, "W", to->rows, to->cols, to->dtype));
    if (overlap4(W, to))
        return fail(SVM_E_INVALID, "W overlaps the packed weights");
    CHECK(check_ordinal(device));
    OnDevice on(device);
    pack4(*W, *to, (hipStream_t)stream);
    HIP_TRY(hipPeekAtLastError());
    return SVM_OK;
    GUARD_END
}

svm_status svm_unpack_weights(const svm_packed* packed, const svm_array* W,
                              int32_t device, void* stream)
{
    ENTRY_BEGIN
    CHECK(check_packed4(packed));
    CHECK(check_array(W, "W", packed->rows, packed->cols, packed->dtype));
    if (overlap4(W, packed))
        return fail(SVM_E_INVALID, "W overlaps the packed weights");
    CHECK(check_ordinal(device));
    OnDevice on(device);
    unpack4(*packed, *W, (hipStream_t)stream);
    HIP_TRY(hipPeekAtLastError());
    return SVM_OK;
    GUARD_END
}

svm_status svm_linear_packed_workspace(const svm_array* X,
                                       const svm_packed* W, int64_t* bytes)
{
    ENTRY_BEGIN
    if (!bytes) return fail(SVM_E_INVALID, "bytes is NULL");
    *bytes = 0;
    CHECK(check_linear4_inputs(X, W));
    Linear4Call a{*X, *W, kNone, kNone, kNone, SVM_ACT_NONE};
    Pieces count;
    linear4(a, count, nullptr);
    *bytes = count.used;
    return SVM_OK;
    GUARD_END
}

svm_status svm_linear_packed(const svm_array* X, const svm_packed* W,
                             const svm_array* bias, const svm_array* residual,
                             int32_t act, const svm_array* Y, void* work,
                             int64_t work_bytes, int32_t device, void* stream)
{
    ENTRY_BEGIN
    CHECK(check_act(act));
    CHECK(check_linear4_inputs(X, W));
    const int64_t m = X->rows, n = W->rows;
    const int32_t t = X->dtype;
    if (bias) CHECK(check_array(bias, "bias", 1, n, t));
    if (residual) CHECK(check_array(residual, "residual", m, n, t));
    CHECK(check_array(Y, "Y", m, n, t));
    CHECK(check_apart(Y, "Y", {X, bias}));
    if (overlap4(Y, W))
        return fail(SVM_E_INVALID, "Y overlaps the packed weights");
    if (!same(Y, residual)) CHECK(check_apart(Y, "Y", {residual}));
    Linear4Call a{*X, *W, or_none(bias), or_none(residual), *Y, act};
    Pieces count;
    linear4(a, count, nullptr);
    CHECK(check_work(work, work_bytes, count.used));
    CHECK(check_ordinal(device));
    if (m == 0) return SVM_OK;
    OnDevice on(device);
    Pieces ws{static_cast<unsigned char*>(work), true};
    linear4(a, ws, (hipStream_t)stream);
    HIP_TRY(hipPeekAtLastError());
    return SVM_OK;
    GUARD_END
}

svm_status svm_group_norm_workspace(int64_t rows, int64_t positions,
                                    int64_t cols, int64_t groups,
                                    int32_t dtype, int64_t* bytes)
{
    ENTRY_BEGIN
    if (!bytes) return fail(SVM_E_INVALID, "bytes is NULL");
    *bytes = 0;
    CHECK(check_groups(rows, positions, cols, groups));
    if (dtype < SVM_F32 || dtype > SVM_F16)
        return fail(SVM_E_INVALID, "unknown type");
    GroupCall a;
    a.X = {nullptr, rows, cols, cols, dtype, 1};
    a.weight = a.bias = a.Y = kNone;
    a.positions = positions;
    a.groups = groups;
    Pieces count;
    group_norm(a, count, nullptr);
    *bytes = count.used;
    return SVM_OK;
    GUARD_END
}

svm_status svm_group_norm(const svm_array* X, int64_t positions,
                          int64_t groups, const svm_array* weight,
                          const svm_array* bias, double eps, int32_t act,
                          const svm_array* Y, float* mean, float* rstd,
                          void* work, int64_t work_bytes, int32_t device,
                          void* stream)
{
    ENTRY_BEGIN
    CHECK(check_act(act));
    CHECK(check_first(X, "X"));
    const int64_t m = X->rows, n = X->cols;
    CHECK(check_groups(m, positions, n, groups));
    if (weight) CHECK(check_array(weight, "weight", 1, n, X->dtype));
    if (bias) CHECK(check_array(bias, "bias", 1, n, X->dtype));
    if (!std::isfinite(eps) || eps < 0)
        return fail(SVM_E_INVALID, "eps must be finite and >= 0");
    CHECK(check_array(Y, "Y", m, n, X->dtype));
    CHECK(check_apart(Y, "Y", {weight, bias}));
    if (!same(Y, X)) CHECK(check_apart(Y, "Y", {X}));
    CHECK(check_float(mean, "mean"));
    CHECK(check_float(rstd, "rstd"));
    const int64_t stats = m / positions * groups;
    const svm_array M{mean, 1, stats, stats, SVM_F32, 1};
    const svm_array R{rstd, 1, stats, stats, SVM_F32, 1};
    if (stats) {
        CHECK(check_apart(&M, "mean", {&R, X, Y, weight, bias}));
        CHECK(check_apart(&R, "rstd", {X, Y, weight, bias}));
    }
    GroupCall a{*X,  or_none(weight), or_none(bias), *Y,
                positions, groups, (float)eps, act, mean, rstd};
    Pieces count;
    group_norm(a, count, nullptr);
    CHECK(check_work(work, work_bytes, count.used));
    CHECK(check_ordinal(device));
    if (m == 0) return SVM_OK;
    OnDevice on(device);
    Pieces ws{static_cast<unsigned char*>(work), true};
    group_norm(a, ws, (hipStream_t)stream);
    HIP_TRY(hipPeekAtLastError());
    return SVM_OK;
    GUARD_END
}

svm_status svm_group_norm_backward_workspace(int64_t rows, int64_t positions,
                                             int64_t cols, int64_t groups,
                                             int32_t dtype, int64_t* bytes)
{
    ENTRY_BEGIN
    if (!bytes) return fail(SVM_E_INVALID, "bytes is NULL");
    *bytes = 0;
    CHECK(check_groups(rows, positions, cols, groups));
    if (dtype < SVM_F32 || dtype > SVM_F16)
        return fail(SVM_E_INVALID, "unknown type");
    GroupGradCall a;
    a.X = {nullptr, rows, cols, cols, dtype, 1};
    a.dY = a.X;
    a.weight = a.bias = a.residual = a.dX = a.dweight = a.dbias = kNone;
    a.positions = positions;
    a.groups = groups;
    a.sums = true;
    Pieces count;
    group_norm_backward(a, count, nullptr);
    *bytes = count.used;
    return SVM_OK;
    GUARD_END
}

svm_status svm_group_norm_backward(
    const svm_array* dY, const svm_array* X, int64_t positions,
    int64_t groups, const float* mean, const float* rstd,
    const svm_array* weight, const svm_array* bias, int32_t act,
    const svm_array* residual, const svm_array* dX, const svm_array* dweight,
    const svm_array* dbias, void* work, int64_t work_bytes, int32_t device,
    void* stream)
{
    ENTRY_BEGIN
    CHECK(check_act(act));
    CHECK(check_first(dY, "dY"));
    const int64_t m = dY->rows, n = dY->cols;
    const int32_t t = dY->dtype;
    CHECK(check_groups(m, positions, n, groups));
    CHECK(check_array(X, "X", m, n, t));
    if (m > 0 && (!mean || !rstd))
        return fail(SVM_E_INVALID, "mean or rstd is NULL");
    CHECK(check_float(mean, "mean"));
    CHECK(check_float(rstd, "rstd"));
    if (weight) CHECK(check_array(weight, "weight", 1, n, t));
    if (bias) CHECK(check_array(bias, "bias", 1, n, t));
    if (residual) CHECK(check_array(residual, "residual", m, n, t));
    if (dX) {
        CHECK(check_array(dX, "dX", m, n, t));
        CHECK(check_apart(dX, "dX", {X, weight, bias, dweight, dbias}));
        if (!same(dX, dY)) CHECK(check_apart(dX, "dX", {dY}));
        if (!same(dX, residual)) CHECK(check_apart(dX, "dX", {residual}));
    }
    if (dweight) {
        CHECK(check_array(dweight, "dweight", 1, n, t));
        CHECK(check_apart(dweight, "dweight",
                          {dY, X, weight, bias, residual, dbias}));
    }
    if (dbias) {
        CHECK(check_array(dbias, "dbias", 1, n, t));
        CHECK(check_apart(dbias, "dbias", {dY, X, weight, bias, residual}));
    }
    const int64_t stats = m / positions * groups;
    if (stats) {  // other blocks read them while the outputs are written
        const svm_array M{const_cast<float*>(mean), 1, stats, stats, SVM_F32,
                          1};
        const svm_array R{const_cast<float*>(rstd), 1, stats, stats, SVM_F32,
                          1};
        CHECK(check_apart(dX, "dX", {&M, &R}));
        CHECK(check_apart(dweight, "dweight", {&M, &R}));
        CHECK(check_apart(dbias, "dbias", {&M, &R}));
    }
    GroupGradCall a{*dY,          *X,
                    or_none(weight),   or_none(bias),
                    or_none(residual), or_none(dX),
                    or_none(dweight),  or_none(dbias),
                    positions,    groups,
                    act,          mean,
                    rstd,         dweight || dbias};
    Pieces count;
    group_norm_backward(a, count, nullptr);
    CHECK(check_work(work, work_bytes, count.used));
    CHECK(check_ordinal(device));
    OnDevice on(device);
    Pieces ws{static_cast<unsigned char*>(work), true};
    group_norm_backward(a, ws, (hipStream_t)stream);
    HIP_TRY(hipPeekAtLastError());
    return SVM_OK;
    GUARD_END
}

}  // extern "C"
