// Internal declarations of the feature-map operators: the fused linear layer,
// layer norm, the squared hinge loss and the AdamW step.
#pragma once

#include "common.hpp"

namespace msvm {

constexpr int64_t kMaxWidth = (int64_t)1 << 21;  // columns of an array
constexpr int kAdamBlock = 256;  // values that share a scale (8-bit states)

inline size_t dtype_bytes(int32_t t) { return t == SVM_F32 ? 4 : 2; }

// Pieces of a caller's workspace, each at a multiple of 256 bytes from its
// start.  With run false they are only counted, so that one function lays
// the workspace out for the size query and for the call.
struct Pieces {
    unsigned char* base = nullptr;
    bool run = false;
    int64_t used = 0;
    template <class T>
    T* take(int64_t count)
    {
        T* p = base ? reinterpret_cast<T*>(base + used) : nullptr;
        used += (count * (int64_t)sizeof(T) + 255) / 256 * 256;
        return p;
    }
};

struct LinearArgs {
    svm_array X, W, Y, Z, bias, residual;  // data NULL: not there
    int32_t act = SVM_ACT_NONE;
};
// Lays out the workspace in `ws`; with ws.run set it queues the work too.
void linear_forward(const LinearArgs& a, Pieces& ws, hipStream_t s);

struct LinearGradArgs {
    svm_array dY, X, W, Z, dX, dW, dbias;
    int32_t act = SVM_ACT_NONE;
};
void linear_backward(const LinearGradArgs& a, Pieces& ws, hipStream_t s);

struct NormArgs {
    svm_array X, weight, bias, Y;
    float eps = 0.0f;
    float *mean = nullptr, *rstd = nullptr;
};
void norm_forward(const NormArgs& a, hipStream_t s);

struct NormGradArgs {
    svm_array dY, X, weight, residual, dX, dweight, dbias;
    const float *mean = nullptr, *rstd = nullptr;
};
int64_t norm_backward_bytes(int64_t rows, int64_t cols);
void norm_backward(const NormGradArgs& a, Pieces& ws, hipStream_t s);

// out[c] = sum over the np rows of part (np x cols, fp32), rounded to the
// type; the two sums of a gradient in one launch (either out may be NULL).
void launch_column_sums(const float* part0, const float* part1, int64_t np,
                        int64_t cols, int32_t dtype, void* out0, void* out1,
                        hipStream_t s);

int64_t hinge_bytes(int64_t rows, int64_t cols);
void hinge_loss(const svm_array& S, const int32_t* labels, float scale,
                const svm_array& dS, float* loss, Pieces& ws, hipStream_t s);

void adamw_step(const svm_adamw_tensor* t, int32_t n,
                const svm_adamw_params& p, hipStream_t s);
void adamw_state(const int8_t* m, const uint8_t* v, const float* ms,
                 const float* vs, int64_t n, float* mo, float* vo,
                 hipStream_t s);

}  // namespace msvm
