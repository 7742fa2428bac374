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
// ... with the gradients' factor on the device (nullable): where it is not
// finite the step is left out.
void adamw_step_clipped(const svm_adamw_tensor* t, int32_t n,
                        const svm_adamw_params& p, const float* factor,
                        hipStream_t s);
// ... and that counts the steps left out, on the device (nullable): the
// corrections are those of the steps that were not.
void adamw_step_counted(const svm_adamw_tensor* t, int32_t n,
                        const svm_adamw_params& p, const float* factor,
                        int64_t* left_out, hipStream_t s);
void adamw_state(const int8_t* m, const uint8_t* v, const float* ms,
                 const float* vs, int64_t n, float* mo, float* vo,
                 hipStream_t s);


struct GroupCall {
    svm_array X, weight, bias, Y;  // data NULL: not there
    int64_t positions = 1, groups = 1;
    float eps = 0.0f;
    int32_t act = SVM_ACT_NONE;
    float *mean = nullptr, *rstd = nullptr;
};
// Lays out the workspace in `ws`; with ws.run set it queues the work too.
void group_norm(const GroupCall& c, Pieces& ws, hipStream_t s);

struct GroupGradCall {
    svm_array dY, X, weight, bias, residual, dX, dweight, dbias;
    int64_t positions = 1, groups = 1;
    int32_t act = SVM_ACT_NONE;
    const float *mean = nullptr, *rstd = nullptr;
    bool sums = false;  // dweight or dbias is asked for
};
void group_norm_backward(const GroupGradCall& c, Pieces& ws, hipStream_t s);

// Sizes of weights in 4 bits: tiles of 16 outputs, chunks of 128 inputs,
// groups of a tile row, bytes of the codes and of all.
struct Shape4 {
    int64_t tiles, chunks, groups, code_bytes, bytes;
    int gshift;
    explicit Shape4(const svm_packed& w)
        : Shape4(w.rows, w.cols, w.group, w.dtype) {}
    Shape4(int64_t rows, int64_t cols, int32_t group, int32_t dtype)
        : tiles((rows + 15) / 16), chunks((cols + 127) / 128),
          groups(chunks * (128 / group)), code_bytes(tiles * chunks * 1024),
          bytes(code_bytes +
                tiles * groups * 16 * (int64_t)dtype_bytes(dtype)),
          gshift(group == 32 ? 5 : group == 64 ? 6 : 7)
    {
    }
};

void pack4(const svm_array& W, const svm_packed& to, hipStream_t s);
void unpack4(const svm_packed& w, const svm_array& W, hipStream_t s);

struct Linear4Call {
    svm_array X;
    svm_packed W;
    svm_array bias, residual, Y;  // data NULL: not there
    int32_t act = SVM_ACT_NONE;
};
// Lays out the workspace in `ws`; with ws.run set it queues the work too.
void linear4(const Linear4Call& a, Pieces& ws, hipStream_t s);

// The norm of n gradients as one vector, times |scale|, and the factor that
// brings it down to `most` (nullable).  Lays out `ws`, and queues with
// ws.run set.
void grad_norm(const svm_grad* g, int32_t n, double scale, double most,
               float* norm, float* factor, Pieces& ws, hipStream_t s);

}  // namespace msvm
