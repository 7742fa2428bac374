// The matrix product of the feature-map operators (matmul.hip):
//   C(i, j) = sum_r A(i, r) B(j, r),  i < m, j < n, r < k,
// on the matrix cores, with what happens to the sums fused into its end.
#pragma once

#include "layers.hpp"

namespace msvm {

// One factor, in a 16-bit type.  along = true: element (i, r) at
// data[i ld + r] (the summed index along a row); else at data[r ld + i].
// 32-bit factors come as three bf16 planes whose sum is the factor.
struct Factor {
    const void* data;
    int64_t ld;
    int64_t plane;  // elements from one plane to the next
    bool along;
};

// What happens to the sums.
struct Epilogue {
    const void *bias, *residual;
    void *Y, *Z;
    int64_t ldr, ldy, ldz;
    int act;
};

struct Product {
    Factor A, B;
    int64_t m, n, k;
    int32_t dtype;  // of the outputs; SVM_F32: factors in three planes
    Epilogue e;
};

// Whether the product reads these values as they are: rows at multiples of
// 16 bytes, ld at most kMaxWidth, and (along) a multiple of 8 summed values.
bool factor_fits(const svm_array& a, bool along);

// Queues the product; with ws.run false only counts its workspace.
void product(const Product& p, Pieces& ws, hipStream_t s);

// The product of few rows X with W (both along), in one launch and without a
// workspace; and whether a product is one of these.
bool few_rows(int64_t m, int64_t n, int64_t k);
void few_rows_product(const svm_array& X, const svm_array& W,
                      const Epilogue& e, hipStream_t s);

// Copies rows of a into dst (ldp values to a row, a multiple of 8, zeros
// past the columns); float32 rows into three bf16 planes, `plane` apart.
void launch_planes(const svm_array& a, void* dst, int64_t ldp, int64_t plane,
                   hipStream_t s);

}  // namespace msvm
