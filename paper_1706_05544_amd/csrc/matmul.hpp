// The matrix product of the feature-map operators (matmul.hip):
//   C(i, j) = sum_r A(i, r) B(j, r),  i < m, j < n, r < k,
// on the matrix cores, with what happens to the sums fused into its end.
#pragma once

#include "layers.hpp"

namespace msvm {

// One factor.  along = true: element (i, r) at data[i ld + r] (the summed
// index along a row); else at data[r ld + i].
struct Factor {
    const void* data;
    int64_t ld;
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
    int32_t dtype;
    Epilogue e;
    // SVM_F32, both factors along: the values of B are those of bf16 too
    bool narrow = false;
};

// Whether the product reads these values as they are: with ld at most
// kMaxWidth, 16-bit ones in rows at multiples of 16 bytes and (along) of a
// multiple of 8 summed values, or with zeros up to one.
bool factor_fits(const svm_array& a, bool along);

// A factor of a product from an array: as it is where the product can read
// it so, else a copy in the workspace.
Factor factor_of(const svm_array& a, bool along, Pieces& ws, hipStream_t s);

// Queues the product; with ws.run false only counts its workspace.
void product(const Product& p, Pieces& ws, hipStream_t s);

// The product of few rows X with W (both along), in one launch and without a
// workspace; and whether a product is one of these.
bool few_rows(int64_t m, int64_t n, int64_t k);
void few_rows_product(const svm_array& X, const svm_array& W,
                      const Epilogue& e, hipStream_t s);

// Copies the rows of an array into dst: ldp values to a row, a multiple of 8,
// zeros past the columns.
void launch_padded(const svm_array& a, void* dst, int64_t ldp, hipStream_t s);

}  // namespace msvm
