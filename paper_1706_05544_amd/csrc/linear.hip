// The fused linear layer Y = act(X W^T + b) + R and its gradients.
#include "elem.hpp"
#include "matmul.hpp"

namespace msvm {

namespace {

// dZ = dY act'(Z), and the sums of its columns over this block's rows
constexpr int kGradRows = 64;

template <int DT>
__global__ __launch_bounds__(256) void k_act_grad(
    const void* dY_, int64_t ldg, const void* Z_, int64_t ldz, int act,
    int64_t m, int64_t n, void* dZ_, int64_t ldd, float* part)
{
    using T = Elem<DT>;
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t i0 = (int64_t)blockIdx.y * kGradRows;
    if (j >= n) {  // the zeros that end the rows of dZ
        if (dZ_ && j < ldd)
            for (int64_t i = i0; i < m && i < i0 + kGradRows; ++i)
                ((T*)dZ_)[i * ldd + j] = (T)0.0f;
        return;
    }
    const int64_t i1 = i0 + kGradRows < m ? i0 + kGradRows : m;
    float sum = 0.0f;
    for (int64_t i = i0; i < i1; ++i) {
        float g = (float)((const T*)dY_)[i * ldg + j];
        if (Z_) g *= act_slope(act, (float)((const T*)Z_)[i * ldz + j]);
        sum += g;
        if (dZ_) ((T*)dZ_)[i * ldd + j] = (T)g;
    }
    if (part) part[(int64_t)blockIdx.y * n + j] = sum;
}

// Zeros to rows x cols of an array.
template <int DT>
__global__ __launch_bounds__(256) void k_zero(Elem<DT>* out, int64_t ld,
                                              int64_t rows, int64_t cols)
{
    const int64_t all = rows * cols;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < all;
         t += (int64_t)gridDim.x * 256)
        out[t / cols * ld + t % cols] = (Elem<DT>)0.0f;
}

void launch_zero(const svm_array& a, hipStream_t s)
{
    const int64_t nb = (a.rows * a.cols + 255) / 256;
    for_dtype(a.dtype, [&]<int DT>() {
        hipLaunchKernelGGL((k_zero<DT>),
                           dim3((unsigned)(nb < 4096 ? nb : 4096)), dim3(256),
                           0, s, (Elem<DT>*)a.data, a.ld, a.rows, a.cols);
    });
}

template <int DT>
__global__ __launch_bounds__(256) void k_column_sums(
    const float* part0, const float* part1, int64_t np, int64_t cols,
    void* out0, void* out1)
{
    const float* part = blockIdx.y ? part1 : part0;
    void* out = blockIdx.y ? out1 : out0;
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= cols || !out) return;
    double sum = 0.0;
    for (int64_t i = 0; i < np; ++i) sum += part[i * cols + j];
    ((Elem<DT>*)out)[j] = (Elem<DT>)(float)sum;
}

}  // namespace

void launch_column_sums(const float* part0, const float* part1, int64_t np,
                        int64_t cols, int32_t dtype, void* out0, void* out1,
                        hipStream_t s)
{
    if (!out0 && !out1) return;
    for_dtype(dtype, [&]<int DT>() {
        hipLaunchKernelGGL((k_column_sums<DT>),
                           dim3((unsigned)((cols + 255) / 256), 2), dim3(256),
                           0, s, part0, part1, np, cols, out0, out1);
    });
}

namespace {

// A factor of a product from an array: as it is where the product can read
// it so, else a copy in the workspace (32 bits: in three planes).
Factor factor_of(const svm_array& a, bool along, Pieces& ws, hipStream_t s)
{
    Factor f{a.data, a.ld, 0, along, (const float*)a.data, a.ld};
    if (factor_fits(a, along)) return f;
    f.ld = (a.cols + 7) / 8 * 8;
    f.plane = a.rows * f.ld;
    void* copy = ws.take<uint16_t>((a.dtype == SVM_F32 ? 3 : 1) * f.plane);
    f.data = copy;
    if (ws.run) launch_planes(a, copy, f.ld, f.plane, s);
    return f;
}

Epilogue plain(const svm_array& out)
{
    return {nullptr, nullptr, out.data, nullptr, 0, out.ld, 0, SVM_ACT_NONE};
}

}  // namespace

void linear_forward(const LinearArgs& a, Pieces& ws, hipStream_t s)
{
    Product p;
    p.m = a.X.rows;
    p.n = a.W.rows;
    p.k = a.X.cols;
    p.dtype = a.X.dtype;
    if (p.m == 0) return;
    p.A = factor_of(a.X, true, ws, s);
    p.B = factor_of(a.W, true, ws, s);
    p.e = {a.bias.data, a.residual.data, a.Y.data, a.Z.data,
           a.residual.ld, a.Y.ld, a.Z.ld, a.act};
    product(p, ws, s);
}

void linear_backward(const LinearGradArgs& a, Pieces& ws, hipStream_t s)
{
    const int64_t m = a.dY.rows, n = a.dY.cols;
    const int32_t t = a.dY.dtype;
    const bool dx = a.dX.data, dw = a.dW.data, db = a.dbias.data;
    const bool slope = a.act != SVM_ACT_NONE;
    const int64_t np = (m + kGradRows - 1) / kGradRows;
    svm_array dZ = a.dY;
    if (slope && (dx || dw)) {
        dZ.ld = (n + 7) / 8 * 8;
        dZ.data = ws.take<char>(m * dZ.ld * dtype_bytes(t));
    }
    float* part = db ? ws.take<float>(np * n) : nullptr;
    if (ws.run && np > 0 && (slope || db)) {
        for_dtype(t, [&]<int DT>() {
            // rows in slices of at most 65535 blocks (the grid's y)
            for (int64_t b0 = 0; b0 < np; b0 += 65535) {
                const int64_t nb = np - b0 < 65535 ? np - b0 : 65535;
                const int64_t i0 = b0 * kGradRows;
                using T = Elem<DT>;
                hipLaunchKernelGGL(
                    (k_act_grad<DT>),
                    dim3((unsigned)((dZ.ld + 255) / 256), (unsigned)nb),
                    dim3(256), 0, s, (const T*)a.dY.data + i0 * a.dY.ld,
                    a.dY.ld,
                    slope ? (const T*)a.Z.data + i0 * a.Z.ld : nullptr,
                    a.Z.ld, a.act, m - i0, n,
                    slope && (dx || dw) ? (T*)dZ.data + i0 * dZ.ld : nullptr,
                    dZ.ld, db ? part + b0 * n : nullptr);
            }
        });
    }
    if (ws.run && db)
        launch_column_sums(part, nullptr, np, n, t, a.dbias.data, nullptr, s);
    if (!dx && !dw) return;
    if (m == 0) {
        if (dw && ws.run) launch_zero(a.dW, s);
        return;
    }
    // both products read one copy of dZ, where it has to be copied at all
    svm_array part_dz = dZ;
    Factor dz;
    if (dx && slope && t != SVM_F32) {
        // the workspace's own rows end in zeros up to a multiple of 8
        part_dz.cols = dZ.ld;
    }
    dz = factor_of(part_dz, dx, ws, s);
    if (dx) {
        Product p;
        p.A = dz;
        p.A.along = true;
        p.B = factor_of(a.W, false, ws, s);
        p.m = m;
        p.n = a.W.cols;
        p.k = n;
        p.dtype = t;
        p.e = plain(a.dX);
        product(p, ws, s);
    }
    if (dw) {
        Product p;
        p.A = dz;
        p.A.along = false;
        p.B = factor_of(a.X, false, ws, s);
        p.m = n;
        p.n = a.X.cols;
        p.k = m;
        p.dtype = t;
        p.e = plain(a.dW);
        product(p, ws, s);
    }
}

}  // namespace msvm
