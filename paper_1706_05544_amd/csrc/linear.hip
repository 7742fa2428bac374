// The fused linear layer Y = act(X W^T + b) + R and its gradients.
#include "elem.hpp"
#include "matmul.hpp"

namespace msvm {

namespace {

// dZ = dY act'(Z) as a factor of the products (its rows end in zeros up to a
// multiple of 8), and the sums of its columns over this block's rows.  One
// pass over dY and Z: 8 columns to a thread, 32 threads side by side, 8 rows
// at once.  dZ is rounded to the arrays' type, as the 16-bit products need
// their factors; the sums take it unrounded.  Bound by memory: 8192 x 2048 in
// bf16 19.1 us, 5.3 TB/s.  (Done while the products load their tiles it would
// be computed once for each tile of W's columns, with the slopes of gelu.)
constexpr int kGradCols = 256, kGradLanes = 8;

struct GradArgs {
    const void *dY, *Z;
    int64_t ldg, ldz, m, n, rows;  // rows of a block
    void* dZ;
    int64_t ldd;
    float* part;  // the blocks' sums,
    void* sums;   // or the sums themselves, where one block has all rows
    int act;
};

template <int DT>
__global__ __launch_bounds__(256) void k_act_grad(GradArgs p)
{
    __shared__ float red[kGradLanes][kGradCols];
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    const int64_t j = (int64_t)blockIdx.x * kGradCols + tx * 8;
    const int64_t i0 = (int64_t)blockIdx.y * p.rows;
    const int64_t i1 = i0 + p.rows < p.m ? i0 + p.rows : p.m;
    const int count = eight_of(p.n, j);
    float sum[8] = {};
    if (count > 0) {
#pragma unroll 2
        for (int64_t i = i0 + ty; i < i1; i += kGradLanes) {
            Eight<DT> g, z;
            g.load(p.dY, i * p.ldg + j, count);
            if (p.Z) {
                z.load(p.Z, i * p.ldz + j, count);
                act_slopes(p.act, z.v);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    g.v[e] = e < count ? g.v[e] * z.v[e] : 0.0f;
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[e] += g.v[e];
            if (p.dZ) g.store(p.dZ, i * p.ldd + j, 8);
        }
    }
    if (!p.sums) return;
#pragma unroll
    for (int e = 0; e < 8; ++e) red[ty][tx * 8 + e] = sum[e];
    __syncthreads();
    const int64_t c = (int64_t)blockIdx.x * kGradCols + threadIdx.x;
    if (c >= p.n) return;
    float s = 0.0f;
#pragma unroll
    for (int r = 0; r < kGradLanes; ++r) s += red[r][threadIdx.x];
    if (gridDim.y == 1) ((Elem<DT>*)p.sums)[c] = (Elem<DT>)s;
    else p.part[blockIdx.y * p.n + c] = s;
}

// Rows of a block: some 2048 blocks in all, at least 16 rows to one; up to 64
// rows are left to one block, which spares the launch that joins the sums.
int64_t grad_rows(int64_t m, int64_t n)
{
    if (m <= 64) return 64;
    const int64_t across = (n + kGradCols - 1) / kGradCols;
    int64_t rows = (m * across + 2047) / 2048;
    rows = (rows + kGradLanes - 1) / kGradLanes * kGradLanes;
    return rows < 16 ? 16 : rows;
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

// Joins the blocks' sums in a fixed order, two arrays of them in one launch:
// 16 columns to a block, 16 threads to a column.  Bound by latency: 4 to 5 us,
// 9 for the two arrays of 768 rows by 4096.
template <int DT>
__global__ __launch_bounds__(256) void k_column_sums(
    const float* part0, const float* part1, int64_t np, int64_t cols,
    void* out0, void* out1)
{
    __shared__ float red[16][17];
    const float* part = blockIdx.y ? part1 : part0;
    void* out = blockIdx.y ? out1 : out0;
    if (!out) return;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int64_t j = (int64_t)blockIdx.x * 16 + tx;
    float sum = 0.0f;
    if (j < cols) {
#pragma unroll 8
        for (int64_t i = ty; i < np; i += 16) sum += part[i * cols + j];
    }
    red[ty][tx] = sum;
    __syncthreads();
    if (ty == 0 && j < cols) {
        sum = 0.0f;
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += red[r][tx];
        ((Elem<DT>*)out)[j] = (Elem<DT>)sum;
    }
}

}  // namespace

void launch_column_sums(const float* part0, const float* part1, int64_t np,
                        int64_t cols, int32_t dtype, void* out0, void* out1,
                        hipStream_t s)
{
    if (!out0 && !out1) return;
    for_dtype(dtype, [&]<int DT>() {
        hipLaunchKernelGGL((k_column_sums<DT>),
                           dim3((unsigned)((cols + 15) / 16), out1 ? 2 : 1),
                           dim3(256), 0, s, part0, part1, np, cols, out0, out1);
    });
}

// A factor of a product from an array: as it is where the product can read
// it so, else a copy in the workspace.
Factor factor_of(const svm_array& a, bool along, Pieces& ws, hipStream_t s)
{
    if (factor_fits(a, along)) return {a.data, a.ld, along};
    const int64_t ld = (a.cols + 7) / 8 * 8;
    void* copy = ws.take<char>(a.rows * ld * dtype_bytes(a.dtype));
    if (ws.run) launch_padded(a, copy, ld, s);
    return {copy, ld, along};
}

namespace {

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
    p.e = {a.bias.data, a.residual.data, a.Y.data, a.Z.data,
           a.residual.ld, a.Y.ld, a.Z.ld, a.act};
    if (few_rows(p.m, p.n, p.k)) {
        if (ws.run) few_rows_product(a.X, a.W, p.e, s);
        return;
    }
    p.A = factor_of(a.X, true, ws, s);
    p.B = factor_of(a.W, true, ws, s);
    product(p, ws, s);
}

void linear_backward(const LinearGradArgs& a, Pieces& ws, hipStream_t s)
{
    const int64_t m = a.dY.rows, n = a.dY.cols;
    const int32_t t = a.dY.dtype;
    const bool dx = a.dX.data, dw = a.dW.data, db = a.dbias.data;
    const bool slope = a.act != SVM_ACT_NONE;
    // dY itself serves as dZ where there is no slope and its rows can be
    // read as they are; else one pass makes dZ, and the sums with it
    const bool copy =
        (dx || dw) && (slope || !factor_fits(a.dY, dx));
    Factor dz{a.dY.data, a.dY.ld, true};
    if (copy) {
        dz.ld = (n + 7) / 8 * 8;
        dz.data = ws.take<char>(m * dz.ld * dtype_bytes(t));
    }
    const int64_t rows = grad_rows(m, n), np = (m + rows - 1) / rows;
    float* part = db && np > 1 ? ws.take<float>(np * n) : nullptr;
    if (ws.run && m > 0 && (copy || db)) {
        GradArgs g{a.dY.data, slope ? a.Z.data : nullptr,
                   a.dY.ld,   a.Z.ld,
                   m,         n,
                   rows,      copy ? const_cast<void*>(dz.data) : nullptr,
                   dz.ld,     part,
                   a.dbias.data, a.act};
        const dim3 grid((unsigned)((n + kGradCols - 1) / kGradCols),
                        (unsigned)np);
        for_dtype(t, [&]<int DT>() {
            hipLaunchKernelGGL((k_act_grad<DT>), grid, dim3(256), 0, s, g);
        });
    }
    if (ws.run && db && np != 1)
        launch_column_sums(part, nullptr, np, n, t, a.dbias.data, nullptr, s);
    if (!dx && !dw) return;
    if (m == 0) {
        if (dw && ws.run) launch_zero(a.dW, s);
        return;
    }
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
