// The fused linear layer Y = act(X W^T + b) + R and its gradients.
#include "elem.hpp"
#include "layers.hpp"

namespace msvm {

namespace {

constexpr int kTile = 64;  // rows and columns of an output tile
constexpr int kStep = 16;  // of the summed index at a time

// C(i, j) = sum_r A(i, r) B(j, r); element (i, r) of A at A[i ai + r ar].
struct Product {
    const void *A, *B;
    int64_t ai, ar, bj, br;
    int64_t m, n, k;
};

// What happens to the sums: bias, pre-activations out, activation, residual.
struct Epilogue {
    const void *bias, *residual;
    void *Y, *Z;
    int64_t ldr, ldy, ldz;
    int act;
};

template <int DT>
__global__ __launch_bounds__(256) void k_product(Product p, Epilogue e)
{
    using T = Elem<DT>;
    __shared__ float As[kStep][kTile + 1], Bs[kStep][kTile + 1];
    const T* A = (const T*)p.A;
    const T* B = (const T*)p.B;
    const int t = threadIdx.x, tx = t & 15, ty = t >> 4;
    const int64_t i0 = (int64_t)blockIdx.y * kTile;
    const int64_t j0 = (int64_t)blockIdx.x * kTile;
    float acc[4][4] = {};
    for (int64_t r0 = 0; r0 < p.k; r0 += kStep) {
        for (int x = t; x < kTile * kStep; x += 256) {
            const int i = x / kStep, r = x % kStep;
            As[r][i] = i0 + i < p.m && r0 + r < p.k
                           ? (float)A[(i0 + i) * p.ai + (r0 + r) * p.ar]
                           : 0.0f;
            Bs[r][i] = j0 + i < p.n && r0 + r < p.k
                           ? (float)B[(j0 + i) * p.bj + (r0 + r) * p.br]
                           : 0.0f;
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < kStep; ++r)
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int v = 0; v < 4; ++v)
                    acc[u][v] = fmaf(As[r][ty * 4 + u], Bs[r][tx + 16 * v],
                                     acc[u][v]);
        __syncthreads();
    }
    for (int u = 0; u < 4; ++u) {
        const int64_t i = i0 + ty * 4 + u;
        if (i >= p.m) break;
        for (int v = 0; v < 4; ++v) {
            const int64_t j = j0 + tx + 16 * v;
            if (j >= p.n) break;
            float z = acc[u][v];
            if (e.bias) z += (float)((const T*)e.bias)[j];
            if (e.Z) ((T*)e.Z)[i * e.ldz + j] = (T)z;
            float y = act_value(e.act, z);
            if (e.residual) y += (float)((const T*)e.residual)[i * e.ldr + j];
            ((T*)e.Y)[i * e.ldy + j] = (T)y;
        }
    }
}

void launch_product(int32_t dtype, const Product& p, const Epilogue& e,
                    hipStream_t s)
{
    if (p.m == 0 || p.n == 0) return;
    // rows in slices of at most 65535 tiles (the grid's y)
    const int64_t slice = (int64_t)65535 * kTile;
    for (int64_t i0 = 0; i0 < p.m; i0 += slice) {
        Product q = p;
        Epilogue f = e;
        const size_t eb = dtype_bytes(dtype);
        q.m = p.m - i0 < slice ? p.m - i0 : slice;
        q.A = (const char*)p.A + i0 * p.ai * eb;
        f.Y = (char*)e.Y + i0 * e.ldy * eb;
        if (e.Z) f.Z = (char*)e.Z + i0 * e.ldz * eb;
        if (e.residual) f.residual = (const char*)e.residual + i0 * e.ldr * eb;
        const dim3 grid((unsigned)((p.n + kTile - 1) / kTile),
                        (unsigned)((q.m + kTile - 1) / kTile));
        for_dtype(dtype, [&]<int DT>() {
            hipLaunchKernelGGL((k_product<DT>), grid, dim3(256), 0, s, q, f);
        });
    }
}

// dZ = dY act'(Z), and the sums of its columns over this block's rows
constexpr int kGradRows = 64;

template <int DT>
__global__ __launch_bounds__(256) void k_act_grad(
    const void* dY_, int64_t ldg, const void* Z_, int64_t ldz, int act,
    int64_t m, int64_t n, void* dZ_, int64_t ldd, float* part)
{
    using T = Elem<DT>;
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= n) return;
    const int64_t i0 = (int64_t)blockIdx.y * kGradRows;
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

void linear_forward(const LinearArgs& a, Pieces& ws, hipStream_t s)
{
    if (!ws.run) return;
    Product p{a.X.data, a.W.data, a.X.ld, 1, a.W.ld, 1,
              a.X.rows, a.W.rows, a.X.cols};
    Epilogue e{a.bias.data, a.residual.data, a.Y.data, a.Z.data,
               a.residual.ld, a.Y.ld, a.Z.ld, a.act};
    launch_product(a.X.dtype, p, e, s);
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
        dZ.ld = n;
        dZ.data = ws.take<char>(m * n * dtype_bytes(t));
    }
    float* part = db ? ws.take<float>(np * n) : nullptr;
    if (!ws.run) return;
    if (np > 0 && (slope || db)) {
        for_dtype(t, [&]<int DT>() {
            // rows in slices of at most 65535 blocks (the grid's y)
            for (int64_t b0 = 0; b0 < np; b0 += 65535) {
                const int64_t nb = np - b0 < 65535 ? np - b0 : 65535;
                const int64_t i0 = b0 * kGradRows;
                using T = Elem<DT>;
                hipLaunchKernelGGL(
                    (k_act_grad<DT>),
                    dim3((unsigned)((n + 255) / 256), (unsigned)nb),
                    dim3(256), 0, s, (const T*)a.dY.data + i0 * a.dY.ld,
                    a.dY.ld,
                    slope ? (const T*)a.Z.data + i0 * a.Z.ld : nullptr,
                    a.Z.ld, a.act, m - i0, n,
                    slope && (dx || dw) ? (T*)dZ.data + i0 * dZ.ld : nullptr,
                    dZ.ld, db ? part + b0 * n : nullptr);
            }
        });
    }
    if (db)
        launch_column_sums(part, nullptr, np, n, t, a.dbias.data, nullptr, s);
    if (dx) {
        Product p{dZ.data, a.W.data, dZ.ld, 1, 1, a.W.ld, m, a.W.cols, n};
        Epilogue e{nullptr, nullptr, a.dX.data, nullptr,
                   0,       a.dX.ld, 0,         SVM_ACT_NONE};
        launch_product(t, p, e, s);
    }
    if (dw) {
        Product p{dZ.data, a.X.data, 1, dZ.ld, 1, a.X.ld, n, a.X.cols, m};
        Epilogue e{nullptr, nullptr, a.dW.data, nullptr,
                   0,       a.dW.ld, 0,         SVM_ACT_NONE};
        launch_product(t, p, e, s);
    }
}

}  // namespace msvm
