// Layer norm of the rows of a matrix, and its gradients.
#include "elem.hpp"
#include "layers.hpp"

namespace msvm {

namespace {

// Sum over a block of 256 threads, for every thread.
__device__ __forceinline__ float block_sum(float v, float* red)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return red[0] + red[1] + red[2] + red[3];
}

template <int DT>
__global__ __launch_bounds__(256) void k_norm(const Elem<DT>* X, int64_t ldx,
                                              const Elem<DT>* w,
                                              const Elem<DT>* b, float eps,
                                              int64_t n, Elem<DT>* Y,
                                              int64_t ldy, float* mean,
                                              float* rstd)
{
    __shared__ float red[4];
    const int64_t i = blockIdx.x;
    const Elem<DT>* x = X + i * ldx;
    float sum = 0.0f;
    for (int64_t j = threadIdx.x; j < n; j += 256) sum += (float)x[j];
    const float mu = block_sum(sum, red) / (float)n;
    float sq = 0.0f;
    for (int64_t j = threadIdx.x; j < n; j += 256) {
        const float d = (float)x[j] - mu;
        sq = fmaf(d, d, sq);
    }
    const float rs = 1.0f / sqrtf(block_sum(sq, red) / (float)n + eps);
    if (threadIdx.x == 0) {
        if (mean) mean[i] = mu;
        if (rstd) rstd[i] = rs;
    }
    for (int64_t j = threadIdx.x; j < n; j += 256) {
        float y = ((float)x[j] - mu) * rs;
        if (w) y *= (float)w[j];
        if (b) y += (float)b[j];
        Y[i * ldy + j] = (Elem<DT>)y;
    }
}

template <int DT>
__global__ __launch_bounds__(256) void k_norm_grad(
    const Elem<DT>* dY, int64_t ldg, const Elem<DT>* X, int64_t ldx,
    const float* mean, const float* rstd, const Elem<DT>* w,
    const Elem<DT>* res, int64_t ldr, int64_t n, Elem<DT>* dX, int64_t ldd)
{
    __shared__ float red[4];
    const int64_t i = blockIdx.x;
    const Elem<DT>*g = dY + i * ldg, *x = X + i * ldx;
    const float mu = mean[i], rs = rstd[i];
    float s1 = 0.0f, s2 = 0.0f;
    for (int64_t j = threadIdx.x; j < n; j += 256) {
        const float a = (float)g[j] * (w ? (float)w[j] : 1.0f);
        s1 += a;
        s2 = fmaf(a, ((float)x[j] - mu) * rs, s2);
    }
    s1 = block_sum(s1, red) / (float)n;
    s2 = block_sum(s2, red) / (float)n;
    for (int64_t j = threadIdx.x; j < n; j += 256) {
        const float a = (float)g[j] * (w ? (float)w[j] : 1.0f);
        const float xh = ((float)x[j] - mu) * rs;
        float d = rs * (a - s1 - xh * s2);
        if (res) d += (float)res[i * ldr + j];
        dX[i * ldd + j] = (Elem<DT>)d;
    }
}

constexpr int kSumRows = 256;  // rows of a partial sum, at least

int64_t partials(int64_t rows)
{
    const int64_t p = (rows + kSumRows - 1) / kSumRows;
    return p < 1024 ? p : 1024;
}

template <int DT>
__global__ __launch_bounds__(256) void k_norm_sums(
    const Elem<DT>* dY, int64_t ldg, const Elem<DT>* X, int64_t ldx,
    const float* mean, const float* rstd, int64_t m, int64_t n, int64_t per,
    float* pw, float* pb)
{
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= n) return;
    const int64_t i0 = blockIdx.y * per;
    const int64_t i1 = i0 + per < m ? i0 + per : m;
    float sw = 0.0f, sb = 0.0f;
    for (int64_t i = i0; i < i1; ++i) {
        const float g = (float)dY[i * ldg + j];
        sb += g;
        sw = fmaf(g, ((float)X[i * ldx + j] - mean[i]) * rstd[i], sw);
    }
    pw[blockIdx.y * n + j] = sw;
    pb[blockIdx.y * n + j] = sb;
}

}  // namespace

void norm_forward(const NormArgs& a, hipStream_t s)
{
    for_dtype(a.X.dtype, [&]<int DT>() {
        using T = Elem<DT>;
        hipLaunchKernelGGL((k_norm<DT>), dim3((unsigned)a.X.rows), dim3(256),
                           0, s, (const T*)a.X.data, a.X.ld,
                           (const T*)a.weight.data, (const T*)a.bias.data,
                           a.eps, a.X.cols, (T*)a.Y.data, a.Y.ld, a.mean,
                           a.rstd);
    });
}

int64_t norm_backward_bytes(int64_t rows, int64_t cols)
{
    Pieces p;
    p.take<float>(partials(rows) * cols);
    p.take<float>(partials(rows) * cols);
    return p.used;
}

void norm_backward(const NormGradArgs& a, Pieces& ws, hipStream_t s)
{
    const int64_t m = a.X.rows, n = a.X.cols;
    for_dtype(a.X.dtype, [&]<int DT>() {
        using T = Elem<DT>;
        const T *dY = (const T*)a.dY.data, *X = (const T*)a.X.data;
        if (a.dweight.data || a.dbias.data) {
            const int64_t np = partials(m);
            float* pw = ws.take<float>(np * n);
            float* pb = ws.take<float>(np * n);
            if (np > 0)
                hipLaunchKernelGGL(
                    (k_norm_sums<DT>),
                    dim3((unsigned)((n + 255) / 256), (unsigned)np), dim3(256),
                    0, s, dY, a.dY.ld, X, a.X.ld, a.mean, a.rstd, m, n,
                    np ? (m + np - 1) / np : 0, pw, pb);
            launch_column_sums(pw, pb, np, n, a.X.dtype, a.dweight.data,
                               a.dbias.data, s);
        }
        if (a.dX.data && m > 0)
            hipLaunchKernelGGL((k_norm_grad<DT>), dim3((unsigned)m),
                               dim3(256), 0, s, dY, a.dY.ld, X, a.X.ld, a.mean,
                               a.rstd, (const T*)a.weight.data,
                               (const T*)a.residual.data, a.residual.ld, n,
                               (T*)a.dX.data, a.dX.ld);
    });
}

}  // namespace msvm
