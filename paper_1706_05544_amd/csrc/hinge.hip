// Squared hinge loss, one class against the rest, and its gradient.
#include "elem.hpp"
#include "layers.hpp"

namespace msvm {

namespace {

constexpr int64_t kParts = 1024;  // blocks, each with its own partial sum

int64_t parts_of(int64_t rows, int64_t cols)
{
    const int64_t p = (rows * cols + 1023) / 1024;
    return p < kParts ? p : kParts;
}

template <int DT>
__global__ __launch_bounds__(256) void k_hinge(
    const Elem<DT>* S, int64_t lds, const int32_t* labels, float scale,
    int64_t m, int64_t n, Elem<DT>* dS, int64_t ldd, double* part)
{
    __shared__ double red[256];
    const int64_t total = m * n;
    double sum = 0.0;
    for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < total;
         e += (int64_t)gridDim.x * 256) {
        const int64_t i = e / n, c = e % n;
        const int32_t lab = labels[i];
        const bool seen = lab >= 0 && lab < (n == 1 ? 2 : n);
        const float y = lab == (n == 1 ? 1 : c) ? 1.0f : -1.0f;
        float gap = 1.0f - y * (float)S[i * lds + c];
        gap = !seen || gap <= 0.0f ? 0.0f : gap;
        sum += (double)(gap * gap);
        if (dS) dS[i * ldd + c] = (Elem<DT>)(-2.0f * scale * y * gap);
    }
    red[threadIdx.x] = sum;
    for (int h = 128; h > 0; h >>= 1) {
        __syncthreads();
        if ((int)threadIdx.x < h) red[threadIdx.x] += red[threadIdx.x + h];
    }
    if (threadIdx.x == 0) part[blockIdx.x] = red[0];
}

__global__ __launch_bounds__(256) void k_hinge_sum(const double* part,
                                                   int64_t np, float scale,
                                                   float* loss)
{
    __shared__ double red[256];
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < np; i += 256) sum += part[i];
    red[threadIdx.x] = sum;
    for (int h = 128; h > 0; h >>= 1) {
        __syncthreads();
        if ((int)threadIdx.x < h) red[threadIdx.x] += red[threadIdx.x + h];
    }
    if (threadIdx.x == 0) *loss = (float)(red[0] * (double)scale);
}

}  // namespace

int64_t hinge_bytes(int64_t rows, int64_t cols)
{
    Pieces p;
    p.take<double>(parts_of(rows, cols));
    return p.used;
}

void hinge_loss(const svm_array& S, const int32_t* labels, float scale,
                const svm_array& dS, float* loss, Pieces& ws, hipStream_t s)
{
    const int64_t np = parts_of(S.rows, S.cols);
    double* part = ws.take<double>(np);
    if (np > 0)
        for_dtype(S.dtype, [&]<int DT>() {
            using T = Elem<DT>;
            hipLaunchKernelGGL((k_hinge<DT>), dim3((unsigned)np), dim3(256), 0,
                               s, (const T*)S.data, S.ld, labels, scale,
                               S.rows, S.cols, (T*)dS.data, dS.ld, part);
        });
    hipLaunchKernelGGL(k_hinge_sum, dim3(1), dim3(256), 0, s, part, np, scale,
                       loss);
}

}  // namespace msvm
