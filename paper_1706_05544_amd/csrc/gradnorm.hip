// The norm of many gradients as one vector, and the factor that clips it.
//
// One pass over the values, read once, 16 bytes at a time.  Squares and sums
// are held in 64 bits: a 32-bit value's square leaves the range of 32 bits
// from 2e19 on, and the factor then does not depend on how the values fall
// into blocks.  A block takes units of kUnit values of one tensor in turn and
// leaves one sum; a second launch of one block adds those in a fixed order.
// Bound by memory: 70 million bf16 values 28.6 us with both launches, 4.9 TB/s
// (a large copy: 5.0); of few values by the launches, 3.8 and 1.7 us.
#include "elem.hpp"
#include "layers.hpp"

namespace msvm {

namespace {

constexpr int kUnit = 4096;         // values that a block takes at a time
constexpr int kGradBlocks = 2048;   // at most, in a launch
constexpr int kGradsPerLaunch = 128;

// The tensors of one launch travel in its arguments.
struct GradTable {
    const void* data[kGradsPerLaunch];
    int64_t n[kGradsPerLaunch];
    int32_t first[kGradsPerLaunch + 1];  // first unit of each tensor
    int8_t dtype[kGradsPerLaunch];
    int32_t count;
};

__device__ __forceinline__ double wave_sum64(double v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

template <int DT>
__device__ __forceinline__ void add_squares(const void* data, int64_t n,
                                            int64_t at, double (&sum)[2])
{
    Eight<DT> x[2];
#pragma unroll
    for (int p = 0; p < 2; ++p)
        x[p].load(data, at + p * (kUnit / 2), eight_of(n, at + p * (kUnit / 2)));
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const double v = (double)x[p].v[e];
            sum[p] = fma(v, v, sum[p]);
        }
}

__global__ __launch_bounds__(256) void k_grad_squares(GradTable t,
                                                      double* part)
{
    __shared__ double red[4];
    double sum[2] = {0.0, 0.0};
    const int units = t.first[t.count];
    for (int u = (int)blockIdx.x; u < units; u += (int)gridDim.x) {
        int lo = 0, hi = t.count - 1;  // the tensor of this unit
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (t.first[mid] <= u) lo = mid; else hi = mid - 1;
        }
        const int64_t at = (int64_t)(u - t.first[lo]) * kUnit + threadIdx.x * 8;
        if (t.dtype[lo] == SVM_F32)
            add_squares<SVM_F32>(t.data[lo], t.n[lo], at, sum);
        else if (t.dtype[lo] == SVM_BF16)
            add_squares<SVM_BF16>(t.data[lo], t.n[lo], at, sum);
        else
            add_squares<SVM_F16>(t.data[lo], t.n[lo], at, sum);
    }
    const double s = wave_sum64(sum[0] + sum[1]);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) part[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// A NaN or an infinity anywhere leaves a sum that is not finite, and then the
// factor is NaN: no step can take such gradients for clipped ones.
__global__ __launch_bounds__(256) void k_grad_norm(const double* part,
                                                   int64_t np, double scale,
                                                   double most, float* norm,
                                                   float* factor)
{
    __shared__ double red[4];
    double sum = 0.0;
#pragma unroll 4
    for (int64_t i = threadIdx.x; i < np; i += 256) sum += part[i];
    sum = wave_sum64(sum);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x) return;
    const double all =
        sqrt((red[0] + red[1]) + (red[2] + red[3])) * fabs(scale);
    *norm = (float)all;
    if (factor)
        *factor = !(all <= 1.7976931348623157e308) ? __builtin_nanf("")
                  : all > most                     ? (float)(most / all)
                                                   : 1.0f;
}

int64_t units_of(int64_t n) { return (n + kUnit - 1) / kUnit; }

// Calls f(table) for each launch: tensors in their order, long ones in pieces
// (unit numbers are int32).
template <class F>
void for_grad_tables(const svm_grad* g, int32_t n, F&& f)
{
    constexpr int64_t kMost = (int64_t)kUnit << 20;
    GradTable t;
    t.count = 0;
    t.first[0] = 0;
    for (int32_t i = 0; i < n; ++i)
        for (int64_t at = 0; at < g[i].n; at += kMost) {
            const int64_t len = g[i].n - at < kMost ? g[i].n - at : kMost;
            if (t.count == kGradsPerLaunch || t.first[t.count] >= 1 << 29) {
                f(t);
                t.count = 0;
            }
            const int c = t.count++;
            t.data[c] = (const char*)g[i].data + at * dtype_bytes(g[i].dtype);
            t.n[c] = len;
            t.dtype[c] = (int8_t)g[i].dtype;
            t.first[c + 1] = t.first[c] + (int32_t)units_of(len);
        }
    if (t.count) f(t);
}

int64_t blocks_of(const GradTable& t)
{
    const int32_t units = t.first[t.count];
    return units < kGradBlocks ? units : kGradBlocks;
}

}  // namespace

void grad_norm(const svm_grad* g, int32_t n, double scale, double most,
               float* norm, float* factor, Pieces& ws, hipStream_t s)
{
    int64_t np = 0;
    for_grad_tables(g, n, [&](const GradTable& t) { np += blocks_of(t); });
    double* part = ws.take<double>(np);
    if (!ws.run) return;
    double* at = part;
    for_grad_tables(g, n, [&](const GradTable& t) {
        hipLaunchKernelGGL(k_grad_squares, dim3((unsigned)blocks_of(t)),
                           dim3(256), 0, s, t, at);
        at += blocks_of(t);
    });
    hipLaunchKernelGGL(k_grad_norm, dim3(1), dim3(256), 0, s, part, np, scale,
                       most, norm, factor);
}

}  // namespace msvm
