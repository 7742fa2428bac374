// Squared hinge loss, one class against the rest, and its gradient.
//
// One read of the scores and one write of their gradient, 8 values of the
// flattened matrix to a thread; the squares are summed in 64 bits, in a fixed
// order.  Up to kOneBlock scores one block does it all, in one launch: the
// launch is then what the call costs (256 x 1: 3.2 us of 11 to 12); beyond, the
// blocks' sums are joined by a second one.  500000 x 10 in 32 bits: 11.3 us
// and 2.2 for the join, where 42 MB at a large copy's rate are 8.2: of the 2048
// blocks 394 have a second turn, for which the others do not wait but the join
// does.  Whether a score is its row's own class is
// found from the flat index (one division, in 32 bits, for 8 scores), so
// that loads and stores are whole lines for any number of classes.
#include "elem.hpp"
#include "layers.hpp"

namespace msvm {

namespace {

constexpr int64_t kOneBlock = 32768;
constexpr int kOneThreads = 1024, kManyThreads = 256;
constexpr int64_t kMostParts = 2048;

int64_t parts_of(int64_t rows, int64_t cols)
{
    const int64_t p = (rows * cols + kManyThreads * 8 - 1) / (kManyThreads * 8);
    return p < kMostParts ? p : kMostParts;
}

// Sum over the block, for thread 0.
template <int THREADS>
__device__ __forceinline__ double block_total(double v)
{
    __shared__ double red[THREADS / 64];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
    if (threadIdx.x == 0)
        for (int w = 0; w < THREADS / 64; ++w) v += red[w];
    return v;
}

struct HingeView {
    const void* S;
    void* dS;
    int64_t lds, ldd, m, n;
    const int32_t* labels;
    float scale;
    double* part;  // a sum for each block
    float* loss;   // one block: the loss itself
};

template <int DT, int THREADS>
__global__ __launch_bounds__(THREADS) void k_hinge(HingeView p)
{
    const int64_t total = p.m * p.n;
    const int32_t classes = p.n == 1 ? 2 : (int32_t)p.n;
    const float slope = -2.0f * p.scale;
    double sum = 0.0;
    for (int64_t e0 = ((int64_t)blockIdx.x * THREADS + threadIdx.x) * 8;
         e0 < total; e0 += (int64_t)gridDim.x * THREADS * 8) {
        const int count = eight_of(total, e0);
        int64_t i = quotient(e0, p.n, total);
        int32_t c = (int32_t)(e0 - i * p.n);
        Eight<DT> x, d;
        const bool flat = p.lds == p.n;
        if (flat) x.load(p.S, e0, count);
        int32_t lab = p.labels[i];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (e < count) {
                if (!flat)
                    x.v[e] = (float)((const Elem<DT>*)p.S)[i * p.lds + c];
                const bool seen = lab >= 0 && lab < classes;
                const bool at = lab == (p.n == 1 ? 1 : c);
                float gap = at ? 1.0f - x.v[e] : 1.0f + x.v[e];
                gap = !seen || gap <= 0.0f ? 0.0f : gap;
                sum += (double)(gap * gap);
                d.v[e] = at ? slope * gap : -slope * gap;
                if (p.dS && p.ldd != p.n)
                    ((Elem<DT>*)p.dS)[i * p.ldd + c] = (Elem<DT>)d.v[e];
                if (++c == p.n && e + 1 < count) {
                    c = 0;
                    lab = p.labels[++i];
                }
            }
        }
        if (p.dS && p.ldd == p.n) d.store(p.dS, e0, count);
    }
    sum = block_total<THREADS>(sum);
    if (threadIdx.x != 0) return;
    if (THREADS == kOneThreads) *p.loss = (float)(sum * (double)p.scale);
    else p.part[blockIdx.x] = sum;
}

__global__ __launch_bounds__(kManyThreads) void k_hinge_sum(
    const double* part, int64_t np, float scale, float* loss)
{
    double sum = 0.0;
#pragma unroll 8
    for (int64_t i = threadIdx.x; i < np; i += kManyThreads) sum += part[i];
    sum = block_total<kManyThreads>(sum);
    if (threadIdx.x == 0) *loss = (float)(sum * (double)scale);
}

}  // namespace

int64_t hinge_bytes(int64_t rows, int64_t cols)
{
    if (rows * cols <= kOneBlock) return 0;
    Pieces p;
    p.take<double>(parts_of(rows, cols));
    return p.used;
}

void hinge_loss(const svm_array& S, const int32_t* labels, float scale,
                const svm_array& dS, float* loss, Pieces& ws, hipStream_t s)
{
    HingeView v{S.data, dS.data, S.ld,  dS.ld,   S.rows,
                S.cols, labels,  scale, nullptr, loss};
    const bool one = S.rows * S.cols <= kOneBlock;
    const int64_t np = one ? 1 : parts_of(S.rows, S.cols);
    if (!one) v.part = ws.take<double>(np);
    for_dtype(S.dtype, [&]<int DT>() {
        if (one)
            hipLaunchKernelGGL((k_hinge<DT, kOneThreads>), dim3(1),
                               dim3(kOneThreads), 0, s, v);
        else
            hipLaunchKernelGGL((k_hinge<DT, kManyThreads>), dim3((unsigned)np),
                               dim3(kManyThreads), 0, s, v);
    });
    if (!one)
        hipLaunchKernelGGL(k_hinge_sum, dim3(1), dim3(kManyThreads), 0, s,
                           v.part, np, scale, loss);
}

}  // namespace msvm
