// Layer norm of the rows of a matrix, and its gradients.
//
// A row belongs to G lanes (a part of a wave, a wave, or a whole block), each
// with IT pieces of 8 columns, and is read once: it stays in registers
// between the mean, the sum of the squared deviations and the output.  The
// gradient reads dY and X once for dX and for the sums over the rows: a lane
// has the same columns in every row that its group takes, adds up their terms
// in registers, and the groups of a block and then the blocks are joined at
// the end, in a fixed order.  Rows of more than kMostCols columns are read
// again for each sum.
//
// All kernels are bound by memory.  Measured, with the launches: 100000 x 128
// in 32 bits 20.1 us, 5.1 TB/s, which is what a large copy reaches; gradient
// of 16384 x 4096 in bf16 with a residual branch 114 us, of which 9 join the
// sums (a copy of as many bytes: 104); of 68971 x 501 in 32 bits, whose rows
// begin anywhere, 91 us (81).  The counters show every array read and written
// once.  The wide rows, which are read again: 2048 x 32768 in 32 bits 162 us
// (104 if each byte moved once), its gradients 312 (156); in bf16 70 (52) and
// 170 (78).
#include "elem.hpp"
#include "layers.hpp"

namespace msvm {

namespace {

constexpr int64_t kMostCols = 16384;

// Sums of a and b over the G lanes of a row's group; every lane ends with
// them.  red: two floats for each wave of the block.
template <int G>
__device__ __forceinline__ void group_sums(float& a, float& b, float* red)
{
    constexpr int kLane = G < 64 ? G : 64;
#pragma unroll
    for (int off = kLane / 2; off > 0; off >>= 1) {
        a += __shfl_xor(a, off);
        b += __shfl_xor(b, off);
    }
    if constexpr (G > 64) {
        constexpr int kWaves = G / 64;
        const int w = threadIdx.x >> 6;
        __syncthreads();  // the last sums have been read
        if ((threadIdx.x & 63) == 0) red[w] = a, red[kWaves + w] = b;
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int i = 0; i < kWaves; ++i) a += red[i], b += red[kWaves + i];
    }
}

template <int G>
__device__ __forceinline__ float group_sum(float a, float* red)
{
    float b = 0.0f;
    group_sums<G>(a, b, red);
    return a;
}

// The row of a group's next turn lies this far on, and the loop ends for all
// groups of a block together where a row takes the whole block.
template <int G>
constexpr int kThreads = G > 256 ? G : 256;

struct NormView {
    const void *X, *w, *b;
    void* Y;
    int64_t ldx, ldy, m, n;
    float *mean, *rstd;
    float eps;
};

template <int DT, int G, int IT>
__global__ __launch_bounds__(kThreads<G>) void k_norm(NormView p)
{
    constexpr int kGroups = kThreads<G> / G;
    __shared__ float red[G > 64 ? 2 * (G / 64) : 1];
    const int lane = threadIdx.x % G, group = threadIdx.x / G;
    Eight<DT> w[IT], b[IT];
    int count[IT];
#pragma unroll
    for (int t = 0; t < IT; ++t) {
        const int64_t j = ((int64_t)t * G + lane) * 8;
        count[t] = eight_of(p.n, j);
#pragma unroll
        for (int e = 0; e < 8; ++e) w[t].v[e] = 1.0f, b[t].v[e] = 0.0f;
        if (p.w) w[t].load(p.w, j, count[t]);
        if (p.b) b[t].load(p.b, j, count[t]);
    }
    // (divided by, not multiplied by its reciprocal: the mean of a constant
    // row is its value)
    const float cols = (float)p.n;
    for (int64_t i = (int64_t)blockIdx.x * kGroups + group; i < p.m;
         i += (int64_t)gridDim.x * kGroups) {
        Eight<DT> x[IT];
        float s = 0.0f;
#pragma unroll
        for (int t = 0; t < IT; ++t) {
            x[t].load(p.X, i * p.ldx + ((int64_t)t * G + lane) * 8, count[t]);
#pragma unroll
            for (int e = 0; e < 8; ++e) s += x[t].v[e];
        }
        const float mu = group_sum<G>(s, red) / cols;
        s = 0.0f;
#pragma unroll
        for (int t = 0; t < IT; ++t)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[t].v[e] -= mu;
                if (e < count[t]) s = fmaf(x[t].v[e], x[t].v[e], s);
            }
        const float rs =
            1.0f / sqrtf(group_sum<G>(s, red) / cols + p.eps);
        if (lane == 0) {
            if (p.mean) p.mean[i] = mu;
            if (p.rstd) p.rstd[i] = rs;
        }
#pragma unroll
        for (int t = 0; t < IT; ++t) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                x[t].v[e] = fmaf(x[t].v[e] * rs, w[t].v[e], b[t].v[e]);
            x[t].store(p.Y, i * p.ldy + ((int64_t)t * G + lane) * 8, count[t]);
        }
    }
}

// Rows wider than the registers of a block: three passes over each, of which
// the second and third find it in the L2 cache.
template <int DT>
__global__ __launch_bounds__(1024) void k_norm_wide(NormView p)
{
    constexpr int G = 1024;
    __shared__ float red[2 * (G / 64)];
    // (divided by, not multiplied by its reciprocal: the mean of a constant
    // row is its value)
    const float cols = (float)p.n;
    for (int64_t i = blockIdx.x; i < p.m; i += gridDim.x) {
        float s = 0.0f;
        Eight<DT> x, w, b;
        for (int64_t j = threadIdx.x * 8; j < p.n; j += G * 8) {
            x.load(p.X, i * p.ldx + j, eight_of(p.n, j));
#pragma unroll
            for (int e = 0; e < 8; ++e) s += x.v[e];
        }
        const float mu = group_sum<G>(s, red) / cols;
        s = 0.0f;
        for (int64_t j = threadIdx.x * 8; j < p.n; j += G * 8) {
            const int count = eight_of(p.n, j);
            x.load(p.X, i * p.ldx + j, count);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < count) s = fmaf(x.v[e] - mu, x.v[e] - mu, s);
        }
        const float rs =
            1.0f / sqrtf(group_sum<G>(s, red) / cols + p.eps);
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[i] = mu;
            if (p.rstd) p.rstd[i] = rs;
        }
        for (int64_t j = threadIdx.x * 8; j < p.n; j += G * 8) {
            const int count = eight_of(p.n, j);
            x.load(p.X, i * p.ldx + j, count);
            if (p.w) w.load(p.w, j, count);
            if (p.b) b.load(p.b, j, count);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float y = (x.v[e] - mu) * rs;
                if (p.w) y *= w.v[e];
                if (p.b) y += b.v[e];
                x.v[e] = y;
            }
            x.store(p.Y, i * p.ldy + j, count);
        }
    }
}

struct NormGradView {
    const void *dY, *X, *w, *res;
    void* dX;
    int64_t ldg, ldx, ldr, ldd, m, n;
    const float *mean, *rstd;
    float *pw, *pb;  // partial sums, a row for each block
};

template <int DT, int G, int IT>
__global__ __launch_bounds__(kThreads<G>) void k_norm_grad(NormGradView p)
{
    constexpr int kGroups = kThreads<G> / G;
    constexpr int kCols = G * IT * 8;
    __shared__ float red[G > 64 ? 2 * (G / 64) : 1];
    __shared__ float join[kGroups > 1 ? kGroups : 1][kGroups > 1 ? kCols : 1];
    const int lane = threadIdx.x % G, group = threadIdx.x / G;
    RawEight<DT> w[IT];
    float sw[IT][8], sb[IT][8];
    int count[IT];
#pragma unroll
    for (int t = 0; t < IT; ++t) {
        const int64_t j = ((int64_t)t * G + lane) * 8;
        count[t] = eight_of(p.n, j);
#pragma unroll
        for (int e = 0; e < 8; ++e) sw[t][e] = sb[t][e] = 0.0f;
        w[t].ones();
        if (p.w) w[t].load(p.w, j, count[t]);
    }
    const float over = 1.0f / (float)p.n;
    const int64_t turn = (int64_t)gridDim.x * kGroups;
    // The next row is under way while this one is summed (16 bits, where a
    // row takes few registers; 32-bit rows reach the memory's rate without,
    // and 1024 threads with two pieces each have no registers for it).
    constexpr bool kAhead = DT != SVM_F32 && !(G > 256 && IT > 1);
    RawEight<DT> nx[IT], ng[IT], nr[IT];
    auto fetch = [&](int64_t i) {
#pragma unroll
        for (int t = 0; t < IT; ++t) {
            const int64_t j = ((int64_t)t * G + lane) * 8;
            nx[t].load(p.X, i * p.ldx + j, count[t]);
            ng[t].load(p.dY, i * p.ldg + j, count[t]);
            if (p.res) nr[t].load(p.res, i * p.ldr + j, count[t]);
        }
    };
    int64_t i = (int64_t)blockIdx.x * kGroups + group;
    if (kAhead && i < p.m) fetch(i);
    for (; i < p.m; i += turn) {
        if (!kAhead) fetch(i);
        RawEight<DT> r[IT];
        float xh[IT][8], g[IT][8];
        const float mu = p.mean[i], rs = p.rstd[i];
        float s1 = 0.0f, s2 = 0.0f;
        // (past the row's end X is 0, but (0 - mean) rstd may overflow)
#pragma unroll
        for (int t = 0; t < IT; ++t) {
            r[t] = nr[t];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                xh[t][e] = e < count[t] ? (nx[t].at(e) - mu) * rs : 0.0f;
                g[t][e] = ng[t].at(e);
            }
        }
        if (kAhead && i + turn < p.m) fetch(i + turn);
#pragma unroll
        for (int t = 0; t < IT; ++t)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                sw[t][e] = fmaf(g[t][e], xh[t][e], sw[t][e]);
                sb[t][e] += g[t][e];
                g[t][e] *= w[t].at(e);
                s1 += g[t][e];
                s2 = fmaf(g[t][e], xh[t][e], s2);
            }
        if (!p.dX) continue;
        group_sums<G>(s1, s2, red);
        s1 *= over;
        s2 *= over;
#pragma unroll
        for (int t = 0; t < IT; ++t) {
            Eight<DT> d;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                d.v[e] = rs * (g[t][e] - fmaf(xh[t][e], s2, s1));
                if (p.res) d.v[e] += r[t].at(e);
            }
            d.store(p.dX, i * p.ldd + ((int64_t)t * G + lane) * 8, count[t]);
        }
    }
    if (!p.pw) return;
    // the block's row of the partial sums
#pragma unroll
    for (int both = 0; both < 2; ++both) {
        float* out = (both ? p.pb : p.pw) + (int64_t)blockIdx.x * p.n;
        if constexpr (kGroups > 1) {
            __syncthreads();
#pragma unroll
            for (int t = 0; t < IT; ++t)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    join[group][(t * G + lane) * 8 + e] =
                        both ? sb[t][e] : sw[t][e];
            __syncthreads();
            for (int j = threadIdx.x; j < kCols && j < p.n;
                 j += kThreads<G>) {
                float s = 0.0f;
#pragma unroll
                for (int r = 0; r < kGroups; ++r) s += join[r][j];
                out[j] = s;
            }
        } else {
#pragma unroll
            for (int t = 0; t < IT; ++t) {
                Eight<SVM_F32> s;
#pragma unroll
                for (int e = 0; e < 8; ++e) s.v[e] = both ? sb[t][e] : sw[t][e];
                s.store(out, ((int64_t)t * G + lane) * 8, count[t]);
            }
        }
    }
}

// Wide rows: dX with the row read twice.
template <int DT>
__global__ __launch_bounds__(1024) void k_norm_grad_wide(NormGradView p)
{
    constexpr int G = 1024;
    __shared__ float red[2 * (G / 64)];
    const float over = 1.0f / (float)p.n;
    for (int64_t i = blockIdx.x; i < p.m; i += gridDim.x) {
        const float mu = p.mean[i], rs = p.rstd[i];
        float s1 = 0.0f, s2 = 0.0f;
        Eight<DT> g, x, w, r;
        for (int64_t j = threadIdx.x * 8; j < p.n; j += G * 8) {
            const int count = eight_of(p.n, j);
            g.load(p.dY, i * p.ldg + j, count);
            x.load(p.X, i * p.ldx + j, count);
            if (p.w) w.load(p.w, j, count);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < count) {
                    const float a = g.v[e] * (p.w ? w.v[e] : 1.0f);
                    s1 += a;
                    s2 = fmaf(a, (x.v[e] - mu) * rs, s2);
                }
        }
        group_sums<G>(s1, s2, red);
        s1 *= over;
        s2 *= over;
        for (int64_t j = threadIdx.x * 8; j < p.n; j += G * 8) {
            const int count = eight_of(p.n, j);
            g.load(p.dY, i * p.ldg + j, count);
            x.load(p.X, i * p.ldx + j, count);
            if (p.w) w.load(p.w, j, count);
            if (p.res) r.load(p.res, i * p.ldr + j, count);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float a = g.v[e] * (p.w ? w.v[e] : 1.0f);
                float d = rs * (a - fmaf((x.v[e] - mu) * rs, s2, s1));
                if (p.res) d += r.v[e];
                x.v[e] = d;
            }
            x.store(p.dX, i * p.ldd + j, count);
        }
    }
}

// ... and the sums over a block's rows, a thread to a column.
template <int DT>
__global__ __launch_bounds__(256) void k_norm_sums(NormGradView p, int64_t per)
{
    using T = Elem<DT>;
    const int64_t j = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (j >= p.n) return;
    const int64_t i0 = blockIdx.y * per;
    const int64_t i1 = i0 + per < p.m ? i0 + per : p.m;
    float sw = 0.0f, sb = 0.0f;
#pragma unroll 4
    for (int64_t i = i0; i < i1; ++i) {
        const float g = (float)((const T*)p.dY)[i * p.ldg + j];
        sb += g;
        sw = fmaf(g, ((float)((const T*)p.X)[i * p.ldx + j] - p.mean[i]) *
                         p.rstd[i],
                  sw);
    }
    p.pw[blockIdx.y * p.n + j] = sw;
    p.pb[blockIdx.y * p.n + j] = sb;
}

// Calls f with the lanes and pieces of a row of n columns.
template <class F>
void for_width(int64_t n, F&& f)
{
    if (n <= 128) f.template operator()<16, 1>();
    else if (n <= 256) f.template operator()<32, 1>();
    else if (n <= 512) f.template operator()<64, 1>();
    else if (n <= 1024) f.template operator()<64, 2>();
    else if (n <= 2048) f.template operator()<256, 1>();
    else if (n <= 4096) f.template operator()<256, 2>();
    else if (n <= 8192) f.template operator()<1024, 1>();
    else f.template operator()<1024, 2>();
}

// Blocks of the gradient: those that the registers of the kernel let run at
// once (a block more would run alone at the end), but no more than there are
// turns of `groups` rows.
template <int G, int IT>
int64_t grad_blocks(int64_t m)
{
    const int64_t groups = kThreads<G> / G;
    const int64_t turns = (m + groups - 1) / groups;
    const int64_t most = 256 * (G > 256 ? 1 : IT > 1 ? 3 : 4);
    return turns < most ? turns : most;
}

int64_t norm_partials(int64_t m, int64_t n)
{
    if (m == 0) return 0;
    if (n > kMostCols) return (m + 255) / 256 < 1024 ? (m + 255) / 256 : 1024;
    int64_t np = 0;
    for_width(n, [&]<int G, int IT>() {
        np = grad_blocks<G, IT>(m);
    });
    return np;
}

}  // namespace

void norm_forward(const NormArgs& a, hipStream_t s)
{
    NormView v{a.X.data, a.weight.data, a.bias.data, a.Y.data,
               a.X.ld,   a.Y.ld,        a.X.rows,    a.X.cols,
               a.mean,   a.rstd,        a.eps};
    for_dtype(a.X.dtype, [&]<int DT>() {
        if (v.n > kMostCols) {
            hipLaunchKernelGGL((k_norm_wide<DT>),
                               dim3((unsigned)(v.m < 2048 ? v.m : 2048)),
                               dim3(1024), 0, s, v);
            return;
        }
        for_width(v.n, [&]<int G, int IT>() {
            constexpr int kGroups = kThreads<G> / G;
            const int64_t nb = (v.m + kGroups - 1) / kGroups;
            const int64_t most = 256 * 8 * 256 / kThreads<G>;
            hipLaunchKernelGGL((k_norm<DT, G, IT>),
                               dim3((unsigned)(nb < most ? nb : most)),
                               dim3(kThreads<G>), 0, s, v);
        });
    });
}

int64_t norm_backward_bytes(int64_t rows, int64_t cols)
{
    Pieces p;
    p.take<float>(norm_partials(rows, cols) * cols);
    p.take<float>(norm_partials(rows, cols) * cols);
    return p.used;
}

void norm_backward(const NormGradArgs& a, Pieces& ws, hipStream_t s)
{
    const int64_t m = a.X.rows, n = a.X.cols, np = norm_partials(m, n);
    const bool sums = a.dweight.data || a.dbias.data;
    NormGradView v{a.dY.data, a.X.data, a.weight.data, a.residual.data,
                   a.dX.data, a.dY.ld,  a.X.ld,        a.residual.ld,
                   a.dX.ld,   m,        n,             a.mean,
                   a.rstd,    nullptr,  nullptr};
    if (sums) {
        v.pw = ws.take<float>(np * n);
        v.pb = ws.take<float>(np * n);
    }
    if (m > 0 && (sums || v.dX))
        for_dtype(a.X.dtype, [&]<int DT>() {
            if (n > kMostCols) {
                if (sums)
                    hipLaunchKernelGGL(
                        (k_norm_sums<DT>),
                        dim3((unsigned)((n + 255) / 256), (unsigned)np),
                        dim3(256), 0, s, v, (m + np - 1) / np);
                if (v.dX)
                    hipLaunchKernelGGL((k_norm_grad_wide<DT>),
                                       dim3((unsigned)(m < 2048 ? m : 2048)),
                                       dim3(1024), 0, s, v);
                return;
            }
            for_width(n, [&]<int G, int IT>() {
                hipLaunchKernelGGL((k_norm_grad<DT, G, IT>),
                                   dim3((unsigned)np), dim3(kThreads<G>), 0, s,
                                   v);
            });
        });
    if (sums)
        launch_column_sums(v.pw, v.pb, np, n, a.X.dtype, a.dweight.data,
                           a.dbias.data, s);
}

}  // namespace msvm
