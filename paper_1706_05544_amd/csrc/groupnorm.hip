// Group norm with an activation: the forward pass (groupnorm.hpp says how it
// is cut up).  Bound by memory and, nearly as much, by the vector instructions
// (28 a value): 512 x 196 x 512 in bf16 with silu 47 us, 4.4 TB/s (a
// large copy: 5.0); 100000 x 64 in 32 bits, eight threads a sample, 15.4 us,
// 3.3 TB/s.  Groups of a width that is no multiple of 8 take more of them:
// 4000 x 30 x 120 in f16, groups of 15, 31 us, 1.9 TB/s.  Mean and deviations
// are two sums over registers, never a difference of squares.
#include "groupnorm.hpp"

namespace msvm {

namespace {

// Whether the mean is corrected.  The sum of a group's values is rounded at
// their own level, by some units of its last place, and what that makes the
// mean off by is the mean of the deviations from it: their sum, beside that of
// their squares, gives the mean to one rounding and takes the error out of
// the squares (equal values come out as exact zeros).  Values of 16 bits need
// none: the error is far under their own steps.  256 x 196 x 512 in 32 bits
// 37.3 us, without 37.1; 100000 x 64 15.4 and 14.9; for every type 512 x 196 x
// 512 in bf16 would take 41.5 for 40.0, 4000 x 30 x 120 in f16 34.0 for 30.7.
template <int DT>
constexpr bool kCorrect = DT == SVM_F32;

__device__ __forceinline__ bool is_finite(float v)
{
    return fabsf(v) <= 3.402823466e38f;
}

// The sum of squared deviations from a mean, less what that mean is off by:
// `sum` of the deviations, `off` their mean.  (Not finite: as it is.)
__device__ __forceinline__ float squares_about(float squares, float sum,
                                               float off)
{
    const float q = fmaf(-sum, off, squares);
    return q > 0.0f ? q : q <= 0.0f ? 0.0f : squares;
}

// PARTS: only the chunks' means and squared deviations, else the whole of a
// sample.
template <int DT, int T, int IT, bool EVEN, bool PARTS>
__global__ __launch_bounds__(kSlabThreads<T>) void k_group_norm(GroupArgs a)
{
    constexpr int kK = Place<EVEN>::kK;
    constexpr int kBuf = EVEN ? T : 8 * T;
    constexpr int kQ = kCorrect<DT> ? 2 : 1;
    __shared__ float bufs[kSlabs<T>][2 * kBuf];
    __shared__ float stats[kSlabs<T>][2 * kStat<T>];
    const Plan& p = a.p;
    const int slab = threadIdx.x / T, t = threadIdx.x % T;
    float *buf = bufs[slab], *stat = stats[slab];
    const int64_t slice = blockIdx.x % (unsigned)p.slices;
    const int64_t nb = gridDim.x / (unsigned)p.slices;
    const Place<EVEN> at(a, slice, t);
    const int64_t units = a.samples * p.chunks;
    Eights<DT> w8, b8;
    if (!PARTS) {
        w8.load(a.w, at.first(), at.count, 1.0f);
        b8.load(a.b, at.first(), at.count, 0.0f);
    }
    for (int64_t j0 = blockIdx.x / (unsigned)p.slices * kSlabs<T>; j0 < units;
         j0 += nb * kSlabs<T>) {
        const Unit u(a, j0 + slab);
        RawEight<DT> x[IT];
        load_slab<DT, IT>(x, a.X, (u.row + at.row) * a.ldx + at.first(),
                          p.rows * a.ldx,
                          (u.row + u.rows - 1) * a.ldx + at.first(),
                          u.rows > 0 && at.count > 0, at.count, a.endx);
        float v[1][kK] = {};
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            // (a piece past the end is another's again, and adds nothing)
            if (at.row + i * p.rows >= u.rows) continue;
#pragma unroll
            for (int e = 0; e < 8; ++e) v[0][EVEN ? 0 : e] += x[i].at(e);
            settle(v[0]);
        }
        const float size = (float)((int64_t)u.rows * at.each(p));
        group_sums<T, 1, EVEN>(p, at, t, v, buf,
                               [&](int g, const float (&s)[1]) {
                                   stat[g] = s[0] / size;
                               });
        float mu[kK], d[kQ][kK];
#pragma unroll
        for (int k = 0; k < kK; ++k) {
            mu[k] = stat[at.group[k]];
            d[0][k] = d[kQ - 1][k] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            if (at.row + i * p.rows >= u.rows) continue;
            forget(x[i]);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int k = EVEN ? 0 : e;
                const float o = x[i].at(e) - mu[k];
                if (kQ == 2) d[0][k] += o;
                d[kQ - 1][k] = fmaf(o, o, d[kQ - 1][k]);
            }
            settle(d[0]);
            settle(d[kQ - 1]);
        }
        group_sums<T, kQ, EVEN>(
            p, at, t, d, buf, [&](int g, const float (&s)[kQ]) {
                float off = 0.0f, q = s[kQ - 1];
                if (kQ == 2) {
                    off = s[0] / size;
                    q = squares_about(q, s[0], off);
                    if (!is_finite(off)) off = 0.0f;
                }
                if (PARTS) {
                    const int64_t ng = u.n * a.groups + at.g0 + g;
                    const int64_t cp =
                        p.parts_across > 1 ? slice % p.parts_across : 0;
                    a.moments[ng * p.parts() + cp * p.chunks + u.ch] =
                        make_double2((double)stat[g] + (double)off, q);
                } else {
                    if (kQ == 2) stat[g] += off;
                    stat[kStat<T> + g] = 1.0f / sqrtf(q / size + a.eps);
                }
            });
        if (PARTS) continue;
        if (u.rows > 0)
            for (int g = t; g < at.ng; g += T) {
                const int64_t ng = u.n * a.groups + at.g0 + g;
                if (a.mean) a.mean[ng] = stat[g];
                if (a.rstd) a.rstd[ng] = stat[kStat<T> + g];
            }
        float rs[kK];
#pragma unroll
        for (int k = 0; k < kK; ++k) {
            if (kQ == 2) mu[k] = stat[at.group[k]];
            rs[k] = stat[kStat<T> + at.group[k]];
        }
        float w[8], b[8];
        w8.values(w);
        b8.values(b);
        int64_t to = here((u.row + at.row) * a.ldo + at.first());
#pragma unroll
        for (int i = 0; i < IT; ++i, to += p.rows * a.ldo) {
            if (at.row + i * p.rows >= u.rows || at.count == 0) continue;
            forget(x[i]);
            Eight<DT> y;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int k = EVEN ? 0 : e;
                y.v[e] = fmaf((x[i].at(e) - mu[k]) * rs[k], w[e], b[e]);
            }
            act_values(a.act, y.v);
            store_some<DT, EVEN>(y, a.out, to, at.count);
        }
    }
}

constexpr int kAhead = 4;

// Applies joined statistics.  A thread to 8 columns, positions in turn.
template <int DT, bool EVEN>
__global__ __launch_bounds__(256) void k_group_apply(GroupArgs a)
{
    constexpr int kK = Place<EVEN>::kK;
    const Plan& p = a.p;
    const int64_t slice = blockIdx.x % (unsigned)p.slices;
    const int64_t nb = gridDim.x / (unsigned)p.slices;
    const int64_t units = a.samples * p.chunks;
    for_lanes<EVEN>(a, slice, [&](const Place<EVEN>& at, int row, int step,
                                  int count) {
        const int64_t c = at.first();
        Eights<DT> w8, b8;
        w8.load(a.w, c, count, 1.0f);
        b8.load(a.b, c, count, 0.0f);
        for (int64_t j = blockIdx.x / (unsigned)p.slices; j < units; j += nb) {
            const Unit u(a, j);
            float mu[kK], rs[kK];
#pragma unroll
            for (int k = 0; k < kK; ++k) {
                const int64_t g = u.n * a.groups + at.g0 + at.group[k];
                mu[k] = a.mean[g];
                rs[k] = a.rstd[g];
            }
            for (int r0 = row; r0 < u.rows; r0 += step * kAhead) {
                RawEight<DT> x[kAhead];
                load_slab<DT, kAhead>(x, a.X, (u.row + r0) * a.ldx + c,
                                      step * a.ldx,
                                      (u.row + u.rows - 1) * a.ldx + c, true,
                                      count, a.endx);
                float w[8], b[8];
                w8.values(w);
                b8.values(b);
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const int r = r0 + i * step;
                    if (r >= u.rows) continue;
                    forget(x[i]);
                    Eight<DT> y;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int k = EVEN ? 0 : e;
                        y.v[e] = fmaf((x[i].at(e) - mu[k]) * rs[k], w[e],
                                      b[e]);
                    }
                    act_values(a.act, y.v);
                    store_some<DT, EVEN>(y, a.out,
                                         (u.row + r) * a.ldo + c, count);
                }
            }
        }
    });
}

}  // namespace

void group_norm(const GroupCall& c, Pieces& ws, hipStream_t s)
{
    const int64_t samples = c.X.rows / c.positions;
    GroupArgs a{};
    a.X = c.X.data;
    a.w = c.weight.data;
    a.b = c.bias.data;
    a.out = c.Y.data;
    a.ldx = c.X.ld;
    a.endx = end_of(c.X);
    a.ldo = c.Y.ld;
    a.samples = samples;
    a.positions = c.positions;
    a.groups = c.groups;
    a.eps = c.eps;
    a.act = c.act;
    a.mean = c.mean;
    a.rstd = c.rstd;
    a.p = plan_of(samples, c.positions, c.X.cols, c.groups, c.X.dtype, false);
    const Plan& p = a.p;
    const int64_t all = samples * c.groups;
    if (p.split()) {
        a.moments = ws.take<double2>(all * p.parts());
        float* mean = ws.take<float>(all);
        float* rstd = ws.take<float>(all);
        if (!a.mean) a.mean = mean;
        if (!a.rstd) a.rstd = rstd;
    }
    if (!ws.run || samples == 0) return;
    for_dtype(c.X.dtype, [&]<int DT>() {
        const dim3 grid((unsigned)(blocks_across(a, 1 << 20) * p.slices));
        for_plan<DT, false>(p, [&]<int T, int IT, bool EVEN>() {
            if (!p.split()) {
                hipLaunchKernelGGL((k_group_norm<DT, T, IT, EVEN, false>),
                                   grid, dim3(kSlabThreads<T>), 0, s, a);
                return;
            }
            if constexpr (T >= 256 && IT <= 8) {
                hipLaunchKernelGGL((k_group_norm<DT, T, IT, EVEN, true>),
                                   grid, dim3(kSlabThreads<T>), 0, s, a);
            }
        });
        if (!p.split()) return;
        launch_join<false>(a, nullptr, s);
        GroupArgs b = a;
        b.p = apply_plan(a, kAhead);
        const dim3 turns((unsigned)(blocks_across(b, 1 << 20) * p.slices));
        if (p.even)
            hipLaunchKernelGGL((k_group_apply<DT, true>), turns, dim3(256), 0,
                               s, b);
        else
            hipLaunchKernelGGL((k_group_apply<DT, false>), turns, dim3(256), 0,
                               s, b);
    });
}

}  // namespace msvm
