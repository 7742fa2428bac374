// Gradients of group norm with an activation (groupnorm.hpp says how they are
// cut up).  One sweep over a slab for the sums by groups and by columns; the
// slab and what the activation's slope made of dY stay in registers for dX.
// Bound by memory and the vector instructions (46 a value, 30 of 60 us), with
// two waves to a SIMD to overlap them: the kernel takes all 256 registers, 12
// for each of 8 pieces.  256 x 196 x 512 in bf16
// with silu and a residual 60 us, 3.4 TB/s (a large copy: 5.0).  Cut into
// chunks, where dX is a pass of its own: 6 x 3977 x 231 in f16 37 us, 17 for
// the sums, 14 for dX, 5 for each of the two launches that join sums.
#include "groupnorm.hpp"

namespace msvm {

namespace {

constexpr int kGradBlocks = 2048;  // that keep sums for weight and bias

// The slope of the activation at z = xh w + b, xh = (x - mu) rs.  For relu it
// is a matter of z's sign: where 32 bits' rounding may have turned that, 64
// bits settle it (the slope would be off by all of itself).
template <int DT, bool EVEN>
__device__ __forceinline__ void slopes(
    int act, const RawEight<DT>& x, const float (&mu)[Place<EVEN>::kK],
    const float (&rs)[Place<EVEN>::kK], const float (&xh)[8],
    const float (&w)[8], const float (&b)[8], float (&s)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = fmaf(xh[e], w[e], b[e]);
    if (act == SVM_ACT_RELU) {
        bool near = false;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            near |= fabsf(s[e]) <=
                    1e-6f * (fabsf(xh[e] * w[e]) + fabsf(b[e]));
        if (near) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                // (none of this is to be made ahead of the branch)
                float m = mu[EVEN ? 0 : e], r = rs[EVEN ? 0 : e];
                float wv = w[e], bv = b[e];
                asm volatile("" : "+v"(m), "+v"(r), "+v"(wv), "+v"(bv));
                const double z = fma(((double)x.at(e) - (double)m) * (double)r,
                                     (double)wv, (double)bv);
                s[e] = z > 0.0 ? 1.0f : z < 0.0 ? -1.0f : (float)z;
            }
        }
    }
    if (act == SVM_ACT_NONE) {
#pragma unroll
        for (int e = 0; e < 8; ++e) s[e] = 1.0f;
    } else {
        act_slopes(act, s);
    }
}

template <bool EVEN>
__device__ __forceinline__ void load_stats(const GroupArgs& a,
                                           const Place<EVEN>& at, int64_t n,
                                           float (&mu)[Place<EVEN>::kK],
                                           float (&rs)[Place<EVEN>::kK])
{
#pragma unroll
    for (int k = 0; k < Place<EVEN>::kK; ++k) {
        const int64_t g = n * a.groups + at.g0 + at.group[k];
        mu[k] = a.mean[g];
        rs[k] = a.rstd[g];
    }
}

// PARTS: only the sums, by chunks and for weight and bias.  A block keeps to
// one slice and adds up in registers what its columns get over its units.
// (Waves to a SIMD at the least: some are a register or two past the next.)
template <int IT, bool EVEN>
constexpr int kWavesAtLeast = IT > 2 ? 2 : IT > 1 ? (EVEN ? 3 : 2)
                                                  : (EVEN ? 4 : 3);

template <int DT, int T, int IT, bool EVEN, bool PARTS>
__global__ __launch_bounds__(kSlabThreads<T>, (kWavesAtLeast<IT, EVEN>))
void k_group_grad(GroupArgs a)
{
    constexpr int kK = Place<EVEN>::kK;
    __shared__ float bufs[kSlabs<T>][2 * 8 * T];
    __shared__ float stats[kSlabs<T>][2 * kStat<T>];
    const Plan& p = a.p;
    const int slab = threadIdx.x / T, t = threadIdx.x % T;
    float *buf = bufs[slab], *stat = stats[slab];
    const int64_t slice = blockIdx.x % (unsigned)p.slices;
    const int64_t nb = gridDim.x / (unsigned)p.slices;
    const Place<EVEN> at(a, slice, t);
    const int64_t units = a.samples * p.chunks;
    Eights<DT> w8, b8;
    w8.load(a.w, at.first(), at.count, 1.0f);
    b8.load(a.b, at.first(), at.count, 0.0f);
    float sb[8] = {}, sw[8] = {};  // over the block's units
    const float over = 1.0f / (float)(a.positions * p.each);
    for (int64_t j0 = blockIdx.x / (unsigned)p.slices * kSlabs<T>; j0 < units;
         j0 += nb * kSlabs<T>) {
        const Unit u(a, j0 + slab);
        RawEight<DT> x[IT], g[IT];
        const bool any = u.rows > 0 && at.count > 0;
        const int64_t last = u.row + u.rows - 1;
        load_slab<DT, IT>(x, a.X, (u.row + at.row) * a.ldx + at.first(),
                          p.rows * a.ldx, last * a.ldx + at.first(), any,
                          at.count, a.endx);
        load_slab<DT, IT>(g, a.dY, (u.row + at.row) * a.ldg + at.first(),
                          p.rows * a.ldg, last * a.ldg + at.first(), any,
                          at.count, a.endg);
        // (a slab without a unit: statistics of 0, so that its xh are 0 and add
        // nothing; with any sample's they may be infinite, and 0 times them NaN)
        float mu[kK], rs[kK];
        load_stats<EVEN>(a, at, u.n < a.samples ? u.n : a.samples - 1, mu, rs);
        if (kSlabs<T> > 1 && u.rows == 0) {
#pragma unroll
            for (int k = 0; k < kK; ++k) mu[k] = rs[k] = 0.0f;
        }
        float w[8], b[8];
        w8.values(w);
        b8.values(b);
        // by group: the sums of a = dZ w and of a xh
        float dz[IT][8], v[2][kK] = {};
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            if (i > 0 && i * p.rows >= u.rows) break;
            // (a piece past the end is another's again, and adds nothing)
            const bool there = at.row + i * p.rows < u.rows;
            forget(x[i]);
            forget(g[i]);
            float xh[8], s[8];
#pragma unroll
            for (int e = 0; e < 8; ++e)
                xh[e] = (x[i].at(e) - mu[EVEN ? 0 : e]) * rs[EVEN ? 0 : e];
            slopes<DT, EVEN>(a.act, x[i], mu, rs, xh, w, b, s);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = there ? g[i].at(e) * s[e] : 0.0f;
                const float q = d * w[e];
                dz[i][e] = d;
                sb[e] += d;
                sw[e] = fmaf(d, xh[e], sw[e]);
                v[0][EVEN ? 0 : e] += q;
                v[1][EVEN ? 0 : e] = fmaf(q, xh[e], v[1][EVEN ? 0 : e]);
            }
            settle(sb);
            settle(sw);
            settle(v[0]);
            settle(v[1]);
        }
        if (!PARTS && !a.out) continue;
        group_sums<T, 2, EVEN>(p, at, t, v, buf,
                               [&](int q, const float (&s)[2]) {
                                   stat[q] = PARTS ? s[0] : s[0] * over;
                                   stat[kStat<T> + q] =
                                       PARTS ? s[1] : s[1] * over;
                               });
        if (PARTS) {
            if (u.rows > 0)
                for (int q = t; q < at.ng; q += T) {
                    const int64_t ng = u.n * a.groups + at.g0 + q;
                    const int64_t cp =
                        p.parts_across > 1 ? slice % p.parts_across : 0;
                    a.part[ng * p.parts() + cp * p.chunks + u.ch] =
                        make_float2(stat[q], stat[kStat<T> + q]);
                }
            continue;
        }
        float s1[kK], s2[kK];
#pragma unroll
        for (int k = 0; k < kK; ++k) {
            s1[k] = stat[at.group[k]];
            s2[k] = stat[kStat<T> + at.group[k]];
        }
        int64_t to = here((u.row + at.row) * a.ldo + at.first());
        constexpr int kAhead = IT < 4 ? IT : 4;
        RawEight<DT> res[kAhead];
#pragma unroll
        for (int i = 0; i < IT; ++i, to += p.rows * a.ldo) {
            const int r = at.row + i * p.rows;
            if (a.res && i % kAhead == 0)
                load_slab<DT, kAhead>(
                    res, a.res, (u.row + r) * a.ldr + at.first(),
                    p.rows * a.ldr, last * a.ldr + at.first(), any, at.count,
                    a.endr);
            if (r >= u.rows || at.count == 0) continue;
            forget(x[i]);
            Eight<DT> d;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int k = EVEN ? 0 : e;
                const float xh = (x[i].at(e) - mu[k]) * rs[k];
                d.v[e] = rs[k] * (dz[i][e] * w[e] - fmaf(xh, s2[k], s1[k]));
            }
            if (a.res) {
#pragma unroll
                for (int e = 0; e < 8; ++e) d.v[e] += res[i % kAhead].at(e);
            }
            store_some<DT, EVEN>(d, a.out, to, at.count);
        }
    }
    if (!a.pw) return;
    // the block's row of the partial sums: over positions and slabs
    const int wide = p.lanes * 8;
    __syncthreads();
    if (at.row < p.rows) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            buf[at.row * wide + at.lane * 8 + e] = sb[e];
            buf[8 * T + at.row * wide + at.lane * 8 + e] = sw[e];
        }
    }
    __syncthreads();
    const int64_t to = blockIdx.x / (unsigned)p.slices * (a.groups * p.each) + at.col;
    for (int c = threadIdx.x; c < 2 * at.cols; c += kSlabThreads<T>) {
        const int q = c >= at.cols, d = c - q * at.cols;
        float sum = 0.0f;
        for (int i = 0; i < kSlabs<T>; ++i)
#pragma unroll 4
            for (int r = 0; r < p.rows; ++r)
                sum += bufs[i][q * 8 * T + r * wide + d];
        (q ? a.pw : a.pb)[to + d] = sum;
    }
}

constexpr int kAhead = 4;

// dX from joined sums.  A thread to 8 columns, positions in turn.
template <int DT, bool EVEN>
__global__ __launch_bounds__(256) void k_group_dx(GroupArgs a)
{
    constexpr int kK = Place<EVEN>::kK;
    const Plan& p = a.p;
    const int64_t slice = blockIdx.x % (unsigned)p.slices;
    const int64_t nb = gridDim.x / (unsigned)p.slices;
    const int64_t units = a.samples * p.chunks;
    const float over = 1.0f / (float)(a.positions * p.each);
    for_lanes<EVEN>(a, slice, [&](const Place<EVEN>& at, int row, int step,
                                  int count) {
        const int64_t c = at.first();
        Eights<DT> w8, b8;
        w8.load(a.w, c, count, 1.0f);
        b8.load(a.b, c, count, 0.0f);
        for (int64_t j = blockIdx.x / (unsigned)p.slices; j < units; j += nb) {
            const Unit u(a, j);
            float mu[kK], rs[kK], s1[kK], s2[kK];
            load_stats<EVEN>(a, at, u.n, mu, rs);
#pragma unroll
            for (int k = 0; k < kK; ++k) {
                const float2 s =
                    a.sums[u.n * a.groups + at.g0 + at.group[k]];
                s1[k] = s.x * over;
                s2[k] = s.y * over;
            }
            for (int r0 = row; r0 < u.rows; r0 += step * kAhead) {
                RawEight<DT> x[kAhead], g[kAhead], res[kAhead];
                const int64_t at0 = u.row + r0, last = u.row + u.rows - 1;
                load_slab<DT, kAhead>(x, a.X, at0 * a.ldx + c, step * a.ldx,
                                      last * a.ldx + c, true, count, a.endx);
                load_slab<DT, kAhead>(g, a.dY, at0 * a.ldg + c, step * a.ldg,
                                      last * a.ldg + c, true, count, a.endg);
                if (a.res)
                    load_slab<DT, kAhead>(res, a.res, at0 * a.ldr + c,
                                          step * a.ldr, last * a.ldr + c,
                                          true, count, a.endr);
                float w[8], b[8];
                w8.values(w);
                b8.values(b);
#pragma unroll
                for (int i = 0; i < kAhead; ++i) {
                    const int r = r0 + i * step;
                    if (r >= u.rows) continue;
                    forget(x[i]);
                    forget(g[i]);
                    Eight<DT> d;
                    float xh[8], s[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        xh[e] = (x[i].at(e) - mu[EVEN ? 0 : e]) *
                                rs[EVEN ? 0 : e];
                    slopes<DT, EVEN>(a.act, x[i], mu, rs, xh, w, b, s);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int k = EVEN ? 0 : e;
                        d.v[e] = rs[k] * (g[i].at(e) * s[e] * w[e] -
                                          fmaf(xh[e], s2[k], s1[k]));
                    }
                    if (a.res) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) d.v[e] += res[i].at(e);
                    }
                    store_some<DT, EVEN>(d, a.out,
                                         (u.row + r) * a.ldo + c, count);
                }
            }
        }
    });
}

}  // namespace

void group_norm_backward(const GroupGradCall& c, Pieces& ws, hipStream_t s)
{
    const int64_t samples = c.X.rows / c.positions, n = c.X.cols;
    GroupArgs a{};
    a.X = c.X.data;
    a.dY = c.dY.data;
    a.res = c.residual.data;
    a.w = c.weight.data;
    a.b = c.bias.data;
    a.out = c.dX.data;
    a.ldx = c.X.ld;
    a.ldg = c.dY.ld;
    a.ldr = c.residual.ld;
    a.ldo = c.dX.ld;
    a.endx = end_of(c.X);
    a.endg = end_of(c.dY);
    a.endr = end_of(c.residual);
    a.samples = samples;
    a.positions = c.positions;
    a.groups = c.groups;
    a.act = c.act;
    a.mean = const_cast<float*>(c.mean);
    a.rstd = const_cast<float*>(c.rstd);
    a.p = plan_of(samples, c.positions, n, c.groups, c.X.dtype, true);
    const Plan& p = a.p;
    const int64_t rows = samples ? blocks_across(a, kGradBlocks) : 0;
    const int64_t all = samples * c.groups;
    if (c.sums) {
        a.pw = ws.take<float>(rows * n);
        a.pb = ws.take<float>(rows * n);
    }
    float2* joined = nullptr;
    if (p.split()) {
        a.part = ws.take<float2>(all * p.parts());
        joined = ws.take<float2>(all);
        a.sums = joined;
    }
    if (!ws.run) return;
    if (samples > 0 && (c.sums || a.out))
        for_dtype(c.X.dtype, [&]<int DT>() {
            const dim3 grid((unsigned)(rows * p.slices));
            for_plan<DT, true>(p, [&]<int T, int IT, bool EVEN>() {
                if (!p.split()) {
                    hipLaunchKernelGGL((k_group_grad<DT, T, IT, EVEN, false>),
                                       grid, dim3(kSlabThreads<T>), 0, s, a);
                    return;
                }
                if constexpr (T >= 256)
                    hipLaunchKernelGGL((k_group_grad<DT, T, IT, EVEN, true>),
                                       grid, dim3(kSlabThreads<T>), 0, s, a);
            });
            if (!p.split() || !a.out) return;
            launch_join<true>(a, joined, s);
            GroupArgs b = a;
            b.p = apply_plan(a, kAhead);
            const dim3 turns((unsigned)(blocks_across(b, 1 << 20) * p.slices));
            if (p.even)
                hipLaunchKernelGGL((k_group_dx<DT, true>), turns, dim3(256), 0,
                                   s, b);
            else
                hipLaunchKernelGGL((k_group_dx<DT, false>), turns, dim3(256),
                                   0, s, b);
        });
    if (c.sums)
        launch_column_sums(a.pw, a.pb, rows, n, c.X.dtype, c.dweight.data,
                           c.dbias.data, s);
}

}  // namespace msvm
