// Group norm with an activation over samples x positions x channels, channels
// last, and its gradients.
//
// A unit of work is a slab: the positions of one sample (or a chunk of them)
// by a slice of columns, whole groups side by side, wide enough to fill the
// memory's lines (groups of more than kWideCols channels are cut into slices
// of their own).  T threads hold a slab in registers, each 8 columns of every
// R-th position, from its read to its write: sums over positions go through
// LDS once for all columns and are then added up by groups, whatever a
// group's width.  Where a sample's slab is too large, or slabs are too few to
// fill the card, the positions are cut into chunks: one launch for the chunks'
// statistics, one that joins them, and one that applies them and reads the
// values again.  The gradient takes one sweep for the sums by columns, from
// which both the groups' sums and those for weight and bias come.
#include "elem.hpp"
#include "layers.hpp"

namespace msvm {

namespace {

constexpr int64_t kWideCols = 4096;
constexpr int kGroupUnits = 2048;  // blocks that keep sums for weight and bias

// How a call is cut up.  All by the sizes and the type.
struct Plan {
    int threads, pieces;   // of a slab: T, and IT pieces of 8 for each
    int lanes, rows;       // lanes across the slice; positions at a time
    int64_t each;          // channels of a group
    int64_t groups;        // of a slice (1 where a group has several slices)
    int64_t cols;          // of a slice
    int64_t slices, parts_across;  // of a row; of a group
    int64_t chunk, chunks; // positions of a chunk; chunks of a sample
    __host__ __device__ bool split() const { return chunks > 1 || parts_across > 1; }
    __host__ __device__ int64_t parts() const { return chunks * parts_across; }
};

struct GroupArgs {
    const void *X, *dY, *res, *w, *b;
    void* out;
    int64_t ldx, ldg, ldr, ldo;
    int64_t samples, positions, groups;
    float eps;
    int act;
    float *mean, *rstd;     // written by the forward pass, else read
    float2* part;           // statistics of the chunks
    const float2* sums;     // joined sums of a gradient
    float *pw, *pb;         // rows of partial sums for weight and bias
    Plan p;
};

// What a thread has of the slab of its slice.
struct Place {
    int64_t col, g0;  // first column and group
    int lane, row;    // of the 8-column pieces; first position
    int count;        // columns that there are, of 8
    int cols, ng;     // of this slice
    int group[8];     // of the thread's columns, in the slice

    __device__ __forceinline__ Place(const GroupArgs& a, int64_t slice, int t)
    {
        const Plan& p = a.p;
        lane = t % p.lanes;
        row = t / p.lanes;
        if (p.parts_across > 1) {
            g0 = slice / p.parts_across;
            const int64_t c = (slice - g0 * p.parts_across) * p.cols;
            col = g0 * p.each + c;
            cols = (int)(p.each - c < p.cols ? p.each - c : p.cols);
            ng = 1;
        } else {
            g0 = slice * p.groups;
            col = g0 * p.each;
            const int64_t left = a.groups - g0;
            ng = (int)(left < p.groups ? left : p.groups);
            cols = ng * (int)p.each;
        }
        count = row < p.rows ? eight_of(cols, lane * 8) : 0;
        const bool one = p.parts_across > 1;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int g = one ? 0 : (lane * 8 + e) / (int)p.each;
            group[e] = g < ng ? g : ng - 1;
        }
    }
};

// Adds up the threads' sums of a slab over its positions, a column to a
// thread: col[c], c < cols, of Q quantities.  buf: 8 T floats for each.
template <int T, int Q>
__device__ __forceinline__ void column_sums(const Plan& p, const Place& at,
                                            int t, const float (&v)[Q][8],
                                            float* buf)
{
    const int wide = p.lanes * 8;
    __syncthreads();  // what was there has been read
    if (at.row < p.rows) {
#pragma unroll
        for (int q = 0; q < Q; ++q)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                buf[q * 8 * T + at.row * wide + at.lane * 8 + e] = v[q][e];
    }
    __syncthreads();
    for (int c = t; c < Q * at.cols; c += T) {
        const int q = c >= at.cols;  // (Q is 1 or 2)
        float* s = buf + q * 8 * T + (c - q * at.cols);
        float sum = 0.0f;
#pragma unroll 8
        for (int r = 0; r < p.rows; ++r) sum += s[r * wide];
        s[0] = sum;
    }
    __syncthreads();
}

// Adds up a slab's columns by groups: stat[q][g].  A team of lanes to a group.
// With w the columns count w[c] times.
// Groups of a slice, and columns (the plan keeps to both).
template <int T>
constexpr int kStat = T < 256 ? 2 * T : 512;
template <int T>
constexpr int kSliceCols = T < 512 ? 8 * T : (int)kWideCols;

template <int T, int Q>
__device__ __forceinline__ void group_sums(const Plan& p, const Place& at,
                                           int t, const float* buf,
                                           const float* w, float* stat)
{
    int team = T < 64 ? T : 64;
    while (team > 1 && team * at.ng > T) team >>= 1;
    const int each = p.parts_across > 1 ? at.cols : (int)p.each;
    const int l = t % team;
    for (int g = t / team; g < at.ng; g += T / team) {
        float sum[Q] = {};
        for (int d = l; d < each; d += team) {
            const int c = g * each + d;
#pragma unroll
            for (int q = 0; q < Q; ++q)
                sum[q] = w ? fmaf(buf[q * 8 * T + c], w[c], sum[q])
                           : sum[q] + buf[q * 8 * T + c];
        }
        for (int off = team >> 1; off > 0; off >>= 1)
#pragma unroll
            for (int q = 0; q < Q; ++q) sum[q] += __shfl_xor(sum[q], off);
        if (l == 0) {
#pragma unroll
            for (int q = 0; q < Q; ++q) stat[q * kStat<T> + g] = sum[q];
        }
    }
    __syncthreads();
}

template <int T>
constexpr int kSlabThreads = T > 256 ? T : 256;

// Where unit j of a slice begins, and how many positions it has.
struct Unit {
    int64_t n, ch, row;
    int rows;
    __device__ __forceinline__ Unit(const GroupArgs& a, int64_t j)
    {
        n = a.p.chunks > 1 ? j / a.p.chunks : j;
        ch = a.p.chunks > 1 ? j - n * a.p.chunks : 0;
        const int64_t r0 = ch * a.p.chunk;
        row = n * a.positions + r0;
        const int64_t left = a.positions - r0;
        rows = j < a.samples * a.p.chunks
                   ? (int)(left < a.p.chunk ? left : a.p.chunk)
                   : 0;
    }
};

__device__ __forceinline__ void load_eight(int dt, const void* p, int64_t at,
                                           int count, float fill,
                                           float (&v)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        v[e] = fill;
        if (p && e < count) {
            if (dt == SVM_F32) v[e] = ((const float*)p)[at + e];
            else if (dt == SVM_BF16) v[e] = (float)((const __bf16*)p)[at + e];
            else v[e] = (float)((const _Float16*)p)[at + e];
        }
    }
}

// PARTS: only the chunks' statistics, else the whole of a sample.
template <int DT, int T, int IT, bool PARTS>
__global__ __launch_bounds__(kSlabThreads<T>) void k_group_norm(GroupArgs a)
{
    constexpr int kSlabs = kSlabThreads<T> / T;
    __shared__ float bufs[kSlabs][8 * T], stats[kSlabs][2 * kStat<T>];
    const Plan& p = a.p;
    const int slab = threadIdx.x / T, t = threadIdx.x % T;
    float *buf = bufs[slab], *stat = stats[slab];
    const int64_t slice = blockIdx.x % p.slices;
    const int64_t nb = gridDim.x / p.slices;
    const Place at(a, slice, t);
    const int64_t units = a.samples * p.chunks;
    float w[8], b[8];
    if (!PARTS) {
        load_eight(DT, a.w, at.col + at.lane * 8, at.count, 1.0f, w);
        load_eight(DT, a.b, at.col + at.lane * 8, at.count, 0.0f, b);
    }
    for (int64_t j0 = blockIdx.x / p.slices * kSlabs; j0 < units;
         j0 += nb * kSlabs) {
        const Unit u(a, j0 + slab);
        const int64_t first = u.row * a.ldx + at.col + at.lane * 8;
        RawEight<DT> x[IT];
        float v[1][8] = {};
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            const int r = at.row + i * p.rows;
            x[i].load(a.X, first + r * a.ldx, r < u.rows ? at.count : 0);
        }
#pragma unroll
        for (int i = 0; i < IT; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[0][e] += x[i].at(e);
        column_sums<T, 1>(p, at, t, v, buf);
        group_sums<T, 1>(p, at, t, buf, nullptr, stat);
        const float size =
            (float)((int64_t)u.rows *
                    (p.parts_across > 1 ? (int64_t)at.cols : p.each));
        float mu[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            mu[e] = stat[at.group[e]] / size;
            v[0][e] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            const bool there = at.row + i * p.rows < u.rows;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float d = x[i].at(e) - mu[e];
                if (there && e < at.count) v[0][e] = fmaf(d, d, v[0][e]);
            }
        }
        column_sums<T, 1>(p, at, t, v, buf);
        group_sums<T, 1>(p, at, t, buf, nullptr, stat + kStat<T>);
        if (u.rows > 0)
            for (int g = t; g < at.ng; g += T) {
                const int64_t ng = u.n * a.groups + at.g0 + g;
                const float m = stat[g] / size, q = stat[kStat<T> + g];
                if (PARTS) {
                    const int64_t cp =
                        p.parts_across > 1 ? slice % p.parts_across : 0;
                    a.part[ng * p.parts() + cp * p.chunks + u.ch] =
                        make_float2(m, q);
                } else {
                    if (a.mean) a.mean[ng] = m;
                    if (a.rstd) a.rstd[ng] = 1.0f / sqrtf(q / size + a.eps);
                }
            }
        if (PARTS) continue;
        float rs[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            rs[e] = 1.0f / sqrtf(stat[kStat<T> + at.group[e]] / size + a.eps);
        const int64_t to = u.row * a.ldo + at.col + at.lane * 8;
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            const int r = at.row + i * p.rows;
            Eight<DT> y;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                y.v[e] = fmaf((x[i].at(e) - mu[e]) * rs[e], w[e], b[e]);
            act_values(a.act, y.v);
            if (r < u.rows && at.count > 0)
                y.store(a.out, to + r * a.ldo, at.count);
        }
    }
}

// Joins the chunks' statistics of a group, a wave to a group: the mean of
// the parts' means by their sizes, and the squares about it.  SUMS: adds the
// parts of a gradient's two sums instead.
template <bool SUMS>
__global__ __launch_bounds__(256) void k_group_join(GroupArgs a, float2* sums)
{
    const Plan& p = a.p;
    const int lane = threadIdx.x & 63;
    const int64_t all = a.samples * a.groups;
    const int64_t parts = p.parts();
    const float size = (float)(a.positions * p.each);
    for (int64_t g = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); g < all;
         g += (int64_t)gridDim.x * 4) {
        const float2* q = a.part + g * parts;
        float s0 = 0.0f, s1 = 0.0f;
        auto count = [&](int64_t i) {
            const int64_t cp = i / p.chunks, ch = i - cp * p.chunks;
            const int64_t r = a.positions - ch * p.chunk;
            const int64_t c = p.parts_across > 1 ? p.each - cp * p.cols
                                                 : p.each;
            const int64_t wide = p.parts_across > 1 ? p.cols : p.each;
            return (float)((r < p.chunk ? r : p.chunk) *
                           (c < wide ? c : wide));
        };
        for (int64_t i = lane; i < parts; i += 64) {
            const float2 v = q[i];
            s0 += SUMS ? v.x : v.x * count(i);
            s1 += v.y;
        }
        s0 = SUMS ? wave_sum(s0) : wave_sum(s0) / size;
        s1 = wave_sum(s1);
        if (SUMS) {
            if (lane == 0) sums[g] = make_float2(s0, s1);
            continue;
        }
        float far = 0.0f;
        for (int64_t i = lane; i < parts; i += 64) {
            const float d = q[i].x - s0;
            far = fmaf(d * d, count(i), far);
        }
        s1 += wave_sum(far);
        if (lane == 0) {
            a.mean[g] = s0;
            a.rstd[g] = 1.0f / sqrtf(s1 / size + a.eps);
        }
    }
}

// mean and rstd of a thread's columns
__device__ __forceinline__ void load_stats(const GroupArgs& a, const Place& at,
                                           int64_t n, float (&mu)[8],
                                           float (&rs)[8])
{
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int64_t g = n * a.groups + at.g0 + at.group[e];
        mu[e] = a.mean[g];
        rs[e] = a.rstd[g];
    }
}

// The slope of the activation at z = (x - mu) rs w + b.  For relu it is a
// matter of z's sign, which is settled in 64 bits: within 32 bits' rounding of
// 0 the slope would be off by all of itself.
__device__ __forceinline__ void slopes(const GroupArgs& a,
                                       const float (&x)[8],
                                       const float (&mu)[8],
                                       const float (&rs)[8],
                                       const float (&xh)[8],
                                       const float (&w)[8],
                                       const float (&b)[8], float (&s)[8])
{
    if (a.act == SVM_ACT_RELU) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const double z = fma(((double)x[e] - (double)mu[e]) *
                                     (double)rs[e], (double)w[e],
                                 (double)b[e]);
            s[e] = z > 0.0 ? 1.0f : 0.0f;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        s[e] = a.act == SVM_ACT_NONE ? 1.0f : fmaf(xh[e], w[e], b[e]);
    act_slopes(a.act, s);
}

// Applies joined statistics: the output, or with GRAD dX from the joined sums.
// A thread to 8 columns, positions in turn.  Bound by memory.
template <int DT, bool GRAD>
__global__ __launch_bounds__(256) void k_group_apply(GroupArgs a)
{
    const Plan& p = a.p;
    const int64_t slice = blockIdx.x % p.slices;
    const int64_t nb = gridDim.x / p.slices;
    // (the plan's lanes fit 256 threads or take them in turns)
    const int64_t units = a.samples * p.chunks;
    const int step = p.lanes < 256 ? 256 / p.lanes : 1;
    for (int t0 = 0; t0 < p.lanes; t0 += 256) {
        const int t = p.lanes < 256 ? (int)threadIdx.x
                                    : t0 + (int)threadIdx.x;
        if (p.lanes >= 256 && t >= p.lanes) continue;
        const Place at(a, slice, t);
        const int row = p.lanes < 256 ? at.row : 0;
        const int count = row < step ? eight_of(at.cols, at.lane * 8) : 0;
        if (count == 0) continue;
        const int64_t c = at.col + at.lane * 8;
        float w[8], b[8];
        load_eight(DT, a.w, c, count, 1.0f, w);
        load_eight(DT, a.b, c, count, 0.0f, b);
        const float over = 1.0f / (float)(a.positions * p.each);
        for (int64_t j = blockIdx.x / p.slices; j < units; j += nb) {
            const Unit u(a, j);
            float mu[8], rs[8], s1[8], s2[8];
            load_stats(a, at, u.n, mu, rs);
            if (GRAD) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float2 s =
                        a.sums[u.n * a.groups + at.g0 + at.group[e]];
                    s1[e] = s.x * over;
                    s2[e] = s.y * over;
                }
            }
#pragma unroll 4
            for (int r = row; r < u.rows; r += step) {
                const int64_t i = u.row + r;
                Eight<DT> x, y;
                x.load(a.X, i * a.ldx + c, count);
                if (!GRAD) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        y.v[e] = fmaf((x.v[e] - mu[e]) * rs[e], w[e], b[e]);
                    act_values(a.act, y.v);
                } else {
                    Eight<DT> g, q;
                    float xh[8], s[8];
                    g.load(a.dY, i * a.ldg + c, count);
                    if (a.res) q.load(a.res, i * a.ldr + c, count);
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        xh[e] = (x.v[e] - mu[e]) * rs[e];
                    slopes(a, x.v, mu, rs, xh, w, b, s);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float d = g.v[e] * s[e] * w[e];
                        y.v[e] = rs[e] * (d - fmaf(xh[e], s2[e], s1[e]));
                        if (a.res) y.v[e] += q.v[e];
                    }
                }
                y.store(a.out, i * a.ldo + c, count);
            }
        }
    }
}

// The gradients of slabs in registers.  PARTS: only the sums, by chunks and
// for weight and bias.  A block keeps to one slice and adds up what its
// columns get over all of its units.
template <int DT, int T, int IT, bool PARTS>
__global__ __launch_bounds__(kSlabThreads<T>) void k_group_grad(GroupArgs a)
{
    constexpr int kSlabs = kSlabThreads<T> / T;
    __shared__ float bufs[kSlabs][2 * 8 * T], stats[kSlabs][2 * kStat<T>];
    __shared__ float ws[kSliceCols<T>];  // the slice's weights
    const Plan& p = a.p;
    const int slab = threadIdx.x / T, t = threadIdx.x % T;
    float *buf = bufs[slab], *stat = stats[slab];
    const int64_t slice = blockIdx.x % p.slices;
    const int64_t nb = gridDim.x / p.slices;
    const Place at(a, slice, t);
    const int64_t units = a.samples * p.chunks;
    float w[8], b[8];
    load_eight(DT, a.w, at.col + at.lane * 8, at.count, 1.0f, w);
    load_eight(DT, a.b, at.col + at.lane * 8, at.count, 0.0f, b);
    if (slab == 0 && at.row == 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e < at.count) ws[at.lane * 8 + e] = w[e];
    }
    // sums of columns t, t + T, ... of both kinds over the block's units
    float tot[16] = {};
    const float over = 1.0f / (float)(a.positions * p.each);
    for (int64_t j0 = blockIdx.x / p.slices * kSlabs; j0 < units;
         j0 += nb * kSlabs) {
        const Unit u(a, j0 + slab);
        float mu[8], rs[8];
        if (u.rows > 0) {
            load_stats(a, at, u.n, mu, rs);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) mu[e] = rs[e] = 0.0f;
        }
        const int64_t fx = u.row * a.ldx + at.col + at.lane * 8;
        const int64_t fg = u.row * a.ldg + at.col + at.lane * 8;
        RawEight<DT> x[IT], g[IT];
        float dz[IT][8], v[2][8] = {};
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            const int r = at.row + i * p.rows;
            const int count = r < u.rows ? at.count : 0;
            x[i].load(a.X, fx + r * a.ldx, count);
            g[i].load(a.dY, fg + r * a.ldg, count);
        }
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            const int count = at.row + i * p.rows < u.rows ? at.count : 0;
            float xv[8], xh[8], s[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                xv[e] = x[i].at(e);
                xh[e] = (xv[e] - mu[e]) * rs[e];
            }
            slopes(a, xv, mu, rs, xh, w, b, s);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                // (past the ends neither the sums nor a NaN get in)
                dz[i][e] = e < count ? g[i].at(e) * s[e] : 0.0f;
                v[0][e] += dz[i][e];
                if (e < count) v[1][e] = fmaf(dz[i][e], xh[e], v[1][e]);
            }
        }
        column_sums<T, 2>(p, at, t, v, buf);
        if (a.pw) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int c = t + k * T;
                if (c < at.cols) {
                    tot[k] += buf[c];
                    tot[8 + k] += buf[8 * T + c];
                }
            }
        }
        if (!PARTS && !a.out) continue;
        group_sums<T, 2>(p, at, t, buf, ws, stat);
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
        float s1[8], s2[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            s1[e] = stat[at.group[e]] * over;
            s2[e] = stat[kStat<T> + at.group[e]] * over;
        }
        const int64_t fr = u.row * a.ldr + at.col + at.lane * 8;
        const int64_t fo = u.row * a.ldo + at.col + at.lane * 8;
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            const int r = at.row + i * p.rows;
            const int count = r < u.rows ? at.count : 0;
            Eight<DT> d, q;
            if (a.res) q.load(a.res, fr + r * a.ldr, count);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float xh = (x[i].at(e) - mu[e]) * rs[e];
                d.v[e] = rs[e] * (dz[i][e] * w[e] - fmaf(xh, s2[e], s1[e]));
                if (a.res) d.v[e] += q.v[e];
            }
            if (count > 0) d.store(a.out, fo + r * a.ldo, count);
        }
    }
    if (!a.pw) return;
    // the block's row of the partial sums, its slabs' added up
    const int64_t to = blockIdx.x / p.slices * (a.groups * p.each) + at.col;
    if constexpr (kSlabs > 1) {
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            buf[t + k * T] = tot[k];
            buf[8 * T + t + k * T] = tot[8 + k];
        }
        __syncthreads();
        for (int c = threadIdx.x; c < at.cols; c += kSlabThreads<T>) {
            float sb = 0.0f, sw = 0.0f;
#pragma unroll
            for (int i = 0; i < kSlabs; ++i) {
                sb += bufs[i][c];
                sw += bufs[i][8 * T + c];
            }
            a.pb[to + c] = sb;
            a.pw[to + c] = sw;
        }
    } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const int c = t + k * T;
            if (c < at.cols) {
                a.pb[to + c] = tot[k];
                a.pw[to + c] = tot[8 + k];
            }
        }
    }
}

constexpr int kMostPieces16 = 8, kMostPieces32 = 4;

int most_pieces(int32_t dtype)
{
    return dtype == SVM_F32 ? kMostPieces32 : kMostPieces16;
}

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// The cut of a call.  Slices begin as narrow as fills a line of memory (more
// slabs), and grow while a slab has too little to do.
Plan plan_of(int64_t samples, int64_t positions, int64_t channels,
             int64_t groups, int32_t dtype)
{
    Plan p{};
    p.each = channels / groups;
    p.parts_across = p.each > kWideCols ? up(p.each, kWideCols) : 1;
    if (p.parts_across > 1) {
        p.groups = 1;
        p.cols = kWideCols;
        p.slices = groups * p.parts_across;
    } else {
        const int64_t line = dtype == SVM_F32 ? 32 : 64;
        p.groups = up(line, p.each);
        while (p.groups < groups && positions * p.groups * p.each < 1024 &&
               p.groups * 2 * p.each <= 512)
            p.groups *= 2;
        if (p.groups > groups) p.groups = groups;
        p.cols = p.groups * p.each;
        p.slices = up(groups, p.groups);
    }
    p.lanes = (int)up(p.cols, 8);
    const int most = most_pieces(dtype);
    const int64_t units = samples * p.slices;
    // threads for a slab: few pieces to each where there are few slabs
    int t = 16;
    auto fits = [&](int threads, int pieces) {
        return p.lanes <= threads && p.groups <= 2 * threads &&
               up(positions, threads / p.lanes) <= pieces;
    };
    while (t < 1024 && !fits(t, units * t < 131072 ? 1 : most / 2)) t *= 4;
    const bool whole = fits(t, most) && p.parts_across == 1;
    // a slab for each sample leaves most of the card idle
    const bool few = units * t < 65536 &&
                     samples * positions * channels > 1 << 18;
    p.chunk = positions;
    p.chunks = 1;
    if (!whole || (few && positions > 1)) {
        t = p.lanes > 256 ? 1024 : 256;
        const int64_t rows = t / p.lanes;
        // chunks that fill the card's blocks, but no longer than fits
        int64_t chunk = up(positions * units, 2048);
        if (chunk < rows) chunk = rows;
        if (chunk > rows * most) chunk = rows * most;
        p.chunk = chunk < positions ? chunk : positions;
        p.chunks = up(positions, p.chunk);
    }
    p.threads = t;
    p.rows = t / p.lanes;
    int64_t need = up(p.chunk, p.rows);
    p.pieces = need <= 1 ? 1 : need <= 2 ? 2 : need <= 4 ? 4 : 8;
    return p;
}

// Calls f with the threads and pieces of a plan.
template <int DT, class F>
void for_plan(const Plan& p, F&& f)
{
    auto pieces = [&]<int T>() {
        if (p.pieces == 1) f.template operator()<T, 1>();
        else if (p.pieces == 2) f.template operator()<T, 2>();
        else if (DT == SVM_F32 || p.pieces == 4) f.template operator()<T, 4>();
        else if constexpr (DT != SVM_F32) f.template operator()<T, 8>();
    };
    if (p.threads == 16) pieces.template operator()<16>();
    else if (p.threads == 64) pieces.template operator()<64>();
    else if (p.threads == 256) pieces.template operator()<256>();
    else pieces.template operator()<1024>();
}

// Blocks to a slice: each has a unit or more for each of its slabs.
int64_t blocks_across(const GroupArgs& a, int64_t most)
{
    const int64_t slabs = a.p.threads < 256 ? 256 / a.p.threads : 1;
    int64_t nb = up(a.samples * a.p.chunks, slabs);
    const int64_t cap = most / a.p.slices > 1 ? most / a.p.slices : 1;
    return nb < cap ? nb : cap;
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
    a.ldo = c.Y.ld;
    a.samples = samples;
    a.positions = c.positions;
    a.groups = c.groups;
    a.eps = c.eps;
    a.act = c.act;
    a.mean = c.mean;
    a.rstd = c.rstd;
    a.p = plan_of(samples, c.positions, c.X.cols, c.groups, c.X.dtype);
    const Plan& p = a.p;
    const int64_t all = samples * c.groups;
    if (p.split()) {
        a.part = ws.take<float2>(all * p.parts());
        float* mean = ws.take<float>(all);
        float* rstd = ws.take<float>(all);
        if (!a.mean) a.mean = mean;
        if (!a.rstd) a.rstd = rstd;
    }
    if (!ws.run || samples == 0) return;
    for_dtype(c.X.dtype, [&]<int DT>() {
        const int64_t nb = blocks_across(a, 1 << 20);
        const dim3 grid((unsigned)(nb * p.slices));
        for_plan<DT>(p, [&]<int T, int IT>() {
            if (!p.split()) {
                hipLaunchKernelGGL((k_group_norm<DT, T, IT, false>), grid,
                                   dim3(kSlabThreads<T>), 0, s, a);
                return;
            }
            if constexpr (T >= 256)
                hipLaunchKernelGGL((k_group_norm<DT, T, IT, true>), grid,
                                   dim3(kSlabThreads<T>), 0, s, a);
        });
        if (!p.split()) return;
        const int64_t jb = up(all, 4);
        hipLaunchKernelGGL((k_group_join<false>),
                           dim3((unsigned)(jb < 65536 ? jb : 65536)),
                           dim3(256), 0, s, a, (float2*)nullptr);
        hipLaunchKernelGGL((k_group_apply<DT, false>), grid, dim3(256), 0, s,
                           a);
    });
}

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
    a.samples = samples;
    a.positions = c.positions;
    a.groups = c.groups;
    a.act = c.act;
    a.mean = const_cast<float*>(c.mean);
    a.rstd = const_cast<float*>(c.rstd);
    a.p = plan_of(samples, c.positions, n, c.groups, c.X.dtype);
    const Plan& p = a.p;
    const bool sums = c.sums;
    const int64_t rows = samples ? blocks_across(a, kGroupUnits) : 0;
    const int64_t all = samples * c.groups;
    if (sums) {
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
    if (samples > 0 && (sums || a.out))
        for_dtype(c.X.dtype, [&]<int DT>() {
            const dim3 grid((unsigned)(blocks_across(a, kGroupUnits) *
                                       p.slices));
            for_plan<DT>(p, [&]<int T, int IT>() {
                if (!p.split()) {
                    hipLaunchKernelGGL((k_group_grad<DT, T, IT, false>), grid,
                                       dim3(kSlabThreads<T>), 0, s, a);
                    return;
                }
                if constexpr (T >= 256)
                    hipLaunchKernelGGL((k_group_grad<DT, T, IT, true>), grid,
                                       dim3(kSlabThreads<T>), 0, s, a);
            });
            if (!p.split() || !a.out) return;
            const int64_t jb = up(all, 4);
            hipLaunchKernelGGL((k_group_join<true>),
                               dim3((unsigned)(jb < 65536 ? jb : 65536)),
                               dim3(256), 0, s, a, joined);
            hipLaunchKernelGGL((k_group_apply<DT, true>),
                               dim3((unsigned)(blocks_across(a, 1 << 20) *
                                               p.slices)),
                               dim3(256), 0, s, a);
        });
    if (sums)
        launch_column_sums(a.pw, a.pb, rows, n, c.X.dtype, c.dweight.data,
                           c.dbias.data, s);
}

}  // namespace msvm
