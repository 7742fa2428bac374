// Group norm with an activation over samples x positions x channels, channels
// last: how a call is cut up, and what its kernels (groupnorm.hip) and those
// of its gradients (groupgrad.hip) share.
//
// A unit of work is a slab: the positions of one sample (or a chunk of them)
// by a slice of columns, whole groups side by side, wide enough to fill the
// memory's lines (groups of more than kWideCols channels are cut into slices
// of their own).  T threads hold a slab in registers, each 8 columns of every
// R-th position, from its read to its write.  Where the 8 columns of a thread
// lie in one group, its sum is one number, and the threads' numbers are joined
// through LDS; for groups of other widths the sums are joined by columns
// first.  Where a sample's slab is too large, or slabs are too few to fill the
// card, the positions are cut into chunks: one launch for the chunks' sums,
// one that joins them, and one that applies them and reads the values again.
#pragma once

#include "elem.hpp"
#include "layers.hpp"

namespace msvm {
namespace {

constexpr int64_t kWideCols = 4096;

// Division by d of numbers n with n d < 2^32: one multiplication (by 2^32 / d
// rounded up: too much by n / 2^32, less than the 1 / d to the next quotient).
// Blocks are short, and a handful of divisions would be most of their work.
struct Divisor {
    uint32_t d, m;
    __host__ __device__ Divisor(uint32_t d = 1)
        : d(d), m((uint32_t)((((uint64_t)1 << 32) + d - 1) / d))
    {
    }
    __device__ __forceinline__ int operator()(int n) const
    {
        return d == 1 ? n : (int)__umulhi((uint32_t)n, m);
    }
};

// How a call is cut up.  All by the sizes and the type.
struct Plan {
    int threads, pieces;   // of a slab: T, and IT pieces of 8 for each
    int lanes, rows;       // lanes across the slice; positions at a time
    int64_t each;          // channels of a group
    int64_t groups;        // of a slice (1 where a group has several slices)
    int64_t cols;          // of a slice
    int64_t slices, parts_across;  // of a row; of a group
    int64_t chunk, chunks; // positions of a chunk; chunks of a sample
    bool even;             // the 8 columns of a thread lie in one group
    Divisor by_lanes, by_each, by_wide;  // lanes; each; 8 lanes
    __host__ __device__ bool split() const
    {
        return chunks > 1 || parts_across > 1;
    }
    __host__ __device__ int64_t parts() const { return chunks * parts_across; }
};

struct GroupArgs {
    const void *X, *dY, *res, *w, *b;
    void* out;
    int64_t ldx, ldg, ldr, ldo;
    int64_t samples, positions, groups;
    int64_t endx, endg, endr;  // of the inputs, in values
    float eps;
    int act;
    float *mean, *rstd;     // written by the forward pass, else read
    double2* moments;       // means of the chunks, and squares about them
    float2* part;           // a gradient's sums of the chunks
    const float2* sums;     // joined sums of a gradient
    float *pw, *pb;         // rows of partial sums for weight and bias
    Plan p;
};

// Threads of a block, slabs of it; groups and columns of a slice at most.
template <int T>
constexpr int kSlabThreads = T > 256 ? T : 256;
template <int T>
constexpr int kSlabs = kSlabThreads<T> / T;
template <int T>
constexpr int kStat = T < 256 ? 2 * T : 512;

// What a thread has of the slab of its slice.
template <bool EVEN>
struct Place {
    static constexpr int kK = EVEN ? 1 : 8;  // groups that it may meet
    int64_t col, g0;  // first column and group
    int lane, row;    // of the 8-column pieces; first position
    int count;        // columns that there are, of 8
    int cols, ng;     // of this slice
    int group[kK];    // of the thread's columns, in the slice

    __device__ __forceinline__ Place(const GroupArgs& a, int64_t slice, int t)
    {
        const Plan& p = a.p;
        row = p.by_lanes(t);
        lane = t - row * p.lanes;
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
        // the first column's group, and where the next one begins
        int g = p.parts_across > 1 ? 0 : p.by_each(lane * 8);
        int next = p.parts_across > 1 ? 1 << 30
                                      : (g + 1) * (int)p.each - lane * 8;
#pragma unroll
        for (int e = 0; e < kK; ++e) {
            if (e == next) {
                ++g;
                next += (int)p.each;
            }
            group[e] = g < ng ? g : ng - 1;
        }
    }
    __device__ __forceinline__ int64_t first() const { return col + lane * 8; }
    // channels of a group that are in this slice
    __device__ __forceinline__ int each(const Plan& p) const
    {
        return p.parts_across > 1 ? cols : (int)p.each;
    }
};

// Where unit j of a slice begins, and how many positions it has (none past
// the last unit).
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

// Waits for the threads of a slab (one wave's LDS accesses are in order).
template <int T>
__device__ __forceinline__ void slab_sync()
{
    if constexpr (T <= 64) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    } else {
        __syncthreads();
    }
}

// Adds up Q quantities of a slab's threads by groups: one thread calls
// done(g, the sums) for each, and the others wait for it.  v is a thread's one
// number (EVEN) or its 8 columns' sums.  buf: T or 8 T floats for each
// quantity; its earlier contents have been read by all threads before the
// last slab_sync.
template <int T, int Q, bool EVEN, class F>
__device__ __forceinline__ void group_sums(
    const Plan& p, const Place<EVEN>& at, int t,
    const float (&v)[Q][Place<EVEN>::kK], float* buf, F&& done)
{
    int team = T < 64 ? T : 64;
    while (team > 1 && team * at.ng > T) team >>= 1;
    const int shift = __builtin_ctz(team);
    const int l = t & (team - 1), first = t >> shift, step = T >> shift;
    const int each = at.each(p);
    const int wide = EVEN ? p.lanes : p.lanes * 8;
    constexpr int kOne = EVEN ? T : 8 * T;
    int rows = p.rows, width = each;
    if constexpr (EVEN) {
        if (at.row < p.rows) {
#pragma unroll
            for (int q = 0; q < Q; ++q)
                buf[q * kOne + at.row * wide + at.lane] = v[q][0];
        }
        slab_sync<T>();
        width = each / 8;
    } else {
        if (at.row < p.rows) {
#pragma unroll
            for (int q = 0; q < Q; ++q)
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    buf[q * kOne + at.row * wide + at.lane * 8 + e] = v[q][e];
        }
        slab_sync<T>();
    }
    if (!EVEN && p.rows > 1) {
        // columns first: as many rows are left as the threads have turns
        const int turns = p.by_wide(T);
        rows = turns < 1 ? 1 : turns < p.rows ? turns : p.rows;
        for (int i = t; i < rows * wide; i += T) {
            const int r0 = p.by_wide(i);
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                float* s = buf + q * kOne + (i - r0 * wide);
                float sum = s[r0 * wide];
#pragma unroll 4
                for (int r = r0 + rows; r < p.rows; r += rows)
                    sum += s[r * wide];
                s[r0 * wide] = sum;
            }
        }
        slab_sync<T>();
    }
    const int items = rows * width;
    constexpr int kAtOnce = T <= 16 ? 4 : 1;  // (large teams have few each)
    for (int g = first; g < at.ng; g += step) {
        float sum[Q] = {};
        // (EVEN: i / (each / 8) = 8 i / each)
#pragma unroll kAtOnce
        for (int i = l; i < items; i += team) {
            const int r = p.parts_across > 1
                              ? (int)((unsigned)i / (unsigned)width)
                              : p.by_each(EVEN ? 8 * i : i);
            const int c = r * wide + g * width + (i - r * width);
#pragma unroll
            for (int q = 0; q < Q; ++q) sum[q] += buf[q * kOne + c];
        }
        for (int off = team >> 1; off > 0; off >>= 1)
#pragma unroll
            for (int q = 0; q < Q; ++q) sum[q] += __shfl_xor(sum[q], off);
        if (l == 0) done(g, sum);
    }
    slab_sync<T>();
}

// A vector's values at a thread's columns, or `fill`: loaded raw, so that
// other loads can follow, and turned into 32 bits later.
template <int DT>
struct Eights {
    RawEight<DT> raw;
    __device__ __forceinline__ void load(const void* p, int64_t at, int count,
                                         float fill)
    {
        raw.ones();
        if (fill == 0.0f) {
#pragma unroll
            for (int k = 0; k < RawEight<DT>::kN; ++k)
                raw.v[k] = (Elem<DT>)0.0f;
        }
        if (p) raw.load(p, at, count);
    }
    __device__ __forceinline__ void values(float (&v)[8]) const
    {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = raw.at(e);
    }
};

// The first `count` of eight values to at, in as few stores as there are
// powers of two in it.
template <int DT, bool EVEN>
__device__ __forceinline__ void store_some(const Eight<DT>& y, void* p,
                                           int64_t at, int count)
{
    using T = Elem<DT>;
    if (EVEN || count == 8) {
        y.store(p, at, 8);
        return;
    }
    typedef T Four __attribute__((ext_vector_type(4)));
    typedef T Two __attribute__((ext_vector_type(2)));
    typedef Four LooseFour __attribute__((aligned(sizeof(T))));
    typedef Two LooseTwo __attribute__((aligned(sizeof(T))));
    T* q = (T*)p + at;
    const Four lo = {(T)y.v[0], (T)y.v[1], (T)y.v[2], (T)y.v[3]};
    const Four hi = {(T)y.v[4], (T)y.v[5], (T)y.v[6], (T)y.v[7]};
    if (count & 4) {
        *(LooseFour*)q = lo;
        q += 4;
    }
    const Four left = count & 4 ? hi : lo;
    if (count & 2) {
        *(LooseTwo*)q = Two{left[0], left[1]};
        q += 2;
    }
    if (count & 1) *q = count & 2 ? left[2] : left[0];
}

// The compiler is neither to keep what it made of these registers before (the
// values in 32 bits, twice the room) nor to make it ahead of its turn.
template <int DT>
__device__ __forceinline__ void forget(RawEight<DT>& x)
{
#pragma unroll
    for (int k = 0; k < RawEight<DT>::kN; ++k) asm volatile("" : "+v"(x.v[k]));
}

// These are to be made here (left to the end of a loop, what they are made of
// stays in registers until then).
template <int N>
__device__ __forceinline__ void settle(float (&v)[N])
{
#pragma unroll
    for (int k = 0; k < N; ++k) asm volatile("" : "+v"(v[k]));
}

// The values from `by` on take the first places (by < 8; the last are left).
template <int DT>
__device__ __forceinline__ void shift(RawEight<DT>& x, int by)
{
    typedef uint32_t U4 __attribute__((ext_vector_type(4)));
    uint32_t d[4 * RawEight<DT>::kN];
#pragma unroll
    for (int k = 0; k < RawEight<DT>::kN; ++k) {
        const U4 u = __builtin_bit_cast(U4, x.v[k]);
#pragma unroll
        for (int e = 0; e < 4; ++e) d[4 * k + e] = u[e];
    }
    constexpr int kWords = 4 * RawEight<DT>::kN;
    if constexpr (DT != SVM_F32) {
        if (by & 1)
#pragma unroll
            for (int e = 0; e < kWords; ++e)
                d[e] = __builtin_amdgcn_alignbit(
                    e + 1 < kWords ? d[e + 1] : 0u, d[e], 16);
        by >>= 1;
    }
#pragma unroll
    for (int step = 1; step < kWords; step *= 2)
        if (by & step)
#pragma unroll
            for (int e = 0; e + step < kWords; ++e) d[e] = d[e + step];
#pragma unroll
    for (int k = 0; k < RawEight<DT>::kN; ++k)
        x.v[k] = __builtin_bit_cast(
            decltype(x.v[k] + x.v[k]),
            U4{d[4 * k], d[4 * k + 1], d[4 * k + 2], d[4 * k + 3]});
}

// A value that the compiler knows nothing about: what is made of it is made
// where it is used (offsets of all pieces, made ahead of a loop over slabs,
// would take two registers for each piece and array).
__device__ __forceinline__ int64_t here(int64_t v)
{
    int lo = (int)v, hi = (int)(v >> 32);
    asm volatile("" : "+v"(lo), "+v"(hi));
    return (int64_t)((uint64_t)(uint32_t)hi << 32 | (uint32_t)lo);
}

// The pieces of a slab: all loads before the first use.  `at` is the thread's
// first value, `last` its value in the slab's last position: past that a piece
// is the last one again (a branch around a load would have the next wait for
// it).  Past the slice's columns a piece has what follows in memory, whose
// sums nobody reads; where that would be past the array's end, the eight
// values before the end are loaded and shifted into place.  (Arrays of fewer
// than eight values: plans of one piece, values loaded one by one.)
template <int DT, int IT>
__device__ __forceinline__ void load_slab(RawEight<DT> (&x)[IT], const void* X,
                                          int64_t at, int64_t step,
                                          int64_t last, bool any, int count,
                                          int64_t end)
{
    if (!any) {
#pragma unroll
        for (int i = 0; i < IT; ++i) x[i].ones();
        return;
    }
    if constexpr (IT == 1) {
        const int64_t a = at < last ? at : last;
        x[0].load(X, a, a + 8 <= end ? 8 : count);
    } else {
        int64_t a = here(at);
#pragma unroll
        for (int i = 0; i < IT; ++i) {
            int64_t b = a < last ? a : last;
            b = b < end - 8 ? b : end - 8;
            x[i].load(X, b, 8);
            a += step;
        }
        if (last > end - 8) {
            a = here(at);
#pragma unroll
            for (int i = 0; i < IT; ++i) {
                const int64_t by = (a < last ? a : last) - (end - 8);
                if (by > 0) shift(x[i], (int)by);
                a += step;
            }
        }
    }
}

int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Pieces of a thread at most: 64 registers for the forward pass' raw values;
// the gradient holds the values and 32 bits of each gradient.
int most_pieces(int32_t dtype, bool grad)
{
    if (grad) return dtype == SVM_F32 ? 4 : 8;
    return dtype == SVM_F32 ? 8 : 16;
}

// The pieces that the kernels are made for, from `need` on.
int pieces_of(int threads, int64_t need)
{
    if (need <= 1) return 1;  // (8 threads: never more)
    if (threads == 16) return 2;
    if (need <= 2 && threads == 256) return 2;
    return need <= 4 ? 4 : need <= 8 ? 8 : 16;
}

// The cut of a call.  Slices begin as narrow as fills a line of memory (more
// slabs), and grow while a slab has too little to do.
Plan plan_of(int64_t samples, int64_t positions, int64_t channels,
             int64_t groups, int32_t dtype, bool grad)
{
    Plan p{};
    if (samples == 0) positions = 1;  // (there may be any number of them)
    p.each = channels / groups;
    p.parts_across = p.each > kWideCols ? up(p.each, kWideCols) : 1;
    p.even = p.each % 8 == 0;
    if (p.parts_across > 1) {
        p.groups = 1;
        p.cols = kWideCols;
        p.slices = groups * p.parts_across;
    } else {
        const int64_t line = dtype == SVM_F32 ? 32 : 64;
        p.groups = up(line, p.each);
        // rows of whole eights: slices of whole eights too, so that they begin
        // where 16 bytes do
        int64_t k = 1;
        while (channels % 8 == 0 && k * p.each % 8) k *= 2;
        if (k * p.each <= 512) p.groups = up(p.groups, k) * k;
        while (p.groups < groups && positions * p.groups * p.each < 1024 &&
               p.groups * 2 * p.each <= 512)
            p.groups *= 2;
        if (p.groups > groups) p.groups = groups;
        p.cols = p.groups * p.each;
        p.slices = up(groups, p.groups);
    }
    p.lanes = (int)up(p.cols, 8);
    const int most = most_pieces(dtype, grad);
    // large samples: half a line, where that spares reading them again (64 x
    // 1024 x 256 in groups of 8, bf16: gradients 51.7 us, in chunks 60.7)
    const int64_t room = (int64_t)512 * most * 8;
    const int64_t half = p.groups / 2;
    if (p.parts_across == 1 && p.groups % 2 == 0 && half * p.each % 8 == 0 &&
        half * p.each * (dtype == SVM_F32 ? 4 : 2) >= 64 &&
        positions * p.cols > room && positions * half * p.each <= room) {
        p.groups = half;
        p.cols = p.groups * p.each;
        p.slices = up(groups, p.groups);
        p.lanes = (int)up(p.cols, 8);
    }
    const int64_t units = samples * p.slices;
    constexpr int kThreads[5] = {8, 16, 64, 256, 512};
    constexpr int kPieces[5] = {1, 2, 4, 8, 16};
    auto fits = [&](int i, int64_t pieces) {
        const int t = kThreads[i];
        if (pieces > kPieces[i]) pieces = kPieces[i];
        if (pieces > most) pieces = most;
        return p.lanes <= t && p.groups <= 2 * t &&
               up(positions, t / p.lanes) <= pieces;
    };
    int i = 0;
    // few slabs: more threads to each, so that they are done sooner
    while (i < 4 && !fits(i, units * kThreads[i] < 131072 ? 1 : 16)) ++i;
    bool whole = p.parts_across == 1 && fits(i, 16);
    // a slab for each sample leaves most of the card idle
    if (units * kThreads[i] < 65536 &&
        samples * positions * channels > 1 << 18 && positions > 1)
        whole = false;
    p.chunk = positions;
    p.chunks = 1;
    if (!whole) {
        if (p.parts_across == 1) {
            // the rows whole, up to 512 columns: chunks make enough units
            p.slices = up(channels, 512);
            if (p.slices > groups) p.slices = groups;
            p.groups = up(groups, p.slices);
            p.slices = up(groups, p.groups);
            p.cols = p.groups * p.each;
            p.lanes = (int)up(p.cols, 8);
        }
        i = p.lanes > 256 ? 4 : 3;
        const int64_t rows = kThreads[i] / p.lanes;
        const int64_t deep = most < 8 ? most : 8;
        // chunks enough for two blocks to a CU, but no longer than fits
        // (gradients of 6 x 3977 x 231, f16: 512 units 39.9 us, 384 39.6, 256
        // 41.3, 1024 46.3, 2048 54.2; of 1 x 3977 x 231 27.8, with 256 24.6;
        // of 4 x 2000 x 512, bf16: 25.9, with 256 29.1)
        int64_t chunk = up(positions * samples * p.slices, 512);
        if (chunk < rows) chunk = rows;
        if (chunk > rows * deep) chunk = rows * deep;
        p.chunk = chunk < positions ? chunk : positions;
        p.chunks = up(positions, p.chunk);
    }
    p.threads = kThreads[i];
    p.rows = p.threads / p.lanes;
    p.by_lanes = Divisor((uint32_t)p.lanes);
    p.by_each = Divisor((uint32_t)p.each);
    p.by_wide = Divisor((uint32_t)p.lanes * 8);
    p.pieces = pieces_of(p.threads, up(p.chunk, p.rows));
    if (p.pieces > most) p.pieces = most;
    return p;
}

// Calls f with the threads and pieces of a plan and whether it is even.
template <int DT, bool GRAD, class F>
void for_plan(const Plan& p, F&& f)
{
    constexpr int kMost = GRAD ? (DT == SVM_F32 ? 4 : 8)
                               : (DT == SVM_F32 ? 8 : 16);
    auto go = [&]<int T, int IT>() {
        if (p.even) f.template operator()<T, IT, true>();
        else f.template operator()<T, IT, false>();
    };
    if (p.threads == 8) {
        go.template operator()<8, 1>();
    } else if (p.threads == 16) {
        if (p.pieces == 1) go.template operator()<16, 1>();
        else go.template operator()<16, 2>();
    } else if (p.threads == 64) {
        if (p.pieces == 1) go.template operator()<64, 1>();
        else go.template operator()<64, 4>();
    } else if (p.threads == 256) {
        if (p.pieces == 1) go.template operator()<256, 1>();
        else if (p.pieces == 2) go.template operator()<256, 2>();
        else if (p.pieces == 4) go.template operator()<256, 4>();
        else if constexpr (kMost >= 8) go.template operator()<256, 8>();
    } else {
        if (p.pieces == 1) go.template operator()<512, 1>();
        else if (p.pieces == 4) go.template operator()<512, 4>();
        else if (p.pieces == 8) {
            if constexpr (kMost >= 8) go.template operator()<512, 8>();
        } else if constexpr (kMost >= 16) {
            go.template operator()<512, 16>();
        }
    }
}

// The same for the kernel that applies joined sums: its chunks are as long as
// its threads load ahead, or longer where there are enough of them.
Plan apply_plan(const GroupArgs& a, int ahead)
{
    Plan p = a.p;
    const int64_t turn = (p.lanes < 256 ? 256 / p.lanes : 1) * ahead;
    const int64_t turns =
        up(up(a.positions * a.samples * p.slices, turn), 8192);
    p.chunk = turn * turns < a.positions ? turn * turns : a.positions;
    p.chunks = up(a.positions, p.chunk);
    return p;
}

// Blocks to a slice: each has a unit or more for each of its slabs.
int64_t blocks_across(const GroupArgs& a, int64_t most)
{
    const int64_t slabs = a.p.threads < 256 ? 256 / a.p.threads : 1;
    const int64_t nb = up(a.samples * a.p.chunks, slabs);
    const int64_t cap = most / a.p.slices > 1 ? most / a.p.slices : 1;
    return nb < cap ? nb : cap;
}

__device__ __forceinline__ double wave_sum64(double v)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off);
    return v;
}

// Joins the chunks' sums of a group, a wave to a group: the mean of the
// parts' means by their sizes, in 64 bits (rounded once: equal means give
// themselves), and the squares about it.  SUMS: adds the parts of a gradient's
// two sums instead.
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
        auto count = [&](int64_t i) {
            const int64_t cp = p.parts_across > 1 ? i / p.chunks : 0;
            const int64_t ch = i - cp * p.chunks;
            const int64_t r = a.positions - ch * p.chunk;
            const int64_t c = p.parts_across > 1 ? p.each - cp * p.cols
                                                 : p.each;
            const int64_t wide = p.parts_across > 1 ? p.cols : p.each;
            return (float)((r < p.chunk ? r : p.chunk) *
                           (c < wide ? c : wide));
        };
        if (SUMS) {
            const float2* q = a.part + g * parts;
            float s0 = 0.0f, s1 = 0.0f;
            for (int64_t i = lane; i < parts; i += 64) {
                const float2 v = q[i];
                s0 += v.x;
                s1 += v.y;
            }
            s0 = wave_sum(s0);
            s1 = wave_sum(s1);
            if (lane == 0) sums[g] = make_float2(s0, s1);
            continue;
        }
        const double2* q = a.moments + g * parts;
        double s0 = 0.0;
        float s1 = 0.0f;
        for (int64_t i = lane; i < parts; i += 64) {
            const double2 v = q[i];
            s0 += v.x * (double)count(i);
            s1 += (float)v.y;
        }
        const double mu = wave_sum64(s0) / (double)size;
        s1 = wave_sum(s1);
        float far = 0.0f;
        for (int64_t i = lane; i < parts; i += 64) {
            const float d = (float)(q[i].x - mu);
            far = fmaf(d * d, count(i), far);
        }
        s1 += wave_sum(far);
        if (lane == 0) {
            a.mean[g] = (float)mu;
            a.rstd[g] = 1.0f / sqrtf(s1 / size + a.eps);
        }
    }
}

int64_t end_of(const svm_array& x)
{
    if (x.rows <= 0) return 0;
    return (int64_t)((uint64_t)(x.rows - 1) * (uint64_t)x.ld + x.cols);
}

template <bool SUMS>
void launch_join(const GroupArgs& a, float2* sums, hipStream_t s)
{
    const int64_t nb = up(a.samples * a.groups, 4);
    hipLaunchKernelGGL((k_group_join<SUMS>),
                       dim3((unsigned)(nb < 65536 ? nb : 65536)), dim3(256), 0,
                       s, a, sums);
}

// A thread's columns and rows of an applying kernel: 256 threads, the plan's
// lanes across (more than 256 in turns).  f(at, row, step, count).
template <bool EVEN, class F>
__device__ __forceinline__ void for_lanes(const GroupArgs& a, int64_t slice,
                                          F&& f)
{
    const int lanes = a.p.lanes;
    const int step = lanes < 256 ? 256 / lanes : 1;
    for (int t0 = 0; t0 < lanes; t0 += 256) {
        const int t = t0 + (int)threadIdx.x;
        const Place<EVEN> at(a, slice, t);
        const int row = lanes < 256 ? at.row : 0;
        const int count = row < step && (lanes < 256 || t < lanes)
                              ? eight_of(at.cols, at.lane * 8)
                              : 0;
        if (count > 0) f(at, row, step, count);
        if (lanes < 256) break;
    }
}

}  // namespace
}  // namespace msvm
