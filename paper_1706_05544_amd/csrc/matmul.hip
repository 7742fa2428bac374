// The matrix product of the feature-map operators on the matrix cores.
//
// An output tile of BM x BN belongs to one block; the summed index runs in
// steps of 64.  Both factors' tiles of a step go from HBM straight into LDS
// (16 bytes a lane, no registers between), into the buffer that the step
// before last has left, while the step at hand is multiplied from the other:
//   top of a step: the fragments of its first 32 summed values are in
//   registers;  read those of the second 32, multiply the first;  wait for
//   the next step's tiles, meet the other waves: all have read this buffer;
//   start the loads of the step after next into it, read the next step's
//   first fragments from the other buffer, multiply the second 32.
// So one barrier a step, and a whole step's time for a load to arrive.
//
// LDS rows of a factor stored along the summed index hold 8 pieces of 16
// bytes; piece c of row r lies at c ^ key(r), so that the 8 lanes that read
// at once read 8 different pieces of a 128-byte line.  A factor stored across
// it (rows of the other index) is read with the transposing LDS load, 4 rows
// of 32 bytes at once; there piece c of row r lies at c ^ 2 (r mod 4).
// Loads past a factor's end return zeros (the buffer descriptor's range), so
// edges need no branches; in the last step, pieces past the summed index are
// given an address past the end.
//
// The fragments are multiplied as D^T = B A^T, so that a lane holds four
// consecutive columns of an output row.  The sums go through LDS once more,
// to be finished (bias, activation, residual) and written in whole rows of
// 16 bytes a lane from a rolled loop.
#include "elem.hpp"
#include "matmul.hpp"

namespace msvm {

namespace {

constexpr int kBK = 64;         // summed values of a step
// An address past every descriptor: the rows of a tile end below it, and
// added to a tile's own offsets it does not wrap.
constexpr uint32_t kPast = 0x80000000u;
constexpr int kVmcnt0 = 0x0f70;  // s_waitcnt: loads only

typedef short short4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

template <int DT>
__device__ __forceinline__ floatx4 mfma(short8v a, short8v b, floatx4 c)
{
    if constexpr (DT == SVM_F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(
            __builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
            0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            __builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0,
            0, 0);
}

// Products of the planes of 32-bit factors (0: leading 8 bits), the smallest
// first.  The three that are left out (1 2, 2 1, 2 2) are below 2^-24 of the
// whole.
constexpr uint32_t kSegA = 0x010120;  // plane of product s at 4 s bits
constexpr uint32_t kSegB = 0x001102;
__device__ __forceinline__ int64_t plane_of(uint32_t planes, int seg)
{
    return (planes >> (4 * seg)) & 15;
}

struct Args {
    Factor A, B;
    int64_t m, n, k;
    int nk;             // steps of a product (32 bits: of one of planes)
    int splits, per;    // parts of all steps, steps of a part
    unsigned tm, tn;    // tiles
    float* part;        // splits > 1: sums, splits x m x n
    Epilogue e;
    int wide;           // outputs and residual in aligned rows of 16 bytes
};

// The lane's share of a factor's tile loads: R rows (ALONG) or columns.
template <int R, int NW, bool ALONG>
struct Stage {
    static constexpr int kInstr = R / 8 / NW;  // loads of a wave, 1 KiB each
    static constexpr int kRowLanes = ALONG ? 8 : R / 8;  // 16-byte pieces
    static constexpr int kRows = 64 / kRowLanes;         // rows of a load
    uint32_t off[2];  // byte offset in the tile, for each kind of load
    int piece;        // first summed value of the piece (ALONG, kind 0)

    __device__ __forceinline__ void init(int64_t ld, int lane)
    {
        const int row = lane / kRowLanes, pos = lane % kRowLanes;
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            int c;
            if (ALONG) {
                // rows 8 q + row: key = (r & 3) | ((r >> 2 ^ r >> 4) & 1) << 2
                c = pos ^ ((row & 3) | (((row >> 2) ^ v) & 1) << 2);
            } else {
                const int r = kRows == 2 ? v * 2 + row : row;
                c = pos ^ (2 * (r & 3));
            }
            if (v == 0) piece = c * 8;
            off[v] = (uint32_t)((int64_t)row * ld * 2 + c * 16);
        }
    }

    // Loads the tile whose first element is `base` (bytes left: `left`).
    // summed: summed values left from here (ALONG).
    __device__ __forceinline__ void load(const char* base, int64_t left,
                                         int ld2, int summed, short* lds,
                                         int wave) const
    {
        // (the range ends at a whole dword: a dword that lies half past it
        // would be returned as zero)
        const uint32_t range = left <= 0          ? 0u
                               : left < kPast - 4 ? ((uint32_t)left + 3) & ~3u
                                                  : kPast;
        __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<char*>(base), 0, (int)range, 0x00020000);
        uint32_t o[2] = {off[0], off[1]};
        if (ALONG) {
            if (piece >= summed) o[0] = kPast;
            if ((piece ^ 32) >= summed) o[1] = kPast;
        }
#pragma unroll
        for (int it = 0; it < kInstr; ++it) {
            const int q = wave * kInstr + it;
            // which kind load q is
            const int v = ALONG ? (q >> 1) & 1 : kRows == 2 ? q & 1 : 0;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rs, (__attribute__((address_space(3))) void*)(lds + q * 512),
                16, v ? o[1] : o[0], (uint32_t)(q * kRows) * (uint32_t)ld2, 0,
                0);
        }
    }
};

// Where the loads of a factor are: the tile of the next step.
struct Cursor {
    const char* at;
    int64_t left;  // bytes from there to the factor's end
};

// Reads a fragment: 16 rows (of the factor's other index) x 32 summed values.
template <int R, bool ALONG>
struct Frag {
    int base[2];

    // first: the wave's first row of the tile
    __device__ __forceinline__ void init(int first, int lane)
    {
        const int i = lane & 15, g = lane >> 4;
        if (ALONG) {
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                const int key = (i & 3) | (((i >> 2) ^ v) & 1) << 2;
                base[v] = (first + i) * 64 + (g ^ key) * 8;
            }
        } else {
            const int r = 8 * g + (i >> 2);  // summed value; + 4: same key
            base[0] = r * R;
            base[1] = (i & 3) * 4;
        }
    }

    // fragment f (rows first + 16 f ..), summed values 32 h .. of the step
    __device__ __forceinline__ short8v read(const short* lds, int first, int f,
                                            int h, int lane) const
    {
        if (ALONG) {
            // bit 4 of the row (the wave's first is a multiple of 32)
            const int b = f & 1 ? base[1] : base[0];
            return *(const short8v*)(lds + (b ^ (h * 32)) + f * 16 * 64);
        } else {
            const int key = 2 * ((lane >> 2) & 3);
            const int col = first + f * 16 + base[1];
            const int at = ((col >> 3) ^ key) * 8 + (col & 7);
            using P = __attribute__((address_space(3))) short4v*;
            const short* p = lds + base[0] + h * 32 * R + at;
            short4v a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)p);
            short4v b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (P)(p + 4 * R));
            return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
};

// Eight consecutive values of an output row.
template <int DT>
struct Eight {
    float v[8];

    __device__ __forceinline__ void load(const void* p, int64_t at, bool wide,
                                         int count)
    {
        using T = Elem<DT>;
        const T* q = (const T*)p + at;
        if (wide) {
            if constexpr (DT == SVM_F32) {
                const float4 a = *(const float4*)q, b = *(const float4*)(q + 4);
                v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
                v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
            } else {
                typedef T T8 __attribute__((ext_vector_type(8)));
                const T8 a = *(const T8*)q;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = (float)a[e];
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = e < count ? (float)q[e] : 0.0f;
        }
    }

    __device__ __forceinline__ void store(void* p, int64_t at, bool wide,
                                          int count) const
    {
        using T = Elem<DT>;
        T* q = (T*)p + at;
        if (wide) {
            if constexpr (DT == SVM_F32) {
                *(float4*)q = make_float4(v[0], v[1], v[2], v[3]);
                *(float4*)(q + 4) = make_float4(v[4], v[5], v[6], v[7]);
            } else {
                typedef T T8 __attribute__((ext_vector_type(8)));
                T8 a;
#pragma unroll
                for (int e = 0; e < 8; ++e) a[e] = (T)v[e];
                *(T8*)q = a;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < count) q[e] = (T)v[e];
        }
    }
};

// A sum of 32-bit factors that is not finite, again from the factors
// themselves: an infinity has zeros or other signs in its lower planes.
__device__ __forceinline__ float exact_sum(const Factor& A, const Factor& B,
                                           int64_t i, int64_t j, int64_t k)
{
    const float* a = A.exact + (A.along ? i * A.exact_ld : i);
    const float* b = B.exact + (B.along ? j * B.exact_ld : j);
    const int64_t sa = A.along ? 1 : A.exact_ld;
    const int64_t sb = B.along ? 1 : B.exact_ld;
    float sum = 0.0f;
#pragma unroll 1
    for (int64_t r = 0; r < k; ++r) sum = fmaf(a[r * sa], b[r * sb], sum);
    return sum;
}

// Finishes eight sums of row i from column j on and writes them.
template <int OT>
__device__ __forceinline__ void finish(const Args& p, Eight<OT>& x,
                                       const Eight<OT>& bias,
                                       const Eight<OT>& res, int64_t i,
                                       int64_t j, bool wide, int count)
{
    const Epilogue& e = p.e;
    if constexpr (OT == SVM_F32) {
        bool fine = true;
#pragma unroll
        for (int c = 0; c < 8; ++c)
            fine &= fabsf(x.v[c]) <= 3.402823466e38f;
        if (!fine) {
#pragma unroll 1
            for (int c = 0; c < count; ++c) {
                const float s = exact_sum(p.A, p.B, i, j + c, p.k);
#pragma unroll
                for (int d = 0; d < 8; ++d)
                    if (d == c && !(fabsf(x.v[d]) <= 3.402823466e38f))
                        x.v[d] = s;
            }
        }
    }
#pragma unroll
    for (int c = 0; c < 8; ++c) x.v[c] += bias.v[c];
    if (e.Z) x.store(e.Z, i * e.ldz + j, wide, count);
    act_values(e.act, x.v);
    if (e.residual) {
#pragma unroll
        for (int c = 0; c < 8; ++c) x.v[c] += res.v[c];
    }
    x.store(e.Y, i * e.ldy + j, wide, count);
}

// Tile of block b: each XCD takes a run of consecutive tiles (blocks go to
// the 8 XCDs in turn), in bands of 8 tile rows, so that the tiles that one
// L2 serves at a time share their factors' rows.
__device__ __forceinline__ void tile_of(unsigned b, unsigned tm, unsigned tn,
                                        unsigned& ti, unsigned& tj)
{
    const unsigned total = tm * tn, full = total / 8, rest = total % 8;
    const unsigned x = b % 8, y = b / 8;
    const unsigned t = x * full + (x < rest ? x : rest) + y;
    const unsigned band = t / (8 * tn);
    const unsigned rows = tm - band * 8 < 8 ? tm - band * 8 : 8;
    const unsigned in = t - band * 8 * tn;
    ti = band * 8 + in % rows;
    tj = in / rows;
}

// IT: type of the 16-bit factors; OT: type of the outputs.
template <int IT, int OT, int BM, int BN, int WGM, int WGN, bool AALONG,
          bool BALONG>
__global__ __launch_bounds__(64 * WGM * WGN) void k_product(Args p)
{
    constexpr int NW = WGM * WGN;
    constexpr int FM = BM / WGM / 16, FN = BN / WGN / 16;
    constexpr int kSegs = OT == SVM_F32 ? 6 : 1;
    constexpr int kLds = (BM + BN) * kBK;  // values of a buffer
    __shared__ __align__(1024) short lds0[kLds];
    __shared__ __align__(1024) short lds1[kLds];

    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    unsigned ti, tj;
    tile_of(blockIdx.x, p.tm, p.tn, ti, tj);
    const int64_t i0 = (int64_t)ti * BM, j0 = (int64_t)tj * BN;
    const int wi = wave / WGN * (BM / WGM), wj = wave % WGN * (BN / WGN);

    Stage<BM, NW, AALONG> sa;
    Stage<BN, NW, BALONG> sb;
    Frag<BM, AALONG> fa;
    Frag<BN, BALONG> fb;
    sa.init(p.A.ld, lane);
    sb.init(p.B.ld, lane);
    fa.init(wi, lane);
    fb.init(wj, lane);

    // Steps t0 .. t1 - 1 of the products of planes one after another.
    const int t0 = blockIdx.y * p.per;
    const int all = kSegs * p.nk;
    const int t1 = t0 + p.per < all ? t0 + p.per : all;
    const int lda2 = (int)p.A.ld * 2, ldb2 = (int)p.B.ld * 2;
    const int64_t stepa = AALONG ? 2 * kBK : (int64_t)kBK * lda2;
    const int64_t stepb = BALONG ? 2 * kBK : (int64_t)kBK * ldb2;
    int seg = kSegs > 1 ? t0 / p.nk : 0;
    int tl = t0 - seg * p.nk;  // step of the next loads in its product
    int todo = t1 - t0;        // steps not loaded yet
    Cursor ca, cb;
    auto seek = [&]() {
        const int64_t k0 = (int64_t)tl * kBK;
        ca.at = (const char*)p.A.data +
                (AALONG ? i0 * lda2 + k0 * 2 : k0 * lda2 + i0 * 2);
        ca.left = (AALONG ? (p.m - 1 - i0) * lda2 + (p.k - k0) * 2
                          : (p.k - 1 - k0) * lda2 + (p.m - i0) * 2);
        cb.at = (const char*)p.B.data +
                (BALONG ? j0 * ldb2 + k0 * 2 : k0 * ldb2 + j0 * 2);
        cb.left = (BALONG ? (p.n - 1 - j0) * ldb2 + (p.k - k0) * 2
                          : (p.k - 1 - k0) * ldb2 + (p.n - j0) * 2);
        if (kSegs > 1) {
            ca.at += 2 * plane_of(kSegA, seg) * p.A.plane;
            cb.at += 2 * plane_of(kSegB, seg) * p.B.plane;
        }
    };
    seek();
    // Loads of the next step; past the last one they return zeros.
    auto load = [&](short* lds) {
        const int summed = p.k - (int64_t)tl * kBK < kBK
                               ? (int)(p.k - (int64_t)tl * kBK)
                               : kBK;
        sa.load(ca.at, todo > 0 ? ca.left : 0, lda2, summed, lds, wave);
        sb.load(cb.at, todo > 0 ? cb.left : 0, ldb2, summed, lds + BM * kBK,
                wave);
        --todo;
        ++tl;
        ca.at += stepa;
        ca.left -= stepa;
        cb.at += stepb;
        cb.left -= stepb;
        if (kSegs > 1 && tl == p.nk) {
            tl = 0;
            ++seg;
            seek();
        }
    };

    floatx4 acc[FM][FN];
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int g = 0; g < FN; ++g) acc[f][g] = floatx4{0, 0, 0, 0};

    short8v a0[FM], b0[FN], a1[FM], b1[FN];
    auto frags = [&](const short* lds, int h, short8v* a, short8v* b) {
#pragma unroll
        for (int g = 0; g < FN; ++g)
            b[g] = fb.read(lds + BM * kBK, wj, g, h, lane);
#pragma unroll
        for (int f = 0; f < FM; ++f) a[f] = fa.read(lds, wi, f, h, lane);
    };
    auto multiply = [&](const short8v* a, const short8v* b) {
#pragma unroll
        for (int f = 0; f < FM; ++f)
#pragma unroll
            for (int g = 0; g < FN; ++g)
                acc[f][g] = mfma<IT>(b[g], a[f], acc[f][g]);
    };
    // The reads of a half spread over the products of the other half.
    constexpr int kReads = (AALONG ? FM : 2 * FM) + (BALONG ? FN : 2 * FN);
    constexpr int kMul = FM * FN;
    auto spread = [&]() {
#pragma unroll
        for (int r = 0; r < kReads; ++r) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(
                0x008, kMul / kReads > 2 ? 2 : kMul / kReads ? kMul / kReads : 1,
                0);
        }
    };
    // one step from `cur`, with the next in `oth`
    auto step = [&](short* cur, short* oth) {
        __builtin_amdgcn_sched_barrier(0);
        frags(cur, 1, a1, b1);
        multiply(a0, b0);
        spread();
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(kVmcnt0);
        __syncthreads();
        load(cur);
        __builtin_amdgcn_sched_barrier(0);
        frags(oth, 0, a0, b0);
        multiply(a1, b1);
        spread();
        __builtin_amdgcn_sched_barrier(0);
    };

    load(lds0);
    load(lds1);
    __builtin_amdgcn_s_waitcnt(kVmcnt0);
    __syncthreads();
    frags(lds0, 0, a0, b0);
    for (int t = t0; t < t1; t += 2) {
        step(lds0, lds1);
        if (t + 1 < t1) step(lds1, lds0);
    }
    __builtin_amdgcn_s_waitcnt(kVmcnt0);
    __syncthreads();

    // the wave's own part of the buffers, kRows rows of its columns at a time
    constexpr int kCols = FN * 16, kRows = BM / WGM < 64 ? BM / WGM : 64;
    constexpr int kWaveFloats = 2 * kLds / 2 / NW;
    static_assert(kRows * kCols <= kWaveFloats, "slab");
    static_assert(BM / WGM % 32 == 0 && BN / WGN % 32 == 0, "Frag");
    float* slab = (float*)(wave < NW / 2 ? lds0 : lds1) +
                  (wave % (NW / 2)) * kWaveFloats;
    constexpr int kLanes = kCols / 8;   // lanes of a row
    constexpr int kAtOnce = 64 / kLanes;
    const int lr = lane / kLanes, lc = lane % kLanes * 8;
    const int64_t j = j0 + wj + lc;
    const int64_t left = p.n - j;
    const int count = left >= 8 ? 8 : left > 0 ? (int)left : 0;
    const bool wide = p.wide && count == 8;
    Eight<OT> bias;
#pragma unroll
    for (int c = 0; c < 8; ++c) bias.v[c] = 0.0f;
    if (p.e.bias && p.splits == 1) bias.load(p.e.bias, j, wide, count);
#pragma unroll
    for (int s = 0; s < BM / WGM / kRows; ++s) {
#pragma unroll
        for (int f = 0; f < kRows / 16; ++f)
#pragma unroll
            for (int g = 0; g < FN; ++g) {
                const int r = f * 16 + (lane & 15);
                const int c = g * 4 + (lane >> 4);  // 4 columns each
                *(floatx4*)(slab + r * kCols + ((c ^ (r & 7)) * 4)) =
                    acc[s * (kRows / 16) + f][g];
            }
#pragma unroll 2
        for (int r0 = 0; r0 < kRows; r0 += kAtOnce) {
            const int r = r0 + lr;
            const int64_t i = i0 + wi + s * kRows + r;
            if (i < p.m && count > 0) {
                Eight<OT> x, res;
                const float* q = slab + r * kCols;
                const floatx4 u =
                    *(const floatx4*)(q + (((lc / 4) ^ (r & 7)) * 4));
                const floatx4 v =
                    *(const floatx4*)(q + (((lc / 4 + 1) ^ (r & 7)) * 4));
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    x.v[c] = u[c];
                    x.v[4 + c] = v[c];
                }
                if (p.splits > 1) {
                    Eight<SVM_F32> y;
#pragma unroll
                    for (int c = 0; c < 8; ++c) y.v[c] = x.v[c];
                    const int64_t at =
                        ((int64_t)blockIdx.y * p.m + i) * p.n + j;
                    y.store(p.part, at, count == 8 && (p.n & 3) == 0, count);
                } else {
                    if (p.e.residual)
                        res.load(p.e.residual, i * p.e.ldr + j, wide, count);
                    finish<OT>(p, x, bias, res, i, j, wide, count);
                }
            }
        }
    }
}

// Sums the parts of a split product and finishes it, eight columns a thread.
template <int OT>
__global__ __launch_bounds__(256) void k_join(Args p)
{
    const int64_t groups = (p.n + 7) / 8;
    const int64_t all = p.m * groups;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < all;
         t += (int64_t)gridDim.x * 256) {
        const int64_t i = t / groups, j = t % groups * 8;
        const int count = p.n - j < 8 ? (int)(p.n - j) : 8;
        const bool wide = p.wide && count == 8;
        Eight<OT> x, bias, res;
#pragma unroll
        for (int c = 0; c < 8; ++c) x.v[c] = bias.v[c] = 0.0f;
        for (int s = 0; s < p.splits; ++s) {
            Eight<SVM_F32> y;
            y.load(p.part, ((int64_t)s * p.m + i) * p.n + j,
                   count == 8 && (p.n & 3) == 0, count);
#pragma unroll
            for (int c = 0; c < 8; ++c) x.v[c] += y.v[c];
        }
        if (p.e.bias) bias.load(p.e.bias, j, wide, count);
        if (p.e.residual) res.load(p.e.residual, i * p.e.ldr + j, wide, count);
        finish<OT>(p, x, bias, res, i, j, wide, count);
    }
}

// ---- factors that cannot be read as they are

// The three bf16 parts of a 32-bit value: x = h + m + l, each part what is
// left rounded to nearest (to zero where rounding would overflow).
__device__ __forceinline__ void three_parts(float x, __bf16& h, __bf16& m,
                                            __bf16& l)
{
    h = (__bf16)x;
    if (!(fabsf(x) <= 3.402823466e38f)) {  // infinity, NaN: h alone
        m = l = (__bf16)0.0f;
        return;
    }
    if (!(fabsf((float)h) <= 3.402823466e38f))
        h = __builtin_bit_cast(
            __bf16, (unsigned short)(__builtin_bit_cast(uint32_t, x) >> 16));
    const float r = x - (float)h;
    m = (__bf16)r;
    l = (__bf16)(r - (float)m);
}

template <int DT>
__global__ __launch_bounds__(256) void k_planes(const Elem<DT>* X, int64_t ld,
                                                int64_t rows, int64_t cols,
                                                void* dst, int64_t ldp,
                                                int64_t plane)
{
    const int64_t groups = ldp / 8, all = rows * groups;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < all;
         t += (int64_t)gridDim.x * 256) {
        const int64_t i = t / groups, j = t % groups * 8;
        const Elem<DT>* x = X + i * ld + j;
        if constexpr (DT == SVM_F32) {
            typedef __bf16 B8 __attribute__((ext_vector_type(8)));
            B8 part[3];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                __bf16 h, m, l;
                three_parts(j + e < cols ? x[e] : 0.0f, h, m, l);
                part[0][e] = h, part[1][e] = m, part[2][e] = l;
            }
#pragma unroll
            for (int q = 0; q < 3; ++q)
                *(B8*)((__bf16*)dst + q * plane + i * ldp + j) = part[q];
        } else {
            typedef Elem<DT> T8 __attribute__((ext_vector_type(8)));
            T8 v;
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = j + e < cols ? x[e] : (Elem<DT>)0.0f;
            *(T8*)((Elem<DT>*)dst + i * ldp + j) = v;
        }
    }
}

bool wide_rows(const void* p, int64_t ld, int32_t dtype)
{
    return !p || (((uintptr_t)p & 15) == 0 &&
                  (ld * (int64_t)dtype_bytes(dtype)) % 16 == 0);
}

template <int IT, int OT, int BM, int BN, int WGM, int WGN>
void launch_tiles(const Args& a, hipStream_t s)
{
    const dim3 grid(a.tm * a.tn, (unsigned)a.splits), block(64 * WGM * WGN);
    if (a.A.along && a.B.along)
        hipLaunchKernelGGL((k_product<IT, OT, BM, BN, WGM, WGN, true, true>),
                           grid, block, 0, s, a);
    else if (a.A.along)
        hipLaunchKernelGGL((k_product<IT, OT, BM, BN, WGM, WGN, true, false>),
                           grid, block, 0, s, a);
    else
        hipLaunchKernelGGL((k_product<IT, OT, BM, BN, WGM, WGN, false, false>),
                           grid, block, 0, s, a);
}

template <int IT, int OT>
void launch_any(const Args& a, int tile, hipStream_t s)
{
    if (tile == 256) launch_tiles<IT, OT, 256, 256, 2, 4>(a, s);
    else if (tile == 128) launch_tiles<IT, OT, 128, 128, 2, 2>(a, s);
    else launch_tiles<IT, OT, 64, 64, 2, 2>(a, s);
}

int64_t tiles(int64_t m, int64_t n, int t)
{
    return ((m + t - 1) / t) * ((n + t - 1) / t);
}

constexpr int kCus = 256;

}  // namespace

bool factor_fits(const svm_array& a, bool along)
{
    return a.dtype != SVM_F32 && ((uintptr_t)a.data & 15) == 0 &&
           a.ld % 8 == 0 && a.ld <= kMaxWidth && (!along || a.cols % 8 == 0);
}

void launch_planes(const svm_array& a, void* dst, int64_t ldp, int64_t plane,
                   hipStream_t s)
{
    const int64_t all = a.rows * (ldp / 8);
    if (all == 0) return;
    const int64_t nb = (all + 255) / 256;
    for_dtype(a.dtype, [&]<int DT>() {
        hipLaunchKernelGGL((k_planes<DT>),
                           dim3((unsigned)(nb < 16384 ? nb : 16384)),
                           dim3(256), 0, s, (const Elem<DT>*)a.data, a.ld,
                           a.rows, a.cols, dst, ldp, plane);
    });
}

void product(const Product& p, Pieces& ws, hipStream_t s)
{
    if (p.m == 0 || p.n == 0) return;
    Args a{};
    a.A = p.A;
    a.B = p.B;
    a.m = p.m;
    a.n = p.n;
    a.k = p.k;
    a.e = p.e;
    const int segs = p.dtype == SVM_F32 ? 6 : 1;
    a.nk = (int)((p.k + kBK - 1) / kBK);
    // Tiles: the largest of which there are enough for every CU; then, where
    // there are still too few, the steps are split over blocks.
    int tile = 256;
    if (tiles(p.m, p.n, 256) < kCus) tile = 128;
    if (tile == 128 && tiles(p.m, p.n, 128) < kCus) tile = 64;
    const int64_t nt = tiles(p.m, p.n, tile);
    const int64_t steps = (int64_t)segs * a.nk;
    int64_t splits = 1;
    if (nt < kCus) splits = (2 * kCus) / nt;
    if (splits > steps / 4) splits = steps / 4;
    if (splits < 1) splits = 1;
    a.per = (int)((steps + splits - 1) / splits);
    a.splits = (int)((steps + a.per - 1) / a.per);
    a.tm = (unsigned)((p.m + tile - 1) / tile);
    a.tn = (unsigned)((p.n + tile - 1) / tile);
    if (a.splits > 1) a.part = ws.take<float>(a.splits * p.m * p.n);
    if (!ws.run) return;
    a.wide = wide_rows(a.e.Y, a.e.ldy, p.dtype) &&
             wide_rows(a.e.Z, a.e.ldz, p.dtype) &&
             wide_rows(a.e.residual, a.e.ldr, p.dtype) &&
             ((uintptr_t)a.e.bias & 15) == 0;
    if (p.dtype == SVM_F32) launch_any<SVM_BF16, SVM_F32>(a, tile, s);
    else if (p.dtype == SVM_BF16) launch_any<SVM_BF16, SVM_BF16>(a, tile, s);
    else launch_any<SVM_F16, SVM_F16>(a, tile, s);
    if (a.splits > 1) {
        const int64_t nb = (p.m * ((p.n + 7) / 8) + 255) / 256;
        for_dtype(p.dtype, [&]<int DT>() {
            hipLaunchKernelGGL((k_join<DT>),
                               dim3((unsigned)(nb < 16384 ? nb : 16384)),
                               dim3(256), 0, s, a);
        });
    }
}

}  // namespace msvm
