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
//
// What bounds it: the feeding of the matrix cores, which are at work in half
// of the cycles.  In a row of a hundred calls, normal values in bf16: 8192^3
// 795 us, 1380 TFLOP/s, where a factor lies along, 757 us, 1450, where both
// lie across (a library's product 677 us, 1620; after a pause its first ten
// calls run at 1290).  16384 x 4096 over 4096: 411 us, 1340 (library 358; 430
// after a pause), with bias, gelu, residual and Z 483 to 502, of which the
// finishing takes some 75.
#include <algorithm>
#include <cmath>

#include "elem.hpp"
#include "matmul.hpp"

namespace msvm {

namespace {

constexpr int kStep16 = 64;  // summed values of a step: 16-bit factors,
constexpr int kStep32 = 32;  // 32-bit ones (three parts)
// An address past every descriptor: the rows of a tile end below it, and
// added to a tile's own offsets it does not wrap.
constexpr uint32_t kPast = 0x80000000u;

typedef short short4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef int intx4 __attribute__((ext_vector_type(4)));
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

struct Args {
    Factor A, B;
    int64_t m, n, k;
    int nk;             // steps
    int splits, per;    // parts of all steps, steps of a part
    unsigned tm, tn;    // tiles
    float* part;        // splits > 1: sums, splits x m x n
    Epilogue e;
};

// 16 bytes for each lane from the buffer `rs` at off + soff into LDS, lane
// after lane.  In assembly, so that the compiler does not wait for loads
// under way before LDS reads that it takes to depend on them; meet() waits
// for those that a step needs.  It has no output register, and tells the
// compiler that m0 (where in LDS the loads go) is overwritten.
__device__ __forceinline__ void lds_load(intx4 rs, short* lds, uint32_t off,
                                         uint32_t soff)
{
    const uint32_t to =
        (uint32_t)(uintptr_t)(__attribute__((address_space(3))) short*)lds;
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"  // (m0 is never allocated)
    asm volatile(
        "s_mov_b32 m0, %0\n\ts_nop 0\n\t"
        "buffer_load_dwordx4 %1, %2, %3 offen lds"
        :
        : "s"(to), "v"(off), "s"(rs), "s"(soff)
        : "memory", "m0");
#pragma clang diagnostic pop
}

// The lane's share of a factor's tile loads: R rows (ALONG) or columns.
template <int R, int NW, bool ALONG>
struct Stage {
    static constexpr int kInstr = R / 8 / NW;  // of a wave, 1 KiB each
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
        const uint64_t at = (uint64_t)base;
        const intx4 rs = {(int)(uint32_t)at, (int)(uint32_t)(at >> 32),
                          (int)range, 0x00020000};
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
            lds_load(rs, lds + q * 512, v ? o[1] : o[0],
                     (uint32_t)(q * kRows) * (uint32_t)ld2);
        }
    }
};

// Waits until at most LEFT of the wave's loads are under way (they end in
// order) and its LDS reads are done, then for the block's other waves.
template <int LEFT>
__device__ __forceinline__ void meet()
{
    static_assert(LEFT < 64, "vmcnt");
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("" ::: "memory");
    // vmcnt LEFT, expcnt not waited, lgkmcnt 0
    __builtin_amdgcn_s_waitcnt((LEFT & 15) | (LEFT >> 4) << 14 | 7 << 4);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// A factor's tile loads step by step: R rows or columns.
template <int R, int NW, bool ALONG>
struct Walk {
    static constexpr int BK = kStep16;
    Stage<R, NW, ALONG> stage;
    const char* at;  // the tile of the next step
    int64_t left;    // bytes from there to the factor's end
    int64_t step;
    int ld2;

    // x0: first row or column of the tile, of n; t0: first step, of k values
    __device__ __forceinline__ void init(const Factor& f, int64_t x0, int64_t n,
                                         int64_t t0, int64_t k, int lane)
    {
        stage.init(f.ld, lane);
        ld2 = (int)f.ld * 2;
        step = ALONG ? 2 * BK : (int64_t)BK * ld2;
        const int64_t k0 = t0 * BK;
        at = (const char*)f.data + (ALONG ? x0 * ld2 + k0 * 2
                                          : k0 * ld2 + x0 * 2);
        left = ALONG ? (n - 1 - x0) * ld2 + (k - k0) * 2
                     : (k - 1 - k0) * ld2 + (n - x0) * 2;
    }

    // Loads the next step (`summed` values of it there; none: zeros).
    __device__ __forceinline__ void load(int summed, bool there, short* lds,
                                         int wave)
    {
        stage.load(at, there ? left : 0, ld2, summed, lds, wave);
        at += step;
        left -= step;
    }
};

// Reads a fragment: 16 rows (of the factor's other index) x 32 summed values.
template <int R, int BK, bool ALONG>
struct Frag {
    int base[2];

    // first: the wave's first row of the tile
    __device__ __forceinline__ void init(int first, int lane)
    {
        const int i = lane & 15, g = lane >> 4;
        if (ALONG) {
#pragma unroll
            for (int v = 0; v < 2; ++v) {
                const int key = BK == 64
                                    ? (i & 3) | (((i >> 2) ^ v) & 1) << 2
                                    : (i >> 1) & 3;
                base[v] = (first + i) * BK + (g ^ key) * 8;
            }
        } else {
            const int r = 8 * g + (i >> 2);  // summed value; + 4: same key
            base[0] = r * R;
            base[1] = (i & 3) * 4;
        }
    }

    // fragment f (rows first + 16 f ..), summed values 32 h .. of the step
    // (h = 1 only where BK is 64)
    __device__ __forceinline__ short8v read(const short* lds, int first, int f,
                                            int h, int lane) const
    {
        if (ALONG) {
            // bit 4 of the row (the wave's first is a multiple of 32)
            const int b = f & 1 ? base[1] : base[0];
            return *(const short8v*)(lds + (b ^ (h * 32)) + f * 16 * BK);
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

// ---- 32-bit sums that are not finite
//
// An infinity has zeros for its lower parts, its products with another
// factor's parts differ in sign, and what rounds past the largest bf16 is
// none: sums of three parts that come out not finite are formed again from
// the values as they are, by the 32-bit matrix instruction, a fragment of 16 x
// 16 outputs at a time.  A wave loads 64 summed values of both at once for it
// and shares nothing with the others, so that it is bound by the caches'
// latency: a product all of whose outputs are NaN takes 3 to 10 times one of
// finite values (50000 x 2048 over 784: 1.2 ms, all NaN 5.8; 256 x 256 over
// 100000: 112 us, all NaN 700; formed a sum to a lane it was some 300 times).

__device__ __forceinline__ bool is_finite(float v)
{
    return fabsf(v) <= 3.402823466e38f;
}

// 16 rows of a factor from x0 on (of n), for the matrix instruction: a lane
// has row lane mod 16 and four of every 16 summed values.
template <bool ALONG>
struct Rows16;

template <>
struct Rows16<true> {
    const float* row;
    bool there;

    __device__ __forceinline__ Rows16(const void* data, int64_t ld, int64_t x0,
                                      int64_t n, int lane)
        : row((const float*)data + (x0 + (lane & 15)) * ld),
          there(x0 + (lane & 15) < n)
    {
    }

    // Summed values r0 .. r0 + 63, zeros from `end` on.
    __device__ __forceinline__ void load(int64_t r0, int64_t end, int lane,
                                         floatx4 (&v)[4]) const
    {
        typedef floatx4 Loose __attribute__((aligned(4)));
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int64_t r = r0 + u * 16 + (lane >> 4) * 4;
            v[u] = floatx4{0, 0, 0, 0};
            if (!there) continue;
            if (r + 4 <= end) {
                v[u] = *(const Loose*)(row + r);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (r + e < end) v[u][e] = row[r + e];
            }
        }
    }
};

template <>
struct Rows16<false> {
    const float* col;  // x0 in the factor's first row (the same in all lanes)
    int64_t ld, width;

    __device__ __forceinline__ Rows16(const void* data, int64_t ld, int64_t x0,
                                      int64_t n, int)
        : col((const float*)data + x0), ld(ld), width(n - x0)
    {
    }

    // (row `end` and those after it lie past the descriptor's range: zeros)
    __device__ __forceinline__ void load(int64_t r0, int64_t end, int lane,
                                         floatx4 (&v)[4]) const
    {
        const int64_t left = 4 * ((end - 1 - r0) * ld + width);
        __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<float*>(col + r0 * ld), 0,
            (int)(left < 0xffffffff ? (uint32_t)left : 0xffffffffu),
            0x00020000);
        const int ld4 = (int)ld * 4;
        const int off = (lane >> 4) * 4 * ld4 + (lane & 15) * 4;
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[u][e] = __builtin_bit_cast(
                    float, __builtin_amdgcn_raw_buffer_load_b32(
                               rs, off, (u * 16 + e) * ld4, 0));
    }
};

// The sums of 16 x 16 outputs over summed values r0, r0 + step .., 64 from
// each, up to `end`.
template <bool AALONG, bool BALONG>
__device__ __forceinline__ floatx4 sums_32(const Rows16<AALONG>& a,
                                           const Rows16<BALONG>& b, int64_t r0,
                                           int64_t end, int step, int lane)
{
    floatx4 sum = {0, 0, 0, 0};
#pragma unroll 1
    for (int64_t r = r0; r < end; r += step) {
        floatx4 av[4], bv[4];
        a.load(r, end, lane, av);
        b.load(r, end, lane, bv);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                sum = __builtin_amdgcn_mfma_f32_16x16x4f32(bv[u][e], av[u][e],
                                                           sum, 0, 0, 0);
    }
    return sum;
}

// Forms those sums of a wave's tile again that are not finite: FM x FN
// fragments from row iw and column jw on, summed values [r0, end).
template <int FM, int FN, bool AALONG, bool BALONG>
__device__ __forceinline__ void mend_tile(const Args& p, floatx4 (&acc)[FM][FN],
                                          int64_t iw, int64_t jw, int64_t r0,
                                          int64_t end, int lane)
{
    static_assert(FM * FN <= 32, "a bit for each fragment");
    const int64_t il = iw + (lane & 15), jl = jw + (lane >> 4) * 4;
    unsigned bad = 0;  // fragments with such a sum, the same in every lane
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int g = 0; g < FN; ++g) {
            bool any = false;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                any |= !is_finite(acc[f][g][e]) && jl + g * 16 + e < p.n;
            if (__ballot(any && il + f * 16 < p.m)) bad |= 1u << (f * FN + g);
        }
    while (bad) {
        const int q = __builtin_ctz(bad);
        bad &= bad - 1;
        const floatx4 sum = sums_32(
            Rows16<AALONG>(p.A.data, p.A.ld, iw + q / FN * 16, p.m, lane),
            Rows16<BALONG>(p.B.data, p.B.ld, jw + q % FN * 16, p.n, lane), r0,
            end, 64, lane);
#pragma unroll
        for (int f = 0; f < FM; ++f)
#pragma unroll
            for (int g = 0; g < FN; ++g)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (q == f * FN + g && !is_finite(acc[f][g][e]))
                        acc[f][g][e] = sum[e];
    }
}

// Finishes eight sums of row i from column j on and writes them.
template <int OT>
__device__ __forceinline__ void finish(const Epilogue& e, Eight<OT>& x,
                                       const Eight<OT>& bias,
                                       const RawEight<OT>& res, int64_t i,
                                       int64_t j, int count)
{
#pragma unroll
    for (int c = 0; c < 8; ++c) x.v[c] += bias.v[c];
    if (e.Z) x.store(e.Z, i * e.ldz + j, count);
    act_values(e.act, x.v);
    if (e.residual) {
#pragma unroll
        for (int c = 0; c < 8; ++c) x.v[c] += res.at(c);
    }
    x.store(e.Y, i * e.ldy + j, count);
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

// The rows of a wave's tile that go through LDS at a time.
constexpr int slab_rows(int fm) { return fm * 16 < 64 ? fm * 16 : 64; }

// The wave's own part of the first two buffers: SLAB floats.
template <int SLAB, int NW, int LDS>
__device__ __forceinline__ float* wave_slab(short* lds0, short* lds1, int wave)
{
    static_assert(NW / 2 * SLAB * 4 <= LDS * 2, "slab");
    return (float*)(wave < NW / 2 ? lds0 : lds1) + (wave % (NW / 2)) * SLAB;
}

// Finishes and writes the sums of a wave's tile (FM x FN fragments, from row
// iw and column jw on); `slab` is LDS of its own.
template <int OT, int FM, int FN>
__device__ __forceinline__ void write_tile(const Args& p,
                                           const floatx4 (&acc)[FM][FN],
                                           float* slab, int64_t iw, int64_t jw,
                                           int lane)
{
    constexpr int kCols = FN * 16, kRows = slab_rows(FM);
    constexpr int kLanes = kCols / 8;   // lanes of a row
    constexpr int kAtOnce = 64 / kLanes;
    const int lr = lane / kLanes, lc = lane % kLanes * 8;
    const int64_t j = jw + lc;
    const int count = eight_of(p.n, j);
    Eight<OT> bias;
#pragma unroll
    for (int c = 0; c < 8; ++c) bias.v[c] = 0.0f;
    if (p.e.bias && p.splits == 1) bias.load(p.e.bias, j, count);
    constexpr int kTurns = kRows / kAtOnce, kGroup = kTurns < 2 ? kTurns : 2;
#pragma unroll
    for (int s = 0; s < FM * 16 / kRows; ++s) {
#pragma unroll
        for (int f = 0; f < kRows / 16; ++f)
#pragma unroll
            for (int g = 0; g < FN; ++g) {
                const int r = f * 16 + (lane & 15);
                const int c = g * 4 + (lane >> 4);  // 4 columns each
                *(floatx4*)(slab + r * kCols + ((c ^ (r & 7)) * 4)) =
                    acc[s * (kRows / 16) + f][g];
            }
        // turns of kAtOnce rows, kGroup of them with their residuals loaded
        // together, before any of them is written
#pragma unroll 1
        for (int t0 = 0; t0 < kTurns; t0 += kGroup) {
            RawEight<OT> res[kGroup];
            const int64_t i0 = iw + s * kRows + t0 * kAtOnce + lr;
#pragma unroll
            for (int u = 0; u < kGroup; ++u)
                if (p.e.residual && p.splits == 1 && i0 + u * kAtOnce < p.m)
                    res[u].load(p.e.residual,
                                (i0 + u * kAtOnce) * p.e.ldr + j, count);
#pragma unroll
            for (int u = 0; u < kGroup; ++u) {
                const int r = (t0 + u) * kAtOnce + lr;
                const int64_t i = i0 + u * kAtOnce;
                if (i >= p.m || count == 0) continue;
                Eight<OT> x;
                const float* q = slab + r * kCols;
                const floatx4 lo =
                    *(const floatx4*)(q + (((lc / 4) ^ (r & 7)) * 4));
                const floatx4 hi =
                    *(const floatx4*)(q + (((lc / 4 + 1) ^ (r & 7)) * 4));
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    x.v[c] = lo[c];
                    x.v[4 + c] = hi[c];
                }
                if (p.splits > 1) {
                    Eight<SVM_F32> y;
#pragma unroll
                    for (int c = 0; c < 8; ++c) y.v[c] = x.v[c];
                    y.store(p.part,
                            ((int64_t)blockIdx.y * p.m + i) * p.n + j, count);
                    continue;
                }
                finish<OT>(p.e, x, bias, res[u], i, j, count);
            }
        }
    }
}

// 16-bit factors.  ST: buffers, and so steps whose loads are under way.  Tiles
// of 256 read LDS least for each matrix instruction, and two buffers of them
// are all that LDS holds; those of 128 and 64 serve products with few tiles,
// whose loads' latency shows, and have four.  (Tiles of 256 on four waves of
// 128 x 128: slower, their sums must move between the two register files.)
template <int OT, int BM, int BN, int WGM, int WGN, int ST, bool AALONG,
          bool BALONG>
__global__ __launch_bounds__(64 * WGM * WGN) void k_product(Args p)
{
    constexpr int NW = WGM * WGN;
    constexpr int FM = BM / WGM / 16, FN = BN / WGN / 16;
    constexpr int kBK = kStep16, kSlab = slab_rows(FM) * FN * 16;
    constexpr int kLds = (BM + BN) * kBK;  // values of a buffer
    // (arrays of their own, so that the compiler knows a buffer that is being
    // loaded from one that is being read)
    __shared__ __align__(1024) short lds0[kLds];
    __shared__ __align__(1024) short lds1[kLds];
    __shared__ __align__(1024) short lds2[ST > 2 ? kLds : 8];
    __shared__ __align__(1024) short lds3[ST > 2 ? kLds : 8];
    static_assert(ST == 2 || ST == 4, "buffers");
    constexpr int kLoads = (BM + BN) / 8 / NW;  // of a wave in a step

    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    unsigned ti, tj;
    tile_of(blockIdx.x, p.tm, p.tn, ti, tj);
    const int64_t i0 = (int64_t)ti * BM, j0 = (int64_t)tj * BN;
    const int wi = wave / WGN * (BM / WGM), wj = wave % WGN * (BN / WGN);

    Frag<BM, kBK, AALONG> fa;
    Frag<BN, kBK, BALONG> fb;
    fa.init(wi, lane);
    fb.init(wj, lane);
    const int t0 = blockIdx.y * p.per;
    const int t1 = t0 + p.per < p.nk ? t0 + p.per : p.nk;
    Walk<BM, NW, AALONG> wa;
    Walk<BN, NW, BALONG> wb;
    wa.init(p.A, i0, p.m, t0, p.k, lane);
    wb.init(p.B, j0, p.n, t0, p.k, lane);
    int tl = t0;  // step of the next loads
    auto load = [&](short* lds) {
        const int64_t summed = p.k - (int64_t)tl * kBK;
        const int have = summed < kBK ? (int)summed : kBK;
        wa.load(have, tl < t1, lds, wave);
        wb.load(have, tl < t1, lds + BM * kBK, wave);
        ++tl;
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
                acc[f][g] = mfma<OT>(b[g], a[f], acc[f][g]);
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
        meet<(ST - 2) * kLoads>();
        load(cur);
        __builtin_amdgcn_sched_barrier(0);
        frags(oth, 0, a0, b0);
        multiply(a1, b1);
        spread();
        __builtin_amdgcn_sched_barrier(0);
    };

    load(lds0);
    load(lds1);
    if (ST > 2) {
        load(lds2);
        load(lds3);
    }
    meet<(ST - 1) * kLoads>();
    frags(lds0, 0, a0, b0);
    for (int t = t0; t < t1; t += ST) {
        step(lds0, lds1);
        if (t + 1 < t1) step(lds1, ST > 2 ? lds2 : lds0);
        if (ST > 2) {
            if (t + 2 < t1) step(lds2, lds3);
            if (t + 3 < t1) step(lds3, lds0);
        }
    }
    meet<0>();

    write_tile<OT, FM, FN>(p, acc,
                           wave_slab<kSlab, NW, kLds>(lds0, lds1, wave),
                           i0 + wi, j0 + wj, lane);
}

// A thread's share of a 32-bit factor's tile (R rows or columns, 32 summed
// values, T threads): pieces of 8 values from memory to registers, split there
// into three bf16 parts and written to LDS, a plane for each part.  Rows may
// begin anywhere; what lies past the factor's end comes as zeros.  LDS rows
// along the summed index have 4 pieces, two rows to 128 bytes: piece c of row
// r lies at c ^ (r / 2 mod 4).
template <int R, int T, bool ALONG>
struct Split {
    static constexpr int kN = R * 4 / T;  // pieces of a thread
    struct Raw {
        floatx4 v[kN][2];
    };
    uint32_t off[kN];  // byte offset in the tile
    int lds[kN];
    const char* at;    // the tile of the next step
    int64_t left, step;

    __device__ __forceinline__ void init(const Factor& f, int64_t x0, int64_t n,
                                         int64_t t0, int64_t k)
    {
        const int64_t k0 = t0 * kStep32;
        step = 4 * (ALONG ? kStep32 : kStep32 * f.ld);
        at = (const char*)f.data + 4 * (ALONG ? x0 * f.ld + k0
                                              : k0 * f.ld + x0);
        left = 4 * (ALONG ? (n - 1 - x0) * f.ld + k - k0
                          : (k - 1 - k0) * f.ld + n - x0);
#pragma unroll
        for (int q = 0; q < kN; ++q) {
            const int c = q * T + (int)threadIdx.x;
            const int across = ALONG ? 4 : R / 8;
            const int row = c / across, piece = c % across;
            off[q] = (uint32_t)((int64_t)row * f.ld * 4 + piece * 32);
            lds[q] = ALONG ? row * kStep32 + (piece ^ ((row >> 1) & 3)) * 8
                           : row * R + (piece ^ (2 * (row & 3))) * 8;
        }
    }

    // The next step's pieces (all of its summed values are there, or with
    // there = false none: zeros).
    __device__ __forceinline__ void load(Raw& raw, bool there)
    {
        const uint32_t range = !there || left <= 0 ? 0u
                               : left < 0xffffffff ? (uint32_t)left
                                                   : 0xffffffffu;
        __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc(
            const_cast<char*>(at), 0, (int)range, 0x00020000);
#pragma unroll
        for (int q = 0; q < kN; ++q)
#pragma unroll
            for (int h = 0; h < 2; ++h)
                raw.v[q][h] = __builtin_bit_cast(
                    floatx4, __builtin_amdgcn_raw_buffer_load_b128(
                              rs, (int)(off[q] + 16 * h), 0, 0));
        at += step;
        left -= step;
    }

    static __device__ __forceinline__ void split(const Raw& raw,
                                                 Bf16x8 (&part)[kN][3])
    {
#pragma unroll
        for (int q = 0; q < kN; ++q) {
            float v[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = raw.v[q][e / 4][e % 4];
            three_parts(v, part[q]);
        }
    }

    template <int PARTS>
    __device__ __forceinline__ void write(const Bf16x8 (&part)[kN][3],
                                          short* buf) const
    {
#pragma unroll
        for (int q = 0; q < kN; ++q)
#pragma unroll
            for (int s = 0; s < PARTS; ++s)
                *(Bf16x8*)(buf + s * R * kStep32 + lds[q]) = part[q][s];
    }

    // The last, partial step: `summed` summed values from k0 on, the others
    // zeros, straight to LDS.
    template <int PARTS>
    __device__ __forceinline__ void tail(const Factor& f, int64_t x0, int64_t n,
                                         int64_t k0, int summed, short* buf)
    {
#pragma unroll
        for (int q = 0; q < kN; ++q) {
            const int c = q * T + (int)threadIdx.x;
            const int across = ALONG ? 4 : R / 8;
            const int row = c / across, piece = c % across;
            Eight<SVM_F32> x;
            Bf16x8 part[3];
            if (ALONG)
                x.load(f.data, (x0 + row) * f.ld + k0 + piece * 8,
                       x0 + row < n ? eight_of(summed, piece * 8) : 0);
            else
                x.load(f.data, (k0 + row) * f.ld + x0 + piece * 8,
                       row < summed ? eight_of(n, x0 + piece * 8) : 0);
            three_parts(x.v, part);
#pragma unroll
            for (int s = 0; s < PARTS; ++s)
                *(Bf16x8*)(buf + s * R * kStep32 + lds[q]) = part[s];
        }
    }
};

// 32-bit factors, each in three bf16 parts h, m, l: of the nine products of
// parts the six that reach 2^-24 of the whole.  All six come from one reading
// of the parts' fragments, so that here LDS is read half as much for each
// matrix instruction as with 16-bit factors.  A step (32 summed values):
//   h and h' are in registers; read m and m', multiply h h';  read l and l',
//   split the values that have come for the step after next, multiply h m',
//   m h', m m';  meet the other waves, write those to the buffer that this
//   step has left, load the values of the step after those, read the next h
//   and h', multiply h l', l h'.
// (Values two or four steps ahead made no step shorter, at any tile.)
// Six bf16 products for one: at 1270 TFLOP/s they alone would take 759 us for
// 50000 x 2048 over 784; with cosines of the sums it takes 956 to 975 (168
// TFLOP/s of the 32-bit product), a library's 32-bit product 1043 with no cosine.
// The matrix cores are at work in 43 % of the cycles; the splitting (vector
// instructions) and the LDS traffic of three parts take the rest.
// NARROW: B's values are those of bf16, so that h' is all of them: three
// products, of which each reads a part of A's.  Unpacked 4-bit weights: 5000 x
// 2048 over 784 97 us, with the six 138; 16384 x 2048 over 2048 373 and 645.
template <int BM, int BN, int WGM, int WGN, bool AALONG, bool BALONG,
          bool NARROW>
__global__ __launch_bounds__(64 * WGM * WGN) void k_product32(Args p)
{
    constexpr int NW = WGM * WGN, T = 64 * NW;
    constexpr int FM = BM / WGM / 16, FN = BN / WGN / 16;
    constexpr int kBK = kStep32, kSlab = slab_rows(FM) * FN * 16;
    constexpr int kB = 3 * BM * kBK;            // where B's planes begin
    constexpr int kParts = NARROW ? 1 : 3;      // of B
    constexpr int kPlanes = (3 * BM + kParts * BN) * kBK;
    constexpr int kOut = NW / 2 * kSlab * 2;
    constexpr int kLds = kPlanes > kOut ? kPlanes : kOut;  // of a buffer
    __shared__ __align__(1024) short lds0[kLds];
    __shared__ __align__(1024) short lds1[kLds];

    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    unsigned ti, tj;
    tile_of(blockIdx.x, p.tm, p.tn, ti, tj);
    const int64_t i0 = (int64_t)ti * BM, j0 = (int64_t)tj * BN;
    const int wi = wave / WGN * (BM / WGM), wj = wave % WGN * (BN / WGN);

    Frag<BM, kBK, AALONG> fa;
    Frag<BN, kBK, BALONG> fb;
    fa.init(wi, lane);
    fb.init(wj, lane);
    // whole steps t0 .. t1 - 1; a last one that is not whole comes apart
    const int t0 = blockIdx.y * p.per;
    const int whole = (int)(p.k / kBK);
    const int t1 = t0 + p.per < whole ? t0 + p.per : whole;
    using SA = Split<BM, T, AALONG>;
    using SB = Split<BN, T, BALONG>;
    SA sa;
    SB sb;
    sa.init(p.A, i0, p.m, t0, p.k);
    sb.init(p.B, j0, p.n, t0, p.k);
    typename SA::Raw ra;
    typename SB::Raw rb;
    Bf16x8 pa[SA::kN][3], pb[SB::kN][3];
    int tl = t0;  // step of the next loads
    auto load = [&]() {
        sa.load(ra, tl < t1);
        sb.load(rb, tl < t1);
        ++tl;
    };
    auto split = [&]() {
        SA::split(ra, pa);
        SB::split(rb, pb);
    };
    auto write = [&](short* lds) {
        sa.template write<3>(pa, lds);
        sb.template write<kParts>(pb, lds + kB);
    };

    floatx4 acc[FM][FN];
#pragma unroll
    for (int f = 0; f < FM; ++f)
#pragma unroll
        for (int g = 0; g < FN; ++g) acc[f][g] = floatx4{0, 0, 0, 0};

    short8v ah[FM], bh[FN], am[FM], bm[FN], al[FM], bl[FN], an[FM], bn[FN];
    auto frags = [&](const short* lds, int plane, short8v* a, short8v* b) {
        if (plane < kParts) {
#pragma unroll
            for (int g = 0; g < FN; ++g)
                b[g] = fb.read(lds + kB + plane * BN * kBK, wj, g, 0, lane);
        }
#pragma unroll
        for (int f = 0; f < FM; ++f)
            a[f] = fa.read(lds + plane * BM * kBK, wi, f, 0, lane);
    };
    auto multiply = [&](const short8v* a, const short8v* b) {
#pragma unroll
        for (int f = 0; f < FM; ++f)
#pragma unroll
            for (int g = 0; g < FN; ++g)
                acc[f][g] = mfma<SVM_BF16>(b[g], a[f], acc[f][g]);
    };
    constexpr int kReads = (AALONG ? FM : 2 * FM) + (BALONG ? FN : 2 * FN);
    constexpr int kMul = FM * FN;
    // reads, and with `valu` other arithmetic, between n matrix instructions
    auto spread = [&](int n, int valu) {
#pragma unroll
        for (int r = 0; r < n; ++r) {
            if (r < kReads) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (valu) __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
        }
    };
    // ah, bh: this step's first parts, an, bn: where the next one's go
    auto step = [&](short* cur, short* oth, short8v* ah, short8v* bh,
                    short8v* an, short8v* bn) {
        __builtin_amdgcn_sched_barrier(0);
        frags(cur, 1, am, bm);
        multiply(ah, bh);
        spread(kMul, 0);
        __builtin_amdgcn_sched_barrier(0);
        frags(cur, 2, al, bl);
        split();
        if constexpr (!NARROW) {
            multiply(ah, bm);
            multiply(am, bh);
            multiply(am, bm);
            spread(3 * kMul, 1);
        } else {
            multiply(am, bh);
            spread(kMul, 1);
        }
        meet<63>();
        write(cur);
        load();
        __builtin_amdgcn_sched_barrier(0);
        frags(oth, 0, an, bn);
        if constexpr (!NARROW) multiply(ah, bl);
        multiply(al, bh);
        spread((NARROW ? 1 : 2) * kMul, 0);
        __builtin_amdgcn_sched_barrier(0);
    };

    load();
    split();
    write(lds0);
    load();
    split();
    write(lds1);
    load();
    meet<63>();
    frags(lds0, 0, ah, bh);
    for (int t = t0; t < t1; t += 2) {
        step(lds0, lds1, ah, bh, an, bn);
        if (t + 1 < t1) step(lds1, lds0, an, bn, ah, bh);
    }
    if (t0 + p.per > whole && p.k % kBK) {
        const int64_t k0 = (int64_t)whole * kBK;
        const int summed = (int)(p.k - k0);
        meet<63>();
        sa.template tail<3>(p.A, i0, p.m, k0, summed, lds0);
        sb.template tail<kParts>(p.B, j0, p.n, k0, summed, lds0 + kB);
        meet<63>();
        frags(lds0, 0, ah, bh);
        frags(lds0, 1, am, bm);
        frags(lds0, 2, al, bl);
        if constexpr (!NARROW) multiply(ah, bl);
        multiply(al, bh);
        if constexpr (!NARROW) {
            multiply(am, bm);
            multiply(ah, bm);
        }
        multiply(am, bh);
        multiply(ah, bh);
    }
    const int64_t end = (int64_t)(t0 + p.per) * kBK;
    mend_tile<FM, FN, AALONG, BALONG>(p, acc, i0 + wi, j0 + wj,
                                      (int64_t)t0 * kBK, end < p.k ? end : p.k,
                                      lane);
    meet<63>();
    write_tile<SVM_F32, FM, FN>(p, acc,
                                wave_slab<kSlab, NW, kLds>(lds0, lds1, wave),
                                i0 + wi, j0 + wj, lane);
}

// Sums the parts of a split product and finishes it, eight columns a thread.
// Bound by memory, and for the sizes that are split by the launch (4 us).
template <int OT>
__global__ __launch_bounds__(256) void k_join(Args p)
{
    const int64_t groups = (p.n + 7) / 8;
    const int64_t all = p.m * groups;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < all;
         t += (int64_t)gridDim.x * 256) {
        const int64_t i = quotient(t, groups, all);
        const int64_t j = (t - i * groups) * 8;
        const int count = eight_of(p.n, j);
        Eight<OT> x, bias;
        RawEight<OT> res;
#pragma unroll
        for (int c = 0; c < 8; ++c) x.v[c] = bias.v[c] = 0.0f;
#pragma unroll 4
        for (int s = 0; s < p.splits; ++s) {
            Eight<SVM_F32> y;
            y.load(p.part, ((int64_t)s * p.m + i) * p.n + j, count);
#pragma unroll
            for (int c = 0; c < 8; ++c) x.v[c] += y.v[c];
        }
        if (p.e.bias) bias.load(p.e.bias, j, count);
        if (p.e.residual) res.load(p.e.residual, i * p.e.ldr + j, count);
        finish<OT>(p.e, x, bias, res, i, j, count);
    }
}

// ---- few rows

// Y for at most 16 MT rows of X: 16 columns (rows of W) to a block, the
// summed index split over its waves and the waves' sums joined in LDS.  Rows
// of W go from memory to registers, in 32 bytes a lane (128 of a row at
// once), with no LDS between: each is used once, and W is all that counts.
// Rows may begin anywhere, and 32-bit values are split in registers.
// Bound by the read of W where W is large, by latency where it is not: 1 x
// 1024 over 784 in bf16 takes 6.1 us (11.5 with the call around it, in 32 bits
// too); 1 x 4096 over 4096 a call of 11.5 us in bf16, 23.2 in 32 bits.
constexpr int kFewWaves = 8;

struct FewArgs {
    const void *X, *W;
    int64_t ldx, ldw, m, n, k;
    Epilogue e;
};

// 16 values of a row as they lie in memory, and as two fragments (for 32 bits
// two of each part).
template <int DT>
struct Sixteen {
    RawEight<DT> raw[2];
    short8v h[2], m[2], l[2];

    __device__ __forceinline__ void load(const void* p, int64_t at, int64_t left)
    {
#pragma unroll
        for (int u = 0; u < 2; ++u)
            raw[u].load(p, at + u * 8, eight_of(left, u * 8));
    }

    __device__ __forceinline__ void split()
    {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            if constexpr (DT == SVM_F32) {
                float v[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = raw[u].at(e);
                Bf16x8 part[3];
                three_parts(v, part);
                h[u] = __builtin_bit_cast(short8v, part[0]);
                m[u] = __builtin_bit_cast(short8v, part[1]);
                l[u] = __builtin_bit_cast(short8v, part[2]);
            } else {
                h[u] = __builtin_bit_cast(short8v, raw[u].v[0]);
            }
        }
    }
};

template <int DT, int MT>
__global__ __launch_bounds__(64 * kFewWaves) void k_few(FewArgs p)
{
    __shared__ float red[kFewWaves][MT * 16][20];  // (rows 16 apart in banks)
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int i = lane & 15, g = lane >> 4;
    const int64_t j0 = (int64_t)blockIdx.x * 16;
    constexpr int IT = DT == SVM_F32 ? SVM_BF16 : DT;
    floatx4 acc[MT];
#pragma unroll
    for (int t = 0; t < MT; ++t) acc[t] = floatx4{0, 0, 0, 0};
    // past W's or X's rows, and past the summed index, nothing is loaded
    const int64_t wrow = j0 + i < p.n ? (j0 + i) * p.ldw : -1;
    Sixteen<DT> w, x[MT];
    auto fetch = [&](int64_t k0) {
        const int64_t at = k0 + g * 16;
        w.load(p.W, wrow + at, wrow < 0 ? 0 : p.k - at);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            const int64_t r = t * 16 + i;
            x[t].load(p.X, r * p.ldx + at, r < p.m ? p.k - at : 0);
        }
    };
    fetch(wave * 64);
    for (int64_t k0 = wave * 64; k0 < p.k; k0 += 64 * kFewWaves) {
        w.split();
#pragma unroll
        for (int t = 0; t < MT; ++t) x[t].split();
        fetch(k0 + 64 * kFewWaves);
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                if constexpr (DT == SVM_F32) {  // the smallest first
                    acc[t] = mfma<IT>(w.h[u], x[t].l[u], acc[t]);
                    acc[t] = mfma<IT>(w.l[u], x[t].h[u], acc[t]);
                    acc[t] = mfma<IT>(w.m[u], x[t].m[u], acc[t]);
                    acc[t] = mfma<IT>(w.h[u], x[t].m[u], acc[t]);
                    acc[t] = mfma<IT>(w.m[u], x[t].h[u], acc[t]);
                }
                acc[t] = mfma<IT>(w.h[u], x[t].h[u], acc[t]);
            }
    }
    if constexpr (DT == SVM_F32) {  // the wave's sums that are not finite
        const Rows16<true> wr(p.W, p.ldw, j0, p.n, lane);
#pragma unroll
        for (int t = 0; t < MT; ++t) {
            bool any = false;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                any |= !is_finite(acc[t][e]) && j0 + g * 4 + e < p.n;
            if (!__ballot(any && t * 16 + i < p.m)) continue;
            const floatx4 sum =
                sums_32(Rows16<true>(p.X, p.ldx, t * 16, p.m, lane), wr,
                        wave * 64, p.k, 64 * kFewWaves, lane);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (!is_finite(acc[t][e])) acc[t][e] = sum[e];
        }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t)
        *(floatx4*)&red[wave][t * 16 + i][g * 4] = acc[t];
    __syncthreads();
    if (threadIdx.x >= MT * 32) return;
    const int row = threadIdx.x >> 1, c0 = (threadIdx.x & 1) * 8;
    const int64_t j = j0 + c0;
    const int count = eight_of(p.n, j);
    if (row >= p.m || count == 0) return;
    Eight<DT> v, bias;
    RawEight<DT> res;
#pragma unroll
    for (int c = 0; c < 8; ++c) v.v[c] = bias.v[c] = 0.0f;
    if (p.e.bias) bias.load(p.e.bias, j, count);
    if (p.e.residual) res.load(p.e.residual, row * p.e.ldr + j, count);
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w)
#pragma unroll
        for (int c = 0; c < 8; ++c) v.v[c] += red[w][row][c0 + c];
    finish<DT>(p.e, v, bias, res, row, j, count);
}

// ---- factors that cannot be read as they are

template <int DT>
__global__ __launch_bounds__(256) void k_padded(const Elem<DT>* X, int64_t ld,
                                                int64_t rows, int64_t cols,
                                                Elem<DT>* dst, int64_t ldp)
{
    const int64_t groups = ldp / 8, all = rows * groups;
    for (int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x; t < all;
         t += (int64_t)gridDim.x * 256) {
        const int64_t i = quotient(t, groups, all);
        const int64_t j = (t - i * groups) * 8;
        Eight<DT> x;
        x.load(X, i * ld + j, eight_of(cols, j));
        x.store(dst, i * ldp + j, 8);
    }
}

// launch(AALONG, BALONG) for the ways that the factors of a product lie.
template <class F>
void for_factors(const Args& a, F&& launch)
{
    if (a.A.along && a.B.along) launch.template operator()<true, true>();
    else if (a.A.along) launch.template operator()<true, false>();
    else launch.template operator()<false, false>();
}

// WGX: waves across a tile where both factors lie across the summed index.
template <int OT, int BM, int BN, int WGM, int WGN, int WGX, int ST>
void launch16(const Args& a, hipStream_t s)
{
    for_factors(a, [&]<bool AALONG, bool BALONG>() {
        constexpr int kWgn = AALONG || BALONG ? WGN : WGX;
        hipLaunchKernelGGL(
            (k_product<OT, BM, BN, WGM, kWgn, ST, AALONG, BALONG>),
            dim3(a.tm * a.tn, (unsigned)a.splits), dim3(64 * WGM * kWgn), 0, s,
            a);
    });
}

template <int BM, int BN, int WGM, int WGN>
void launch32(const Args& a, bool narrow, hipStream_t s)
{
    if (narrow) {
        hipLaunchKernelGGL((k_product32<BM, BN, WGM, WGN, true, true, true>),
                           dim3(a.tm * a.tn, (unsigned)a.splits),
                           dim3(64 * WGM * WGN), 0, s, a);
        return;
    }
    for_factors(a, [&]<bool AALONG, bool BALONG>() {
        hipLaunchKernelGGL((k_product32<BM, BN, WGM, WGN, AALONG, BALONG,
                                        false>),
                           dim3(a.tm * a.tn, (unsigned)a.splits),
                           dim3(64 * WGM * WGN), 0, s, a);
    });
}

template <int OT>
void launch_product(const Args& a, int tile, bool narrow, hipStream_t s)
{
    if constexpr (OT == SVM_F32) {
        if (tile == 256) launch32<128, 256, 2, 4>(a, narrow, s);
        else if (tile == 128) launch32<128, 128, 2, 4>(a, narrow, s);
        else launch32<64, 64, 2, 2>(a, narrow, s);
    } else {
        // Tiles of 128: eight waves, two to a SIMD, each of which waits while
        // the other multiplies (4096 x 1024 over 1024: 15.0 us, with four
        // waves 16.3); where both factors lie across, the reads of eight
        // waves' fragments cost more than that gains (2048 x 2048 over 8192:
        // 92 us with eight, 87 with four).
        if (tile == 256) launch16<OT, 256, 256, 2, 4, 4, 2>(a, s);
        else if (tile == 128) launch16<OT, 128, 128, 2, 4, 2, 4>(a, s);
        else launch16<OT, 64, 64, 2, 2, 2, 4>(a, s);
    }
}

constexpr int kCus = 256;

}  // namespace

bool factor_fits(const svm_array& a, bool along)
{
    return a.ld <= kMaxWidth &&
           (a.dtype == SVM_F32 ||
            (((uintptr_t)a.data & 15) == 0 && a.ld % 8 == 0 &&
             (!along || a.cols % 8 == 0)));
}

void launch_padded(const svm_array& a, void* dst, int64_t ldp, hipStream_t s)
{
    const int64_t all = a.rows * (ldp / 8);
    if (all == 0) return;
    const int64_t nb = (all + 255) / 256;
    const dim3 grid((unsigned)(nb < 16384 ? nb : 16384)), block(256);
    for_dtype(a.dtype, [&]<int DT>() {
        hipLaunchKernelGGL((k_padded<DT>), grid, block, 0, s,
                           (const Elem<DT>*)a.data, a.ld, a.rows, a.cols,
                           (Elem<DT>*)dst, ldp);
    });
}

bool few_rows(int64_t m, int64_t n, int64_t k)
{
    return m <= 32 && (k <= 32768 || n >= 4096);
}

void few_rows_product(const svm_array& X, const svm_array& W,
                      const Epilogue& e, hipStream_t s)
{
    const FewArgs a{X.data, W.data, X.ld, W.ld, X.rows, W.rows, X.cols, e};
    const dim3 grid((unsigned)((a.n + 15) / 16)), block(64 * kFewWaves);
    for_dtype(X.dtype, [&]<int DT>() {
        if (a.m <= 16)
            hipLaunchKernelGGL((k_few<DT, 1>), grid, block, 0, s, a);
        else
            hipLaunchKernelGGL((k_few<DT, 2>), grid, block, 0, s, a);
    });
}

namespace {

// What a block of a tile costs, measured on this card in us: a step with one
// block to a CU, what each block more adds to a step (those that run at once
// share the matrix cores; large tiles run one after another), and the rest of
// a block (first loads, last writes).
struct TileCost {
    int tile, bm;  // columns; rows
    double one, more, rest;
};
constexpr TileCost kCost16[3] = {{256, 256, 1.65, 1.65, 5.0},
                                 {128, 128, 0.57, 0.57, 4.0},
                                 {64, 64, 0.26, 0.23, 1.5}};
// (Those in 32 bits are of six matrix products.  Narrow factors take three in
// the tile that is best with six: 16384 x 2048 over 2048 373 us in the largest,
// 487 and 599 in the others; 4000 x 1000 over 500 29.2 in tiles of 128 columns,
// 36 in either other; but 5000 x 2048 over 784 97 in tiles of 128, 92.5 in the
// largest, and 1100 x 130 over 20000 64 in tiles of 64, 53 in the largest.)
constexpr TileCost kCost32[3] = {{256, 128, 2.50, 2.50, 10.0},
                                 {128, 128, 1.45, 1.42, 7.0},
                                 {64, 64, 0.65, 0.48, 2.0}};

struct Choice {
    const TileCost* t;
    int64_t splits;
};

// The tile and the number of parts of the summed index that cost least: of a
// product with many tiles the largest, whose factors are read least; of one
// with few, smaller tiles or parts of the summed index keep all CUs at work
// (8192 x 2048 over 2048, bf16: 61 us in tiles of 256, 65 in tiles of 128;
// 2048 x 2048 over 8192 in 32 bits: 335 us in two parts, 408 in smaller
// tiles; 6656 x 209 over 2347: 66 us in four parts, 76 in smaller tiles).
// Parts cost a launch more (8 us with the host's share: 476 x 64 over 2304,
// bf16, takes 14.6 us whole and 19.0 in nine parts), and their sums are
// written and read once (5000 x 1000 over 5000, bf16: 72 us in three parts of
// tiles of 256; over 97 whole, in tiles of 64 or 128).
Choice choose(const Product& p, int nk)
{
    const TileCost* table = p.dtype == SVM_F32 ? kCost32 : kCost16;
    Choice best{table, 1};
    double least = 1e300;
    for (int q = 0; q < 3; ++q) {
        const TileCost& t = table[q];
        const double nt = (double)((p.m + t.bm - 1) / t.bm) *
                          (double)((p.n + t.tile - 1) / t.tile);
        for (int64_t s = 1; s <= 64 && (s == 1 || 2 * s <= nk);
             s += s < 4 ? 1 : s / 2) {
            const double blocks = std::ceil(nt * (double)s / kCus);
            const double step =
                std::max(blocks * t.more, t.one + (blocks - 1) * 0.5 * t.more);
            double us = (double)((nk + s - 1) / s) * step + blocks * t.rest;
            if (s > 1)
                us += 8.0 + (double)s * (double)p.m * (double)p.n * 8 / 5e6;
            if (us < least) {
                least = us;
                best = {&t, s};
            }
        }
    }
    return best;
}

}  // namespace

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
    const bool f32 = p.dtype == SVM_F32;
    const int bk = f32 ? kStep32 : kStep16;
    a.nk = (int)((p.k + bk - 1) / bk);
    const Choice c = choose(p, a.nk);
    const int tile = c.t->tile, bm = c.t->bm;
    a.per = (int)((a.nk + c.splits - 1) / c.splits);
    a.splits = (a.nk + a.per - 1) / a.per;
    a.tn = (unsigned)((p.n + tile - 1) / tile);
    if (a.splits > 1) a.part = ws.take<float>(a.splits * p.m * p.n);
    if (!ws.run) return;
    // A launch has fewer than 2^32 threads: rows in slices of at most 2^22
    // tiles (more than one slice of them is never split).
    const int64_t slice = std::max<int64_t>((1 << 22) / a.tn, 1) * bm;
    for (int64_t i0 = 0; i0 < p.m; i0 += slice) {
        Args q = a;
        const int64_t eb = (int64_t)dtype_bytes(p.dtype);
        q.m = std::min(p.m - i0, slice);
        q.tm = (unsigned)((q.m + bm - 1) / bm);
        auto on = [&](const void* x, int64_t ld) {
            return x ? (const char*)x + i0 * ld * eb : nullptr;
        };
        q.A.data = on(a.A.data, a.A.along ? a.A.ld : 1);
        q.e.Y = (void*)on(a.e.Y, a.e.ldy);
        q.e.Z = (void*)on(a.e.Z, a.e.ldz);
        q.e.residual = on(a.e.residual, a.e.ldr);
        if (f32) launch_product<SVM_F32>(q, tile, p.narrow, s);
        else if (p.dtype == SVM_BF16)
            launch_product<SVM_BF16>(q, tile, false, s);
        else launch_product<SVM_F16>(q, tile, false, s);
    }
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
