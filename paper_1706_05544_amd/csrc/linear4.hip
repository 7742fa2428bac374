// Weights in 4 bits with a scale to each group of inputs, and the linear layer
// on them.
//
// A code is a sign and three bits of magnitude, 0 0.5 1 1.5 2 3 4 6: the 4-bit
// floats that this card turns into two 16-bit ones in one instruction.  They
// are exact in either 16-bit type, so they go through the matrix instructions
// as they are and each group's sum is multiplied by the group's scale in 32
// bits: no weight is rounded on the way.
//
// Memory layout: tiles of 16 outputs by 128 inputs, 1024 bytes each, the
// tiles of 16 outputs one after another along the inputs.  Lane l of the
// matrix instruction holds 8 consecutive inputs (l / 16) of output l % 16 in
// each of the tile's four steps of 32 inputs: its four steps lie side by side,
// 16 bytes.  Behind the codes the scales, in the same order of tiles: for each
// of 16 outputs those of its groups in the tile (4, 2 or 1) side by side.
#include "elem.hpp"
#include "matmul.hpp"

namespace msvm {

namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));
typedef uint32_t uint4v __attribute__((ext_vector_type(4)));
typedef short short8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));

constexpr float kMost = 3.402823466e38f;

// The scale of a group whose largest magnitude is `top`: a sixth of it (the
// product with the 32-bit number nearest to 1/6) with six significant bits
// kept, so that a scale times a code (two significant bits) is a value of any
// of the types.  In f16 it is a whole number of steps of 2^-23 besides: half
// of it is a value too.
template <int DT>
__device__ __forceinline__ float scale_of(float top)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, top * (1.0f / 6.0f));
    const float s = __builtin_bit_cast(float, b & ~((1u << 18) - 1));
    if constexpr (DT == SVM_F16)
        return floorf(s * 8388608.0f) * (1.0f / 8388608.0f);
    return s;
}

// The code of w: the nearest magnitude, a value on a border the even code.
__device__ __forceinline__ uint32_t code_of(float w, float s)
{
    if (!(s > 0.0f)) return w < 0.0f ? 8u : 0u;
    const float x = fabsf(w) / s;
    uint32_t c = x > 0.25f;
    c += x >= 0.75f;
    c += x > 1.25f;
    c += x >= 1.75f;
    c += x > 2.5f;
    c += x >= 3.5f;
    c += x > 5.0f;
    return c | (w < 0.0f ? 8u : 0u);
}

struct PackArgs {
    const void* W;
    int64_t ldw, n, k, chunks, all;
    unsigned char* codes;
    void* scales;
};

// A wave to a tile: a group's 32 inputs are the four lanes of an output in one
// step, so its largest magnitude takes two exchanges.  Rounding is done once,
// when weights are laid out; bound by its division and comparisons: 67 million
// f16 weights 63 to 70 us, 2.4 TB/s and more.
template <int DT, int GROUP>
__global__ __launch_bounds__(256) void k_pack4(PackArgs p)
{
    using T = Elem<DT>;
    constexpr int kSteps = GROUP / 32, kGroups = 4 / kSteps;
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    for (int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); w < p.all;
         w += (int64_t)gridDim.x * 4) {
        const int64_t tile = w / p.chunks, c = w - tile * p.chunks;
        const int64_t row = tile * 16 + r;
        Eight<DT> x[4];
        float top[4];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int64_t at = c * 128 + s * 32 + g * 8;
            x[s].load(p.W, row * p.ldw + at,
                      row < p.n ? eight_of(p.k, at) : 0);
            top[s] = 0.0f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float a = fabsf(x[s].v[e]);
                top[s] = fmaxf(top[s], a <= kMost ? a : __builtin_inff());
            }
            top[s] = fmaxf(top[s], __shfl_xor(top[s], 16));
            top[s] = fmaxf(top[s], __shfl_xor(top[s], 32));
        }
        uint4v out;
#pragma unroll
        for (int q = 0; q < kGroups; ++q) {
            float t = 0.0f;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) t = fmaxf(t, top[q * kSteps + s]);
            // a weight that is not finite shows in all of its group
            const bool bad = !(t <= kMost);
            const float sc = bad ? __builtin_nanf("") : scale_of<DT>(t);
            if (g == 0)
                ((T*)p.scales)[(w * 16 + r) * kGroups + q] = (T)sc;
#pragma unroll
            for (int s = 0; s < kSteps; ++s) {
                uint32_t d = 0;
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    d |= (bad ? 0u : code_of(x[q * kSteps + s].v[e], sc))
                         << (4 * e);
                out[q * kSteps + s] = d;
            }
        }
        *(uint4v*)(p.codes + w * 1024 + lane * 16) = out;
    }
}

// Two codes (byte SEL of d) as 32-bit values, 16-bit ones.
template <int SEL>
__device__ __forceinline__ floatx2 two32(uint32_t d)
{
    return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(d, 1.0f, SEL);
}

// ... times `by`, a power of two, as 16-bit ones.
template <int DT>
__device__ __forceinline__ short8v eight16(uint32_t d, float by)
{
    if constexpr (DT == SVM_F16) {
        half2v v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, by, 0),
                       __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, by, 1),
                       __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, by, 2),
                       __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, by, 3)};
        return __builtin_bit_cast(short8v, v);
    } else {
        bf16x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d, by, 0),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d, by, 1),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d, by, 2),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d, by, 3)};
        return __builtin_bit_cast(short8v, v);
    }
}

struct UnpackArgs {
    const unsigned char* codes;
    const void* scales;
    int64_t n, k, chunks, all;
    int gshift;
    void* W;
    int64_t ldw;
};

// A wave to a tile.  Exact: scale times code is a value of the type.  Bound by
// memory: 67 million f16 weights 32.2 us, 5.3 TB/s; 1.6 million to 32 bits 4.5
// us, of which a launch is 2.
template <int DT>
__global__ __launch_bounds__(256) void k_unpack4(UnpackArgs p)
{
    using T = Elem<DT>;
    const int lane = threadIdx.x & 63, r = lane & 15, g = lane >> 4;
    for (int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6); w < p.all;
         w += (int64_t)gridDim.x * 4) {
        const int64_t tile = w / p.chunks, c = w - tile * p.chunks;
        const int64_t row = tile * 16 + r;
        const uint4v d = *(const uint4v*)(p.codes + w * 1024 + lane * 16);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const int64_t at = c * 128 + s * 32 + g * 8;
            const float sc = (float)((const T*)p.scales)[
                ((w * 16 + r) << (7 - p.gshift)) + ((s * 32) >> p.gshift)];
            const floatx2 v0 = two32<0>(d[s]), v1 = two32<1>(d[s]),
                          v2 = two32<2>(d[s]), v3 = two32<3>(d[s]);
            Eight<DT> x;
            x.v[0] = v0[0] * sc, x.v[1] = v0[1] * sc;
            x.v[2] = v1[0] * sc, x.v[3] = v1[1] * sc;
            x.v[4] = v2[0] * sc, x.v[5] = v2[1] * sc;
            x.v[6] = v3[0] * sc, x.v[7] = v3[1] * sc;
            if (row < p.n)
                x.store(p.W, row * p.ldw + at, eight_of(p.k, at));
        }
    }
}

template <int DT>
__device__ __forceinline__ floatx4 mfma32(short8v a, short8v b, floatx4 c)
{
    if constexpr (DT == SVM_F16) {
        typedef _Float16 V __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(
            __builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
    } else {
        typedef __bf16 V __attribute__((ext_vector_type(8)));
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            __builtin_bit_cast(V, a), __builtin_bit_cast(V, b), c, 0, 0, 0);
    }
}

// Eight values of X as factors of the matrix instructions: one for 16-bit
// types, three bf16 parts for 32 bits, each what is left cut to the eight bits
// of a bf16 (8 + 8 + 8 bits: all of them, from 2^-109 on).  An infinity is
// the first part alone.
template <int DT>
struct Factor8 {
    static constexpr int kParts = DT == SVM_F32 ? 3 : 1;
    short8v v[kParts];

    __device__ __forceinline__ void from(const RawEight<DT>& x)
    {
        if constexpr (DT != SVM_F32) {
            v[0] = __builtin_bit_cast(short8v, x.v[0]);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float f = x.at(e);
                const uint32_t b = __builtin_bit_cast(uint32_t, f);
                v[0][e] = (short)(b >> 16);
                float r = f - __builtin_bit_cast(float, b & 0xffff0000u);
                if (fabsf(f) == __builtin_inff()) r = 0.0f;
                const uint32_t m = __builtin_bit_cast(uint32_t, r);
                v[1][e] = (short)(m >> 16);
                r -= __builtin_bit_cast(float, m & 0xffff0000u);
                v[2][e] = (short)(__builtin_bit_cast(uint32_t, r) >> 16);
            }
        }
    }
};

constexpr int kWaves = 8;  // of a block

struct Linear4Args {
    const void* X;
    const unsigned char* codes;
    const void* scales;
    int64_t ldx, m, n, k, chunks;
    Epilogue e;
};

// What a lane has of a chunk of 128 inputs: codes and scales of NT tiles of
// outputs, and its row's inputs.
template <int DT, int NT, int GPC>
struct Stage {
    using T = Elem<DT>;
    typedef T Scales __attribute__((ext_vector_type(GPC)));
    uint4v code[NT];
    Scales scale[NT];
    RawEight<DT> x[4];

    // t, row: the lane's tiles and where its row begins (beyond the last tile
    // and row the last again, whose sums are not used)
    __device__ __forceinline__ void load(const Linear4Args& p,
                                         const int64_t (&t)[NT], int64_t row,
                                         int64_t c, int lane)
    {
        const int i = lane & 15, g = lane >> 4;
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            const int64_t w = t[b] * p.chunks + c;
            code[b] = *(const uint4v*)(p.codes + w * 1024 + lane * 16);
            scale[b] = ((const Scales*)p.scales)[w * 16 + i];
        }
        if (c * 128 + 128 <= p.k) {
#pragma unroll
            for (int s = 0; s < 4; ++s)
                x[s].load(p.X, row + c * 128 + s * 32 + g * 8, 8);
        } else {
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int64_t at = c * 128 + s * 32 + g * 8;
                x[s].load(p.X, row + at, eight_of(p.k, at));
            }
        }
    }

    // acc += this chunk's products, times `by`.  A group's are added up by the
    // matrix instruction and multiplied by its scale once.
    template <int REGS>
    __device__ __forceinline__ void add(float (&acc)[NT][REGS],
                                        float by = 1.0f) const
    {
        constexpr int kSteps = 4 / GPC;
#pragma unroll
        for (int q = 0; q < GPC; ++q) {
            floatx4 part[NT];
#pragma unroll
            for (int b = 0; b < NT; ++b) part[b] = floatx4{0, 0, 0, 0};
#pragma unroll
            for (int s = q * kSteps; s < (q + 1) * kSteps; ++s) {
                short8v w[NT];
#pragma unroll
                for (int b = 0; b < NT; ++b) w[b] = eight16<DT>(code[b][s], by);
                Factor8<DT> f;
                f.from(x[s]);
#pragma unroll
                for (int r = Factor8<DT>::kParts - 1; r >= 0; --r)
#pragma unroll
                    for (int b = 0; b < NT; ++b)
                        part[b] = mfma32<DT>(f.v[r], w[b], part[b]);
            }
#pragma unroll
            for (int b = 0; b < NT; ++b)
#pragma unroll
                for (int v = 0; v < REGS; ++v)
                    acc[b][v] =
                        fmaf(part[b][v], (float)scale[b][q], acc[b][v]);
        }
    }
};

// A group's sum of inputs times codes may leave 32 bits where its scale would
// bring it back (from |X| = 4e35 on; in f16 never).  A wave with a sum that is
// not finite forms a tile's sums again, of codes times kDown, and puts them in
// the place of those that were not.  Seldom: a tile and a chunk at a time, and
// nothing of it is made ahead, so that it takes no registers from the rest.
constexpr float kDown = 1.0f / 4096.0f;

template <int DT, int GPC, bool FEW>
__device__ __forceinline__ void sums_again(const Linear4Args& p, int64_t tile,
                                           int64_t row, int wave, float* red,
                                           int pad)
{
    constexpr int kRegs = FEW ? 1 : 4;
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    float acc[1][kRegs] = {};
    const int64_t t[1] = {tile};
#pragma clang loop unroll(disable)
    for (int64_t c = wave; c < p.chunks; c += kWaves) {
        Stage<DT, 1, GPC> now;
        now.load(p, t, row, c, lane);
        now.template add<kRegs>(acc, kDown);
    }
    const int i = lane & 15, g = lane >> 4;
#pragma unroll
    for (int v = 0; v < kRegs; ++v) {
        float& sum = red[(FEW ? g : g * 4 + v) * pad + i];
        if (!(fabsf(sum) <= kMost)) sum = acc[0][v] * (1.0f / kDown);
    }
}

// Few rows: 16 NT outputs to a block and 16 rows, the inputs in chunks of 128
// taken in turn by its waves, whose sums are joined at the end in a fixed
// order.  The codes come straight from memory to the lane that multiplies
// them, the next chunk's while this one's are used (two chunks ahead, and 4 or
// 16 waves, were slower).
// FEW: up to 4 rows, every fourth of the 16 that the matrix instruction takes,
// so that a lane has one sum to scale and not four.
// Bound by the read of the codes where they are many: 1 x 4096 over 16384 in
// f16 7.3 us in a row of calls, 8.4 by the trace, 4.3 TB/s; by latency where
// they are few: 1 x 784 over 1024 4.4 us, of which an empty launch is 2; and
// for more rows by what is read of X from the caches, again for every 16 NT
// outputs: 32 x 4096 over 4096 in bf16 7.2 us, 128 rows 12.9.
template <int DT, int NT, int GPC, bool FEW>
__global__ __launch_bounds__(64 * kWaves) void k_linear4(Linear4Args p)
{
    constexpr int kCols = NT * 16, kPad = kCols + 4;
    constexpr int kRegs = FEW ? 1 : 4;
    constexpr int kRows = FEW ? 4 : 16;
    __shared__ float red[kWaves][kRows][kPad];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int i = lane & 15, g = lane >> 4;
    const int64_t t0 = (int64_t)blockIdx.x * NT;
    const int64_t r0 = (int64_t)blockIdx.y * 16;
    const int64_t tiles = (p.n + 15) / 16;
    int64_t t[NT];
#pragma unroll
    for (int b = 0; b < NT; ++b) t[b] = t0 + b < tiles ? t0 + b : tiles - 1;
    const int64_t at = FEW ? i >> 2 : r0 + i;
    const int64_t row = (at < p.m ? at : p.m - 1) * p.ldx;
    float acc[NT][kRegs] = {};
    Stage<DT, NT, GPC> next;
    if (wave < p.chunks) next.load(p, t, row, wave, lane);
    for (int64_t c = wave; c < p.chunks; c += kWaves) {
        const Stage<DT, NT, GPC> now = next;
        if (c + kWaves < p.chunks) next.load(p, t, row, c + kWaves, lane);
        now.template add<kRegs>(acc);
    }
    float all = 0.0f;  // NaN where one of them is not finite
#pragma unroll
    for (int b = 0; b < NT; ++b)
#pragma unroll
        for (int v = 0; v < kRegs; ++v) {
            red[wave][FEW ? g : g * 4 + v][b * 16 + i] = acc[b][v];
            all = fmaf(acc[b][v], 0.0f, all);
        }
    if (DT != SVM_F16 && __any(all != 0.0f)) {
#pragma clang loop unroll(disable)
        for (int b = 0; b < NT; ++b)
            sums_again<DT, GPC, FEW>(p, t0 + b < tiles ? t0 + b : tiles - 1,
                                     row, wave, &red[wave][0][b * 16], kPad);
    }
    __syncthreads();
    // a thread to eight outputs
    static_assert(kRows * NT * 2 <= 64 * kWaves, "one turn");
    const int mine = (int)threadIdx.x / (NT * 2);
    const int c0 = (int)threadIdx.x % (NT * 2) * 8;
    const int64_t r = r0 + mine, j = t0 * 16 + c0;
    const int count = mine < kRows && r < p.m ? eight_of(p.n, j) : 0;
    if (count == 0) return;
    Eight<DT> v;
    RawEight<DT> bias, res;
    if (p.e.bias) bias.load(p.e.bias, j, count);
    if (p.e.residual) res.load(p.e.residual, r * p.e.ldr + j, count);
#pragma unroll
    for (int e = 0; e < 8; ++e) v.v[e] = 0.0f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
#pragma unroll
        for (int e = 0; e < 8; ++e) v.v[e] += red[w][mine][c0 + e];
    if (p.e.bias) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v.v[e] += bias.at(e);
    }
    act_values(p.e.act, v.v);
    if (p.e.residual) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v.v[e] += res.at(e);
    }
    v.store(p.e.Y, r * p.e.ldy + j, count);
}

unsigned tile_blocks(int64_t waves)
{
    const int64_t nb = (waves + 3) / 4;
    return (unsigned)(nb < 16384 ? nb : 16384);
}

const void* scales_of(const svm_packed& w)
{
    return (const char*)w.data + Shape4(w).code_bytes;
}

void launch_unpack(const svm_packed& w, int64_t cols, void* to, int64_t ld,
                   hipStream_t s)
{
    const Shape4 sh(w);
    const UnpackArgs a{(const unsigned char*)w.data, scales_of(w), w.rows,
                       cols, sh.chunks, sh.tiles * sh.chunks, sh.gshift, to,
                       ld};
    for_dtype(w.dtype, [&]<int DT>() {
        hipLaunchKernelGGL((k_unpack4<DT>), dim3(tile_blocks(a.all)),
                           dim3(256), 0, s, a);
    });
}

// Whether rows are few enough for k_linear4, whose time grows with them (and
// a block's waves, with few inputs to each, are done sooner): 384 x 4096 over
// 4096 in bf16 takes 33.0 us, unpacked and multiplied 38.2, 512 rows 41.8 and
// 39.1; 1024 x 784 over 1024 takes 10.0 and 12.2, 2048 rows 20 and 16.1; in
// 32 bits 256 x 4096 over 4096 51.7 and 59.0, 384 rows 72.3 and 71.7; 1024 x
// 784 over 1024 21.2 and 23.7, 2048 rows 42 and 29.1.
bool few_rows4(int64_t m, int64_t n, int64_t k)
{
    return m <= (n * k <= 1 << 20 ? 1024 : 384);
}

}  // namespace

void pack4(const svm_array& W, const svm_packed& to, hipStream_t s)
{
    const Shape4 sh(to);
    const PackArgs a{W.data, W.ld, to.rows, to.cols, sh.chunks,
                     sh.tiles * sh.chunks, (unsigned char*)to.data,
                     const_cast<void*>(scales_of(to))};
    const dim3 grid(tile_blocks(a.all)), block(256);
    for_dtype(W.dtype, [&]<int DT>() {
        if (to.group == 32)
            hipLaunchKernelGGL((k_pack4<DT, 32>), grid, block, 0, s, a);
        else if (to.group == 64)
            hipLaunchKernelGGL((k_pack4<DT, 64>), grid, block, 0, s, a);
        else
            hipLaunchKernelGGL((k_pack4<DT, 128>), grid, block, 0, s, a);
    });
}

void unpack4(const svm_packed& w, const svm_array& W, hipStream_t s)
{
    launch_unpack(w, w.cols, W.data, W.ld, s);
}

void linear4(const Linear4Call& a, Pieces& ws, hipStream_t s)
{
    const int64_t m = a.X.rows;
    if (m == 0) return;
    const Epilogue e{a.bias.data, a.residual.data, a.Y.data, nullptr,
                     a.residual.ld, a.Y.ld, 0, a.act};
    const Shape4 sh(a.W);
    if (!few_rows4(m, a.W.rows, a.W.cols)) {
        // many rows: the weights once, as the product kernels take them
        const int64_t ld = (a.W.cols + 7) / 8 * 8;
        void* W = ws.take<char>(a.W.rows * ld * dtype_bytes(a.W.dtype));
        if (ws.run) launch_unpack(a.W, ld, W, ld, s);
        const svm_array w{W, a.W.rows, a.W.cols, ld, a.W.dtype, 1};
        Product p;
        p.m = m;
        p.n = a.W.rows;
        p.k = a.W.cols;
        p.dtype = a.W.dtype;
        p.e = e;
        p.A = factor_of(a.X, true, ws, s);
        p.B = factor_of(w, true, ws, s);
        p.narrow = p.dtype == SVM_F32;
        product(p, ws, s);
        return;
    }
    if (!ws.run) return;
    const Linear4Args k{a.X.data, (const unsigned char*)a.W.data,
                        scales_of(a.W), a.X.ld, m, a.W.rows, a.W.cols,
                        sh.chunks, e};
    for_dtype(a.W.dtype, [&]<int DT>() {
        auto run = [&]<int NT, int GPC, bool FEW>() {
            hipLaunchKernelGGL((k_linear4<DT, NT, GPC, FEW>),
                               dim3((unsigned)((sh.tiles + NT - 1) / NT),
                                    (unsigned)((m + 15) / 16)),
                               dim3(64 * kWaves), 0, s, k);
        };
        auto go = [&]<int NT, bool FEW>() {
            if (a.W.group == 32) run.template operator()<NT, 4, FEW>();
            else if (a.W.group == 64) run.template operator()<NT, 2, FEW>();
            else run.template operator()<NT, 1, FEW>();
        };
        // As many tiles of outputs to a block as leave a block for each CU:
        // they share what is read of X, and in 32 bits its splitting (32 x
        // 4096 over 4096, bf16: 11.2 us with one, 7.6 with two, 8.2 with
        // four; 64 x 4096: 18.8, 11.6 and 8.4; 1 x 4096 over 16384: 9.5 with
        // one, 8.5 with two, 8.6 with four).
        const int64_t all = (m + 15) / 16 * sh.tiles;
        if (m <= 4) {
            if (all >= 512) go.template operator()<2, true>();
            else go.template operator()<1, true>();
        } else if (all >= 1024) {
            go.template operator()<4, false>();
        } else if (all >= 512) {
            go.template operator()<2, false>();
        } else {
            go.template operator()<1, false>();
        }
    });
}

}  // namespace msvm
