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
// 16 bytes.  Behind the codes the scales, 16 outputs side by side, group
// after group.
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

// The scale of a group whose largest magnitude is `top`: a sixth of it with
// six significant bits kept, so that a scale times a code (two significant
// bits) is a value of any of the types.  In f16 it is a whole number of steps
// of 2^-23 besides: half of it is a value too.
template <int DT>
__device__ __forceinline__ float scale_of(float top)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, top / 6.0f);
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
    int64_t ldw, n, k, chunks, groups, all;
    unsigned char* codes;
    void* scales;
};

// A wave to a tile: a group's 32 inputs are the four lanes of an output in one
// step, so its largest magnitude takes two exchanges.  Rounding is done once,
// when weights are laid out; bound by memory.
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
                ((T*)p.scales)[(tile * p.groups + c * kGroups + q) * 16 + r] =
                    (T)sc;
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

template <int DT>
__device__ __forceinline__ short8v eight16(uint32_t d)
{
    if constexpr (DT == SVM_F16) {
        half2v v[4] = {__builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, 1.0f, 0),
                       __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, 1.0f, 1),
                       __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, 1.0f, 2),
                       __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(d, 1.0f, 3)};
        return __builtin_bit_cast(short8v, v);
    } else {
        bf16x2 v[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d, 1.0f, 0),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d, 1.0f, 1),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d, 1.0f, 2),
                       __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(d, 1.0f, 3)};
        return __builtin_bit_cast(short8v, v);
    }
}

struct UnpackArgs {
    const unsigned char* codes;
    const void* scales;
    int64_t n, k, chunks, groups, all;
    int gshift;
    void* W;
    int64_t ldw;
};

// A wave to a tile.  Exact: scale times code is a value of the type.
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
                (tile * p.groups + ((c * 128 + s * 32) >> p.gshift)) * 16 + r];
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

struct Linear4Args {
    const void* X;
    const unsigned char* codes;
    const void* scales;
    int64_t ldx, m, n, k, chunks, groups;
    int gshift;
    Epilogue e;
};

// Few rows: 16 NT outputs to a block and 16 MT rows, the inputs in chunks of
// 128 taken in turn by its W waves, whose sums are joined at the end in a
// fixed order.  The codes come straight from memory to the lane that
// multiplies them, the next chunk's while this one's are used.
// FEW: up to 4 rows, every fourth of the 16 that the matrix instruction takes,
// so that a lane has one sum to scale and not four.
template <int DT, int MT, int NT, int W, bool FEW>
__global__ __launch_bounds__(64 * W) void k_linear4(Linear4Args p)
{
    using T = Elem<DT>;
    constexpr int kCols = NT * 16, kPad = kCols + 4;
    constexpr int kRegs = FEW ? 1 : 4;
    __shared__ float red[W][MT * 16][kPad];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int i = lane & 15, g = lane >> 4;
    const int64_t t0 = (int64_t)blockIdx.x * NT;
    const int64_t r0 = (int64_t)blockIdx.y * (MT * 16);
    const int64_t tiles = (p.n + 15) / 16;
    float acc[MT][NT][kRegs];
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int b = 0; b < NT; ++b)
#pragma unroll
            for (int v = 0; v < kRegs; ++v) acc[a][b][v] = 0.0f;
    int64_t xrow[MT];  // -1: no row of X here
#pragma unroll
    for (int a = 0; a < MT; ++a) {
        const int64_t row = FEW ? ((i & 3) == 0 ? i >> 2 : p.m)
                                : r0 + a * 16 + i;
        xrow[a] = row < p.m ? row * p.ldx : -1;
    }
    uint4v code[NT];
    T scale[NT][4];
    RawEight<DT> x[MT][4];
    auto fetch = [&](int64_t c) {
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            // (past the last tile the last one again: its sums are not used)
            const int64_t t = t0 + b < tiles ? t0 + b : tiles - 1;
            code[b] = *(const uint4v*)(p.codes + (t * p.chunks + c) * 1024 +
                                       lane * 16);
#pragma unroll
            for (int s = 0; s < 4; ++s)
                scale[b][s] = ((const T*)p.scales)[
                    (t * p.groups + ((c * 128 + s * 32) >> p.gshift)) * 16 + i];
        }
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int s = 0; s < 4; ++s) {
                const int64_t at = c * 128 + s * 32 + g * 8;
                x[a][s].load(p.X, xrow[a] + at,
                             xrow[a] < 0 ? 0 : eight_of(p.k, at));
            }
    };
    if (wave < p.chunks) fetch(wave);
    for (int64_t c = wave; c < p.chunks; c += W) {
        uint4v d[NT];
        float sc[NT][4];
        Factor8<DT> f[MT][4];
#pragma unroll
        for (int b = 0; b < NT; ++b) {
            d[b] = code[b];
#pragma unroll
            for (int s = 0; s < 4; ++s) sc[b][s] = (float)scale[b][s];
        }
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
            for (int s = 0; s < 4; ++s) f[a][s].from(x[a][s]);
        if (c + W < p.chunks) fetch(c + W);
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int b = 0; b < NT; ++b) {
                const short8v w = eight16<DT>(d[b][s]);
#pragma unroll
                for (int a = 0; a < MT; ++a) {
                    floatx4 part = {0, 0, 0, 0};
#pragma unroll
                    for (int q = Factor8<DT>::kParts - 1; q >= 0; --q)
                        part = mfma32<DT>(f[a][s].v[q], w, part);
#pragma unroll
                    for (int v = 0; v < kRegs; ++v)
                        acc[a][b][v] = fmaf(part[v], sc[b][s], acc[a][b][v]);
                }
            }
    }
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
        for (int b = 0; b < NT; ++b)
#pragma unroll
            for (int v = 0; v < kRegs; ++v)
                red[wave][a * 16 + (FEW ? g : g * 4 + v)][b * 16 + i] =
                    acc[a][b][v];
    __syncthreads();
    for (int it = threadIdx.x; it < MT * 16 * NT * 2; it += 64 * W) {
        const int row = it / (NT * 2), c0 = it % (NT * 2) * 8;
        const int64_t r = r0 + row, j = t0 * 16 + c0;
        const int count = eight_of(p.n, j);
        if (r >= p.m || count == 0) continue;
        Eight<DT> v, bias;
        RawEight<DT> res;
#pragma unroll
        for (int e = 0; e < 8; ++e) v.v[e] = bias.v[e] = 0.0f;
        if (p.e.bias) bias.load(p.e.bias, j, count);
        if (p.e.residual) res.load(p.e.residual, r * p.e.ldr + j, count);
#pragma unroll
        for (int w = 0; w < W; ++w)
#pragma unroll
            for (int e = 0; e < 8; ++e) v.v[e] += red[w][row][c0 + e];
#pragma unroll
        for (int e = 0; e < 8; ++e) v.v[e] += bias.v[e];
        act_values(p.e.act, v.v);
        if (p.e.residual) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v.v[e] += res.at(e);
        }
        v.store(p.e.Y, r * p.e.ldy + j, count);
    }
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
                       cols, sh.chunks, sh.groups, sh.tiles * sh.chunks,
                       sh.gshift, to, ld};
    for_dtype(w.dtype, [&]<int DT>() {
        hipLaunchKernelGGL((k_unpack4<DT>), dim3(tile_blocks(a.all)),
                           dim3(256), 0, s, a);
    });
}

constexpr int64_t kMostFewRows = 64;

}  // namespace

void pack4(const svm_array& W, const svm_packed& to, hipStream_t s)
{
    const Shape4 sh(to);
    const PackArgs a{W.data, W.ld, to.rows, to.cols, sh.chunks, sh.groups,
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
    if (m > kMostFewRows) {
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
        product(p, ws, s);
        return;
    }
    if (!ws.run) return;
    const Linear4Args k{a.X.data, (const unsigned char*)a.W.data,
                        scales_of(a.W), a.X.ld, m, a.W.rows, a.W.cols,
                        sh.chunks, sh.groups, sh.gshift, e};
    for_dtype(a.W.dtype, [&]<int DT>() {
        auto go = [&]<int MT, int NT, int W, bool FEW>() {
            hipLaunchKernelGGL(
                (k_linear4<DT, MT, NT, W, FEW>),
                dim3((unsigned)((sh.tiles + NT - 1) / NT),
                     (unsigned)((m + MT * 16 - 1) / (MT * 16))),
                dim3(64 * W), 0, s, k);
        };
        if (m <= 4) go.template operator()<1, 1, 8, true>();
        else if (m <= 16) go.template operator()<1, 1, 8, false>();
        else if (m <= 32) go.template operator()<2, 1, 8, false>();
        else go.template operator()<4, 1, 8, false>();
    });
}

}  // namespace msvm
