// One AdamW step over many tensors, states in 32 bits or in 8.
#include <cmath>
#include <type_traits>

#include "elem.hpp"
#include "layers.hpp"

namespace msvm {

namespace {

typedef float floatx4 __attribute__((ext_vector_type(4)));

// The tensors of one launch travel in its arguments (no table is copied to
// the device, nothing outlives the call).
constexpr int kPerLaunch = 48;

struct AdamTable {
    void* param[kPerLaunch];
    const void* grad[kPerLaunch];
    float* master[kPerLaunch];
    void *m[kPerLaunch], *v[kPerLaunch];
    float *ms[kPerLaunch], *vs[kPerLaunch];
    int64_t n[kPerLaunch];
    int32_t first[kPerLaunch + 1];  // first block of each tensor
    int32_t count;
};

struct AdamConst {
    float b1, c1, b2, c2;  // c = 1 - b
    float keep;            // 1 - lr weight_decay
    float rate;            // lr / (1 - b1^t)
    float root;            // 1 / sqrt(1 - b2^t)
    float eps, gscale;
};

constexpr float kTiny = 1e-30f;

// The value of an 8-bit code; the code past the steps is NaN.  No operation
// here is contracted: the value depends on the code and the scale alone.
__device__ __forceinline__ float decode8(int c, float scale, int steps)
{
#pragma clang fp contract(off)
    if (c < -steps || c > steps) return __builtin_nanf("");
    const float t = (float)c * (1.0f / (float)steps);
    return (t * fabsf(t)) * scale;
}

constexpr float kMost = 3.402823466e38f;

// One step of four values; r: about sqrt(v).  Not contracted, so that the
// states are the same wherever they are computed.  They are the definition's
// bit for bit; the weight's step is good to a few units of the quotient's last
// place (square root and reciprocal are the hardware's, each good to a unit).
__device__ __forceinline__ void adam_step(const AdamConst& k, const floatx4& g0,
                                          floatx4& p, floatx4& m, floatx4& v,
                                          floatx4& r)
{
#pragma clang fp contract(off)
    bool small = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const float g = g0[e] * k.gscale;
        m[e] = m[e] * k.b1 + g * k.c1;
        v[e] = v[e] * k.b2 + (g * g) * k.c2;
        const float ve = v[e];
        r[e] = __builtin_amdgcn_sqrtf(ve);
        small |= __builtin_amdgcn_classf(ve, 0x80);  // subnormal
    }
    if (small) {  // (the hardware's square root takes them for 0)
#pragma unroll
        for (int e = 0; e < 4; ++e) r[e] = sqrtf(v[e]);
    }
    float q[4], d[4];
    bool far = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        d[e] = r[e] * k.root + k.eps;
        const float i = __builtin_amdgcn_rcpf(d[e]);
        q[e] = m[e] * i;
        q[e] = fmaf(fmaf(-d[e], q[e], m[e]), i, q[e]);
        far |= !(fabsf(q[e]) <= kMost);
    }
    if (far) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (!(fabsf(q[e]) <= kMost)) q[e] = m[e] / d[e];
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) p[e] = p[e] * k.keep - k.rate * q[e];
}

// The codes of four values x (ROOT: of their square roots, r about those) in
// a block with `by` = steps^2 / largest: sqrt(|x| by) to the nearest whole
// number, ties to even.  The hardware's square root is good to a unit of its
// last place, so y to 2e-5, and to 8e-5 where r is one too: only where y comes
// within 2e-4 of a tie are the correctly rounded ones needed.
template <bool ROOT>
__device__ __forceinline__ void encode8(const floatx4& x, const floatx4& r,
                                        float by, bool live, int (&code)[4])
{
#pragma clang fp contract(off)
    constexpr int kSteps = ROOT ? 254 : 127, kBad = ROOT ? 255 : -128;
    float y[4], near = 0.0f;
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        y[e] = __builtin_amdgcn_sqrtf((ROOT ? r[e] : fabsf(x[e])) * by);
        near = fmaxf(near, fabsf(y[e] - rintf(y[e])));
        odd |= !(fabsf(x[e]) <= kMost);
    }
    if (near > 0.4998f) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            y[e] = sqrtf((ROOT ? sqrtf(x[e]) : fabsf(x[e])) * by);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float c = fminf(rintf(y[e]), (float)kSteps);
        if (ROOT) c = fmaxf(c, live && x[e] > 0.0f ? 1.0f : 0.0f);
        else c = copysignf(c, x[e]);
        code[e] = (int)c;
    }
    if (odd) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (!(fabsf(x[e]) <= kMost)) code[e] = kBad;
    }
}

// Four consecutive values: 4 times their size at once where all are there.
template <class T>
struct Four {
    typedef T Wide __attribute__((ext_vector_type(4)));
    typedef Wide Loose __attribute__((aligned(sizeof(T))));

    static __device__ __forceinline__ Wide load(const T* p, int64_t at, int left)
    {
        if (left >= 4) return *(const Loose*)(p + at);
        Wide x;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = e < left ? p[at + e] : (T)0;
        return x;
    }

    static __device__ __forceinline__ void store(T* p, int64_t at, int left,
                                                 Wide x)
    {
        if (left >= 4) {
            *(Loose*)(p + at) = x;
            return;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) p[at + e] = x[e];
    }
};

// A block of kAdamBlock values to a wave, four of them to a lane, so that the
// scales of 8-bit states are a matter of one wave.  One read and one write of
// all that a step touches.  Bound by memory: 67 million values in bf16 with
// master weights and 8-bit states 201 us, 5.3 TB/s; in 32 bits 347 us, 5.4
// TB/s (a large copy: 5.2).  With correctly rounded square roots and divisions
// for every value the former took 249: the vector instructions bound it.
template <int PT, int GT, int BITS, bool MASTER>
__global__ __launch_bounds__(256) void k_adamw(AdamTable t, AdamConst k)
{
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int blk = (int)blockIdx.x * 4 + wave;
    if (blk >= t.first[t.count]) return;
    int lo = 0, hi = t.count - 1;  // the tensor of this block
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (t.first[mid] <= blk) lo = mid; else hi = mid - 1;
    }
    using P = Elem<PT>;
    using G = Elem<GT>;
    const int64_t b = blk - t.first[lo];
    const int64_t at = b * kAdamBlock + lane * 4;
    const int64_t n = t.n[lo];
    // past the tensor's end: its states' last block, with gradient 0
    const int left = n - at >= 4 ? 4 : n - at > 0 ? (int)(n - at) : 0;
    P* param = (P*)t.param[lo];
    float* master = MASTER ? t.master[lo] : nullptr;
    const auto g = Four<G>::load((const G*)t.grad[lo], at, left);
    floatx4 p;
    if (MASTER) {
        p = *(const floatx4*)(master + at);
    } else {
        const auto q = Four<P>::load(param, at, left);
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] = (float)q[e];
    }
    floatx4 m, v, r;
    if (BITS == 8) {
        const auto cm = Four<int8_t>::load((const int8_t*)t.m[lo], at, 4);
        const auto cv = Four<uint8_t>::load((const uint8_t*)t.v[lo], at, 4);
        const float ms = t.ms[lo][b], vs = t.vs[lo][b];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            m[e] = decode8(cm[e], ms, 127);
            r[e] = decode8(cv[e], vs, 254);
            v[e] = r[e] * r[e];
        }
    } else {
        m = *(const floatx4*)((const float*)t.m[lo] + at);
        v = *(const floatx4*)((const float*)t.v[lo] + at);
    }
    floatx4 g4;
#pragma unroll
    for (int e = 0; e < 4; ++e) g4[e] = (float)g[e];
    adam_step(k, g4, p, m, v, r);
    if (MASTER) *(floatx4*)(master + at) = p;
    typename Four<P>::Wide out;
#pragma unroll
    for (int e = 0; e < 4; ++e) out[e] = (P)p[e];
    Four<P>::store(param, at, left, out);
    if (BITS == 8) {
        // (the rounded square root is monotone: that of the largest value is
        // the largest of them)
        float tm = 0.0f, tv = 0.0f;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float am = fabsf(m[e]);
            tm = fmaxf(tm, am <= kMost ? am : 0.0f);
            tv = fmaxf(tv, v[e] <= kMost ? v[e] : 0.0f);
        }
        tm = wave_max(tm);
        const float tr = sqrtf(wave_max(tv));
        const bool lm = tm > kTiny, lr = tr > kTiny;
        const float bm = lm ? 16129.0f / tm : 0.0f;
        const float br = lr ? 64516.0f / tr : 0.0f;
        Four<int8_t>::Wide cm;
        Four<uint8_t>::Wide cv;
        int im[4], iv[4];
        encode8<false>(m, r, bm, lm, im);
        encode8<true>(v, r, br, lr, iv);
#pragma unroll
        for (int e = 0; e < 4; ++e) cm[e] = (int8_t)im[e], cv[e] = (uint8_t)iv[e];
        *(Four<int8_t>::Wide*)((int8_t*)t.m[lo] + at) = cm;
        *(Four<uint8_t>::Wide*)((uint8_t*)t.v[lo] + at) = cv;
        if (lane == 0) {
            t.ms[lo][b] = lm ? tm : 0.0f;
            t.vs[lo][b] = lr ? tr : 0.0f;
        }
    } else {
        *(floatx4*)((float*)t.m[lo] + at) = m;
        *(floatx4*)((float*)t.v[lo] + at) = v;
    }
}

// Four values to a thread in each of kTurns turns, whose codes are all loaded
// before the first is decoded.  Bound by memory: 67 million values 130 us, 5.2
// TB/s (150 with one turn).
constexpr int kTurns = 4;

template <int STEPS>
__device__ __forceinline__ void decode_turns(
    const std::conditional_t<STEPS == 127, int8_t, uint8_t>* code,
    const float* scale, int64_t at, int64_t n, float* out)
{
    using F = Four<std::conditional_t<STEPS == 127, int8_t, uint8_t>>;
    typename F::Wide c[kTurns];
    float s[kTurns];
    int left[kTurns];
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
        const int64_t i = at + t * 1024, more = n - i;
        left[t] = more >= 4 ? 4 : more > 0 ? (int)more : 0;
        c[t] = F::load(code, i, left[t]);
        s[t] = more > 0 ? scale[i / kAdamBlock] : 0.0f;
    }
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
        Four<float>::Wide x;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float r = decode8(c[t][e], s[t], STEPS);
            x[e] = STEPS == 127 ? r : r * r;
        }
        Four<float>::store(out, at + t * 1024, left[t], x);
    }
}

__global__ __launch_bounds__(256) void k_adamw_state(
    const int8_t* m, const uint8_t* v, const float* ms, const float* vs,
    int64_t n, float* mo, float* vo)
{
    const int64_t at =
        (int64_t)blockIdx.x * (1024 * kTurns) + threadIdx.x * 4;
    if (mo) decode_turns<127>(m, ms, at, n, mo);
    if (vo) decode_turns<254>(v, vs, at, n, vo);
}

template <int PT, int GT>
void launch_group(const AdamTable& t, const AdamConst& k, int bits,
                  bool master, hipStream_t s)
{
    const dim3 grid((unsigned)((t.first[t.count] + 3) / 4)), block(256);
    auto go = [&]<int BITS, bool MASTER>() {
        hipLaunchKernelGGL((k_adamw<PT, GT, BITS, MASTER>), grid, block, 0, s,
                           t, k);
    };
    if constexpr (PT != SVM_F32) {
        if (master) {
            if (bits == 8) go.template operator()<8, true>();
            else go.template operator()<32, true>();
            return;
        }
    }
    if (bits == 8) go.template operator()<8, false>();
    else go.template operator()<32, false>();
}

}  // namespace

void adamw_step(const svm_adamw_tensor* t, int32_t n,
                const svm_adamw_params& p, hipStream_t s)
{
    AdamConst k;
    k.b1 = (float)p.beta1;
    k.c1 = (float)(1.0 - p.beta1);
    k.b2 = (float)p.beta2;
    k.c2 = (float)(1.0 - p.beta2);
    k.keep = (float)(1.0 - p.lr * p.weight_decay);
    k.rate = (float)(p.lr / (1.0 - std::pow(p.beta1, (double)p.step)));
    k.root = (float)(1.0 / std::sqrt(1.0 - std::pow(p.beta2, (double)p.step)));
    k.eps = (float)p.eps;
    k.gscale = (float)p.grad_scale;
    AdamTable tab;
    // one kernel for each combination of types among the tensors
    for (int pt = SVM_F32; pt <= SVM_F16; ++pt)
        for (int own = 1; own >= 0; --own)
            for (int master = 0; master < 2; ++master) {
                const int gt = own ? pt : SVM_F32;
                if (pt == SVM_F32 && (!own || master)) continue;
                tab.count = 0;
                tab.first[0] = 0;
                auto flush = [&]() {
                    if (tab.count == 0) return;
                    if (pt == SVM_F32)
                        launch_group<SVM_F32, SVM_F32>(tab, k, p.bits, false,
                                                       s);
                    else if (pt == SVM_BF16 && own)
                        launch_group<SVM_BF16, SVM_BF16>(tab, k, p.bits,
                                                         master, s);
                    else if (pt == SVM_BF16)
                        launch_group<SVM_BF16, SVM_F32>(tab, k, p.bits, master,
                                                        s);
                    else if (own)
                        launch_group<SVM_F16, SVM_F16>(tab, k, p.bits, master,
                                                       s);
                    else
                        launch_group<SVM_F16, SVM_F32>(tab, k, p.bits, master,
                                                       s);
                    tab.count = 0;
                };
                // values of a tensor in one launch (block numbers are int32)
                constexpr int64_t kMost = (int64_t)kAdamBlock << 24;
                for (int32_t i = 0; i < n; ++i) {
                    if (t[i].dtype != pt || t[i].grad_dtype != gt ||
                        (t[i].master != nullptr) != (master != 0))
                        continue;
                    for (int64_t at = 0; at < t[i].n; at += kMost) {
                        const int64_t len =
                            t[i].n - at < kMost ? t[i].n - at : kMost;
                        const int32_t nb =
                            (int32_t)((len + kAdamBlock - 1) / kAdamBlock);
                        if (tab.count == kPerLaunch ||
                            (tab.count > 0 &&
                             (int64_t)tab.first[tab.count] + nb > (1 << 25)))
                            flush();
                        const int c = tab.count;
                        const int64_t sb = p.bits == 8 ? 1 : 4;
                        tab.param[c] =
                            (char*)t[i].param + at * dtype_bytes(pt);
                        tab.grad[c] =
                            (const char*)t[i].grad + at * dtype_bytes(gt);
                        tab.master[c] = t[i].master ? t[i].master + at
                                                    : nullptr;
                        tab.m[c] = (char*)t[i].m + at * sb;
                        tab.v[c] = (char*)t[i].v + at * sb;
                        tab.ms[c] = t[i].m_scale
                                        ? t[i].m_scale + at / kAdamBlock
                                        : nullptr;
                        tab.vs[c] = t[i].v_scale
                                        ? t[i].v_scale + at / kAdamBlock
                                        : nullptr;
                        tab.n[c] = len;
                        if (c == 0) tab.first[0] = 0;
                        tab.first[c + 1] = tab.first[c] + nb;
                        tab.count = c + 1;
                    }
                }
                flush();
            }
}

void adamw_state(const int8_t* m, const uint8_t* v, const float* ms,
                 const float* vs, int64_t n, float* mo, float* vo,
                 hipStream_t s)
{
    // 2^32 values to a launch, a whole number of blocks and scales
    const int64_t most = (int64_t)256 << 24;
    for (int64_t at = 0; at < n; at += most) {
        const int64_t len = n - at < most ? n - at : most;
        hipLaunchKernelGGL(k_adamw_state,
                           dim3((unsigned)((len + kTurns * 1024 - 1) /
                                           (kTurns * 1024))),
                           dim3(256), 0, s, m ? m + at : nullptr,
                           v ? v + at : nullptr,
                           ms ? ms + at / kAdamBlock : nullptr,
                           vs ? vs + at / kAdamBlock : nullptr, len,
                           mo ? mo + at : nullptr, vo ? vo + at : nullptr);
    }
}

}  // namespace msvm
