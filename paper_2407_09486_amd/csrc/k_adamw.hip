// AdamW over many tensors in one launch, states in fp32 or in 8 bits, and the values of 8-bit states.
//
// The step only moves memory: 28 bytes a parameter with fp32 states and gradients, 16 with 8-bit states,
// bf16 gradients and copies (one read and one write of everything). A wave takes 256 consecutive elements
// at a time, four a lane, which is also what shares a pair of 8-bit scales: their maxima are two wave
// reductions, and nothing is shared between waves. A block takes kAdamChunk elements of one tensor, found
// through a table with an entry a block, so a step is one launch for any list of tensors.
//
// No fused multiply-adds: every operation is rounded as the formula is written, so a code of an 8-bit
// state does not depend on how a compiler pairs them.
#include "block_internal.h"

#pragma clang fp contract(off)

namespace enova {

namespace {

constexpr int kPer = 4;                        // elements of a lane
constexpr float kInv127 = 1.0f / 127, kInv255 = 1.0f / 255;

__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1)
        v = fmaxf(v, __shfl_xor(v, d));
    return v;
}

// x / d, correctly rounded, for many x of one d (Markstein's correction): with y the rounded reciprocal of d and q
// within an ulp of the quotient, q + (x - q d) y rounds to it. `near` says that neither 1 / d nor a quotient of up to 1 leaves the range
// of normal numbers (a quotient below it is too small to matter to a code); else the plain division is made.
struct Quotient {
    float d, y;
    bool near;
    __device__ explicit Quotient(float by) : d(by), y(1.0f / by), near(by > 0x1p-100f && by < 0x1p100f) {}
    __device__ float operator()(float x) const
    {
        if (!near)
            return x / d;
        const float q = x * y;
        return __builtin_fmaf(__builtin_fmaf(-q, d, x), y, q);
    }
};

// The square root of x in [0, 1], correctly rounded but for x too small to matter to a code: the hardware's is
// within an ulp, and the sign of x - s (s -+ ulp) tells on which side of the half ulp the root is (Tuckerman's test).
__device__ __forceinline__ float unit_sqrt(float x)
{
    float s = __builtin_amdgcn_sqrtf(x);
    const float below = __int_as_float(__float_as_int(s) - 1), above = __int_as_float(__float_as_int(s) + 1);
    const float rb = __builtin_fmaf(-below, s, x), ra = __builtin_fmaf(-above, s, x);
    s = rb <= 0.0f ? below : s;
    return ra > 0.0f ? above : s;
}

template <class T>
__device__ __forceinline__ void load4(const T *src, int64_t at, int left, bool wide, float (&v)[kPer])
{
    if (wide && left >= kPer) {
        if constexpr (sizeof(T) == 4) {
            const float4 q = *reinterpret_cast<const float4 *>(src + at);
            v[0] = q.x, v[1] = q.y, v[2] = q.z, v[3] = q.w;
        } else {
            const uint2 q = *reinterpret_cast<const uint2 *>(src + at);
            v[0] = __uint_as_float(q.x << 16), v[1] = __uint_as_float(q.x & 0xffff0000u);
            v[2] = __uint_as_float(q.y << 16), v[3] = __uint_as_float(q.y & 0xffff0000u);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        v[e] = e < left ? static_cast<float>(src[at + e]) : 0.0f;
}

template <class T>
__device__ __forceinline__ void store4(T *dst, int64_t at, int left, bool wide, const float (&v)[kPer])
{
    if (wide && left >= kPer) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4 *>(dst + at) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
            T h[kPer];
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                h[e] = static_cast<T>(v[e]);
            *reinterpret_cast<uint2 *>(dst + at) = __builtin_bit_cast(uint2, h);
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (e < left)
            dst[at + e] = static_cast<T>(v[e]);
}

__device__ __forceinline__ uint32_t load_codes(const uint8_t *src, int64_t at, int left, bool wide)
{
    if (wide && left >= kPer)
        return *reinterpret_cast<const uint32_t *>(src + at);
    uint32_t c = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (e < left)
            c |= static_cast<uint32_t>(src[at + e]) << (8 * e);
    return c;
}

__device__ __forceinline__ void store_codes(uint8_t *dst, int64_t at, int left, bool wide, uint32_t c)
{
    if (wide && left >= kPer) {
        *reinterpret_cast<uint32_t *>(dst + at) = c;
        return;
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e)
        if (e < left)
            dst[at + e] = static_cast<uint8_t>(c >> (8 * e));
}

__device__ __forceinline__ void decode4(uint32_t cm, uint32_t cv, float sm, float sv, float (&m)[kPer], float (&v)[kPer])
{
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const float a = static_cast<float>(static_cast<int8_t>(cm >> (8 * e))) * kInv127;
        const float b = static_cast<float>((cv >> (8 * e)) & 255u) * kInv255;
        m[e] = a * fabsf(a) * sm;
        const float r = b * b * sv;
        v[e] = r * r;
    }
}

// The dither of element i at a step: fractions of a turn that both indexes advance by irrational-like
// steps (Weyl sequences), even over the steps for every element; v's is half a turn from m's.
__device__ __forceinline__ uint32_t dither_turn(int64_t i, uint32_t step)
{
    return static_cast<uint32_t>(i) * 2654435769u + step * 1779033703u;
}
__device__ __forceinline__ float turn_fraction(uint32_t t) { return static_cast<float>(t >> 8) * 0x1p-24f; }

constexpr int kSets = kAdamChunk / (kAdamThreads * kPer);      // 256-element blocks of a wave

// What a lane reads of one of its wave's blocks.
template <int BITS>
struct AdamLoads {
    float p[kPer], g[kPer], m[BITS == 8 ? 1 : kPer], v[BITS == 8 ? 1 : kPer];
    uint32_t cm, cv;
    float sm, sv;
    template <class P, class G>
    __device__ void load(const AdamTensor &t, int64_t block, int64_t at, int left, bool wide)
    {
        load4(static_cast<const P *>(t.param), at, left, wide, p);
        load4(static_cast<const G *>(t.grad), at, left, wide, g);
        if constexpr (BITS == 8) {
            cm = load_codes(static_cast<const uint8_t *>(t.m), at, left, wide);
            cv = load_codes(static_cast<const uint8_t *>(t.v), at, left, wide);
            sm = t.m_scale[block / kAdamBlock];
            sv = t.v_scale[block / kAdamBlock];
        } else {
            load4(static_cast<const float *>(t.m), at, left, wide, m);
            load4(static_cast<const float *>(t.v), at, left, wide, v);
        }
    }
};

template <class P, int BITS>
__device__ __forceinline__ void adam_block(const AdamTensor &t, const AdamArgs &a, AdamLoads<BITS> &l, int64_t block, int64_t at,
                                           int left, bool wide, int lane)
{
    float m[kPer], v[kPer], r[kPer];
    if constexpr (BITS == 8) {
        decode4(l.cm, l.cv, l.sm, l.sv, m, v);
    } else {
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            m[e] = l.m[e], v[e] = l.v[e];
    }
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
        const float ge = l.g[e] * a.grad_scale;
        m[e] = m[e] * a.b1 + ge * a.b1c;
        v[e] = v[e] * a.b2 + (ge * ge) * a.b2c;
        r[e] = sqrtf(v[e]);
        // the reciprocal is within an ulp, so the update is within two of the formula's in fp32
        l.p[e] = l.p[e] * a.keep - (m[e] * a.lr) * __builtin_amdgcn_rcpf(r[e] * a.root + a.eps);
    }
    store4(static_cast<P *>(t.param), at, left, wide, l.p);
    if (t.copy)
        store4(static_cast<__bf16 *>(t.copy), at, left, wide, l.p);
    if constexpr (BITS == 8) {
        // elements past the end have g = m = v = 0 and take no part in the maxima
        float mm = 0.0f, mr = 0.0f;
        bool odd = false;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            mm = fmaxf(mm, fabsf(m[e]));
            mr = fmaxf(mr, r[e]);
            odd |= !(fabsf(m[e]) < __builtin_inff()) | !(r[e] < __builtin_inff());
        }
        mm = wave_max(mm);
        mr = wave_max(mr);
        odd = __any(odd);          // a NaN or an infinity: the 256 states stand for NaN from here on
        const Quotient by_m(mm > 0.0f ? mm : 1.0f), by_r(mr > 0.0f ? mr : 1.0f);
        uint32_t cm = 0, cv = 0;
#pragma unroll
        for (int e = 0; e < kPer; ++e) {
            const uint32_t turn = dither_turn(at + e, a.step);
            const float fa = unit_sqrt(by_m(fabsf(m[e]))) * 127.0f + turn_fraction(turn);
            const float fb = unit_sqrt(by_r(r[e])) * 255.0f + turn_fraction(turn + 0x80000000u);
            int qa = odd ? 1 : min(static_cast<int>(fa), 127);
            int qb = odd ? 1 : min(static_cast<int>(fb), 255);
            qb = v[e] > 0.0f ? max(qb, 1) : (odd ? qb : 0);
            qa = m[e] < 0.0f ? -qa : qa;
            cm |= static_cast<uint32_t>(qa & 255) << (8 * e);
            cv |= static_cast<uint32_t>(qb) << (8 * e);
        }
        store_codes(static_cast<uint8_t *>(t.m), at, left, wide, cm);
        store_codes(static_cast<uint8_t *>(t.v), at, left, wide, cv);
        if (lane == 0) {
            const float nan = __builtin_nanf("");
            t.m_scale[block / kAdamBlock] = odd ? nan : mm;
            t.v_scale[block / kAdamBlock] = odd ? nan : mr;
        }
    } else {
        store4(static_cast<float *>(t.m), at, left, wide, m);
        store4(static_cast<float *>(t.v), at, left, wide, v);
    }
}

// A chunk that is whole and aligned reads all its blocks before it works on the first.
template <class P, class G, int BITS>
__global__ void __launch_bounds__(kAdamThreads) k_adamw(const AdamTensor *tensors, const AdamChunk *chunks, AdamArgs a)
{
    const AdamChunk ch = chunks[blockIdx.x];
    const AdamTensor t = tensors[ch.tensor];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t from = static_cast<int64_t>(ch.index) * kAdamChunk + wave * kAdamBlock;
    constexpr int kStride = kAdamThreads / 64 * kAdamBlock;
    if (t.wide && from - wave * kAdamBlock + kAdamChunk <= t.numel) {
        AdamLoads<BITS> l[kSets];
#pragma unroll
        for (int s = 0; s < kSets; ++s)
            l[s].template load<P, G>(t, from + s * kStride, from + s * kStride + lane * kPer, kPer, true);
#pragma unroll
        for (int s = 0; s < kSets; ++s)
            adam_block<P, BITS>(t, a, l[s], from + s * kStride, from + s * kStride + lane * kPer, kPer, true, lane);
        return;
    }
#pragma unroll 1
    for (int s = 0; s < kSets; ++s) {
        const int64_t block = from + s * kStride;
        if (block >= t.numel)       // the wave's 256 elements: the same for all its lanes
            break;
        const int64_t at = block + lane * kPer;
        const int left = static_cast<int>(t.numel - at < kPer ? (t.numel > at ? t.numel - at : 0) : kPer);
        AdamLoads<BITS> l;
        l.template load<P, G>(t, block, at, left, t.wide);
        adam_block<P, BITS>(t, a, l, block, at, left, t.wide, lane);
    }
}

__global__ void __launch_bounds__(kAdamThreads) k_adamw_states(const AdamTensor *tensors, const AdamChunk *chunks,
                                                               const AdamValues *values)
{
    const AdamChunk ch = chunks[blockIdx.x];
    const AdamTensor t = tensors[ch.tensor];
    const AdamValues o = values[ch.tensor];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t from = static_cast<int64_t>(ch.index) * kAdamChunk + wave * kAdamBlock;
    constexpr int kStride = kAdamThreads / 64 * kAdamBlock;
    const uint8_t *const cm = static_cast<const uint8_t *>(t.m), *const cv = static_cast<const uint8_t *>(t.v);
    if (t.wide && o.wide && from - wave * kAdamBlock + kAdamChunk <= t.numel) {
        uint32_t qm[kSets], qv[kSets];
        float sm[kSets], sv[kSets];
#pragma unroll
        for (int s = 0; s < kSets; ++s) {
            const int64_t block = from + s * kStride;
            qm[s] = load_codes(cm, block + lane * kPer, kPer, true);
            qv[s] = load_codes(cv, block + lane * kPer, kPer, true);
            sm[s] = t.m_scale[block / kAdamBlock];
            sv[s] = t.v_scale[block / kAdamBlock];
        }
#pragma unroll
        for (int s = 0; s < kSets; ++s) {
            float m[kPer], v[kPer];
            decode4(qm[s], qv[s], sm[s], sv[s], m, v);
            store4(o.m, from + s * kStride + lane * kPer, kPer, true, m);
            store4(o.v, from + s * kStride + lane * kPer, kPer, true, v);
        }
        return;
    }
#pragma unroll 1
    for (int s = 0; s < kSets; ++s) {
        const int64_t block = from + s * kStride, at = block + lane * kPer;
        if (at >= t.numel)
            break;
        const int left = static_cast<int>(t.numel - at < kPer ? t.numel - at : kPer);
        float m[kPer], v[kPer];
        decode4(load_codes(cm, at, left, t.wide), load_codes(cv, at, left, t.wide), t.m_scale[block / kAdamBlock],
                t.v_scale[block / kAdamBlock], m, v);
        store4(o.m, at, left, o.wide, m);
        store4(o.v, at, left, o.wide, v);
    }
}

__global__ void k_adamw_grads(AdamTensor *t, AdamPointers p)
{
    const int i = threadIdx.x;
    if (i < p.n) {
        t[p.from + i].grad = p.a[i];
        t[p.from + i].wide = static_cast<int32_t>(p.wide >> i & 1);
    }
}
__global__ void k_adamw_values(AdamValues *v, AdamPointers p)
{
    const int i = threadIdx.x;
    if (i < p.n)
        v[p.from + i] = {static_cast<float *>(const_cast<void *>(p.a[i])), static_cast<float *>(p.b[i]), static_cast<int32_t>(p.wide >> i & 1)};
}

template <class P, class G>
hipError_t launch_typed(int bits, const AdamTensor *t, const AdamChunk *c, int n, const AdamArgs &a, hipStream_t st)
{
    if (bits == 8)
        k_adamw<P, G, 8><<<n, kAdamThreads, 0, st>>>(t, c, a);
    else
        k_adamw<P, G, 32><<<n, kAdamThreads, 0, st>>>(t, c, a);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_adamw(int bits, int param_dtype, int grad_dtype, const AdamTensor *t, const AdamChunk *c, int n,
                        const AdamArgs &a, hipStream_t st)
{
    if (param_dtype == ENOVA_F32)
        return grad_dtype == ENOVA_F32 ? launch_typed<float, float>(bits, t, c, n, a, st)
                                       : launch_typed<float, __bf16>(bits, t, c, n, a, st);
    return grad_dtype == ENOVA_F32 ? launch_typed<__bf16, float>(bits, t, c, n, a, st)
                                   : launch_typed<__bf16, __bf16>(bits, t, c, n, a, st);
}

hipError_t launch_adamw_grads(AdamTensor *t, const AdamPointers &p, hipStream_t st)
{
    k_adamw_grads<<<1, kAdamPointers, 0, st>>>(t, p);
    return hipGetLastError();
}

hipError_t launch_adamw_values(AdamValues *v, const AdamPointers &p, hipStream_t st)
{
    k_adamw_values<<<1, kAdamPointers, 0, st>>>(v, p);
    return hipGetLastError();
}

hipError_t launch_adamw_states(const AdamTensor *t, const AdamChunk *c, int n, const AdamValues *v, hipStream_t st)
{
    k_adamw_states<<<n, kAdamThreads, 0, st>>>(t, c, v);
    return hipGetLastError();
}

}  // namespace enova
