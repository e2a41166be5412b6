// The products of the gated block and of the 8-bit codes for up to 64 rows of x: a window or a few, live.
//
// All there is to do is to read the weights once: 16 rows of them a block (of both projections for the gate),
// the reduction dealt out to the block's 16 waves in pieces of 128 bytes, straight from memory into the
// registers of the matrix operation (16 lanes hold a row's neighbouring 16 bytes each, so a row is read in whole
// lines over two operations), and joined through LDS at the end. Few blocks are enough: a block's 16 waves
// have 32 KiB and more on their way.
// Rows may start anywhere: the loads take any address, and where the reduction ends inside a piece its elements
// are read one by one, zeros in the place of the missing ones, for both operands. fp32 operands are taken apart in
// registers (three bf16 parts, six products), so the weights are read once in that type too.
#include "quantize.h"

namespace enova {

namespace {

constexpr int kFewWaves = 16;          // of a block; half as many where three or four fragments of x's rows fill LDS

// The operand of one matrix operation as a lane holds it: 8 elements (16 of int8), as they are or in parts.
template <class T>
struct FewOp {
    static constexpr int kElems = 8, kParts = 1;
    typedef mm_f4 Acc;
    uint4 v;
    __device__ void load(const T *p) { v = reinterpret_cast<const Any16 *>(p)->v; }
    __device__ void load_some(const T *p, int n)
    {
        T e[kElems] = {};
#pragma unroll
        for (int i = 0; i < kElems; ++i)
            if (i < n)
                e[i] = p[i];
        __builtin_memcpy(&v, e, 16);
    }
    __device__ static void mma(const FewOp &a, const FewOp &b, Acc &c) { c = Bf16Mm::mma(a.v, b.v, c); }
};
template <>
struct FewOp<int8_t> {
    static constexpr int kElems = 16;
    typedef mm_i4 Acc;
    uint4 v;
    __device__ void load(const int8_t *p) { v = reinterpret_cast<const Any16 *>(p)->v; }
    __device__ void load_some(const int8_t *p, int n)      // rows are whole 16 bytes
    {
        v = make_uint4(0u, 0u, 0u, 0u);
        if (n > 0)
            load(p);
    }
    __device__ static void mma(const FewOp &a, const FewOp &b, Acc &c) { c = Int8Mm::mma(a.v, b.v, c); }
};
template <>
struct FewOp<float> {
    static constexpr int kElems = 8;
    typedef mm_f4 Acc;
    float f[8];
    __device__ void load(const float *p)
    {
        const uint4 a = reinterpret_cast<const Any16 *>(p)[0].v, b = reinterpret_cast<const Any16 *>(p)[1].v;
        __builtin_memcpy(f, &a, 16);
        __builtin_memcpy(f + 4, &b, 16);
    }
    __device__ void load_some(const float *p, int n)
    {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            f[i] = i < n ? p[i] : 0.0f;
    }
    __device__ void parts(uint4 (&q)[3]) const
    {
        __bf16 a[8], b[8], c[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            a[i] = static_cast<__bf16>(f[i]);
            const float r = f[i] - static_cast<float>(a[i]);
            b[i] = static_cast<__bf16>(r);
            c[i] = static_cast<__bf16>(r - static_cast<float>(b[i]));
        }
        q[0] = __builtin_bit_cast(uint4, a);
        q[1] = __builtin_bit_cast(uint4, b);
        q[2] = __builtin_bit_cast(uint4, c);
    }
    __device__ static void mma(const FewOp &a, const FewOp &b, Acc &c)
    {
        uint4 x[3], y[3];
        a.parts(x);
        b.parts(y);
        c = Bf16Mm::mma(x[2], y[0], c);
        c = Bf16Mm::mma(x[0], y[2], c);
        c = Bf16Mm::mma(x[1], y[1], c);
        c = Bf16Mm::mma(x[1], y[0], c);
        c = Bf16Mm::mma(x[0], y[1], c);
        c = Bf16Mm::mma(x[0], y[0], c);
    }
};

template <class T, int EPI, int NB, int WAVES>
__global__ void __launch_bounds__(WAVES * 64) k_mm_few(MmParams p)
{
    typedef FewOp<T> Op;
    typedef typename Op::Acc Acc;
    constexpr int kMats = EPI == kMmGate ? 2 : 1, kSets = kMats * NB;
    __shared__ Acc joined[WAVES][kSets][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, i = lane % 16, g = lane / 16;
    const int n0 = blockIdx.x * 16;
    // W's rows (the last one again past the end: those columns are not stored), and x's
    const int64_t row = min(n0 + i, p.n - 1);
    const T *w[kMats], *x[NB];
    w[0] = reinterpret_cast<const T *>(static_cast<const char *>(p.w[0]) + row * p.ldw) + g * Op::kElems;
    if constexpr (kMats == 2)
        w[1] = reinterpret_cast<const T *>(static_cast<const char *>(p.w2[0]) + row * p.ldw) + g * Op::kElems;
#pragma unroll
    for (int b = 0; b < NB; ++b)
        x[b] = reinterpret_cast<const T *>(static_cast<const char *>(p.x[0]) + min(16 * b + i, p.m - 1) * p.ldx) + g * Op::kElems;
    Acc acc[kMats][NB];
#pragma unroll
    for (int k = 0; k < kMats; ++k)
#pragma unroll
        for (int b = 0; b < NB; ++b)
            acc[k][b] = Acc{0, 0, 0, 0};
    constexpr int kStep = 4 * Op::kElems, kSlab = 2 * kStep;       // of one operation, and of a wave's turn
    const int whole = p.k / kSlab;
    // 16 pieces of 16 bytes on their way
    constexpr int kAhead = NB * (EPI == kMmGate ? 2 : 1) <= 2 ? 4 : 2;
#pragma unroll kAhead
    for (int slab = wave; slab < whole; slab += WAVES) {
        Op ow[kMats][2], ox[NB][2];
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int at = slab * kSlab + s * kStep;
#pragma unroll
            for (int k = 0; k < kMats; ++k)
                ow[k][s].load(w[k] + at);
#pragma unroll
            for (int b = 0; b < NB; ++b)
                ox[b][s].load(x[b] + at);
        }
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int k = 0; k < kMats; ++k)
#pragma unroll
                for (int b = 0; b < NB; ++b)
                    Op::mma(ow[k][s], ox[b][s], acc[k][b]);
    }
    if (whole * kSlab < p.k && wave == whole % WAVES) {
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int at = whole * kSlab + s * kStep, left = p.k - at - g * Op::kElems;
            Op ow[kMats], ox[NB];
#pragma unroll
            for (int k = 0; k < kMats; ++k)
                ow[k].load_some(w[k] + at, left);
#pragma unroll
            for (int b = 0; b < NB; ++b)
                ox[b].load_some(x[b] + at, left);
#pragma unroll
            for (int k = 0; k < kMats; ++k)
#pragma unroll
                for (int b = 0; b < NB; ++b)
                    Op::mma(ow[k], ox[b], acc[k][b]);
        }
    }
#pragma unroll
    for (int k = 0; k < kMats; ++k)
#pragma unroll
        for (int b = 0; b < NB; ++b)
            joined[wave][k * NB + b][lane] = acc[k][b];
    __syncthreads();
    // a wave for each 16 rows of x: lane l has row l % 16 and columns 4 (l / 16) + 0..3
    if (wave >= NB)
        return;
    Acc sum[kMats];
#pragma unroll
    for (int k = 0; k < kMats; ++k) {
        sum[k] = joined[0][k * NB + wave][lane];
#pragma unroll
        for (int v = 1; v < WAVES; ++v)
            sum[k] += joined[v][k * NB + wave][lane];
    }
    const int64_t m = 16 * wave + i;
    const int n = n0 + 4 * g;
    if (m >= p.m)
        return;
    if constexpr (EPI == kMmGate) {
        if (n >= p.n8)
            return;
        float gv[4], uv[4], h[4], da[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            sum[0][e] = n + e < p.n ? sum[0][e] : 0.0f;
            sum[1][e] = n + e < p.n ? sum[1][e] : 0.0f;
            gv[e] = sum[0][e];
            uv[e] = sum[1][e];
        }
        gate_acts<std::is_same_v<T, float>>(p.act, gv, h, da);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            h[e] *= sum[1][e];
        if (p.c)
            store_operand<4>(static_cast<__bf16 *>(p.c) + m * p.ldc + n, p.plane, h);
        if (p.h32)
            *reinterpret_cast<float4 *>(p.h32 + m * p.ldg + n) = make_float4(h[0], h[1], h[2], h[3]);
        const int64_t at = m * p.ldg + n;
        if (p.ge) {                    // the other four of eight columns are 16 lanes away
            const float tg = finite_top(gv), tu = finite_top(uv);
            const int eg = coded_exponent(fmaxf(tg, __shfl_xor(tg, 16))), eu = coded_exponent(fmaxf(tu, __shfl_xor(tu, 16)));
            store_coded<true>(p.g, at, gv, eg);
            store_coded<false>(p.u, at, uv, eu);
            if (g % 2 == 0) {
                p.ge[at / 8] = static_cast<int8_t>(eg);
                p.ue[at / 8] = static_cast<int8_t>(eu);
            }
        } else if (p.g) {
            *reinterpret_cast<mm_f4 *>(static_cast<float *>(p.g) + at) = sum[0];
            *reinterpret_cast<mm_f4 *>(static_cast<float *>(p.u) + at) = sum[1];
        }
    } else if constexpr (EPI == kMmInt8) {
        const int v[4] = {sum[0][0], sum[0][1], sum[0][2], sum[0][3]};
        Int8Columns<4> columns;
        columns.load(p, n);
        finish_int8<4>(p, m, n, v, columns);
    } else {
        const float v[4] = {sum[0][0], sum[0][1], sum[0][2], sum[0][3]};
        finish_store<4>(p, m, n, v);
    }
}

// The 8-bit product of one row in one launch: every block makes the row's codes for itself, in LDS (it comes
// from the caches, 16 KiB for 8192 values; the launch that would make them once takes longer than that: one row,
// 8192 -> 4096: 24 us with it, 10.7 us so), while its weights are on their way. Four rows, one after the other, took
// longer than the launch (8192 -> 8192: 31 us, five rows with it 19); two and three were not tried.
constexpr int kFusedBytes = 64 * 1024;

template <class T>
__global__ void __launch_bounds__(kFewWaves * 64) k_i8_fused(MmParams p, QuantParams x)
{
    typedef FewOp<int8_t> Op;
    extern __shared__ __attribute__((aligned(16))) int8_t codes[];    // [pitch]
    __shared__ mm_i4 joined[kFewWaves][64];
    __shared__ float tops[kFewWaves], scale;
    constexpr int kThreads = kFewWaves * 64;
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, i = lane % 16, g = lane / 16;
    const int n0 = blockIdx.x * 16, pitch = p.k;
    const int8_t *const w = static_cast<const int8_t *>(p.w[0]) + min(n0 + i, p.n - 1) * p.ldw + g * 16;
    constexpr int kSlab = 128, kAhead = 4;
    const int whole = pitch / kSlab;
    Op ow[kAhead][2];
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
        const int slab = wave + a * kFewWaves;
#pragma unroll
        for (int s = 0; s < 2; ++s)
            ow[a][s].load_some(w + slab * kSlab + s * 64, slab < whole ? 1 : 0);
    }
    const T *const src = static_cast<const T *>(x.x);
    float v[8] = {}, top = 0.0f;       // zeros past the row: codes of 0 there
    for (int c = threadIdx.x * 8; c < x.cols; c += kThreads * 8) {
        quant_values(src, c, x.cols, x.gate, v);
        top = quant_top(v, top);
    }
    top = block_top<kThreads>(top, tops);
    for (int c = threadIdx.x * 8; c < pitch; c += kThreads * 8) {
        if (x.cols > kThreads * 8)                 // else v still holds them
            quant_values(src, c, x.cols, x.gate, v);
        *reinterpret_cast<uint2 *>(codes + c) = quant_codes(v, top);
    }
    if (threadIdx.x == 0)
        scale = quant_scale(top);
    __syncthreads();
    const int8_t *const q = codes + g * 16;        // all 16 rows of the operation are this one
    mm_i4 acc = {0, 0, 0, 0};
#pragma unroll
    for (int a = 0; a < kAhead; ++a) {
        const int slab = wave + a * kFewWaves;
        if (slab < whole)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                Op ox;
                ox.load(q + slab * kSlab + s * 64);
                Op::mma(ow[a][s], ox, acc);
            }
    }
#pragma unroll 4
    for (int slab = wave + kAhead * kFewWaves; slab < whole; slab += kFewWaves)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            Op a, b;
            a.load(w + slab * kSlab + s * 64);
            b.load(q + slab * kSlab + s * 64);
            Op::mma(a, b, acc);
        }
    if (whole * kSlab < pitch && wave == whole % kFewWaves)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const int at = whole * kSlab + s * 64, left = pitch - at - g * 16;
            Op a, b;
            a.load_some(w + at, left);
            b.load_some(q + at, left);
            Op::mma(a, b, acc);
        }
    joined[wave][lane] = acc;
    __syncthreads();
    const int n = n0 + 4 * g;
    if (wave || i || n >= p.n)
        return;
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w)
        acc += joined[w][lane];
    const int sum[4] = {acc[0], acc[1], acc[2], acc[3]};
    Int8Columns<4> columns;
    columns.load(p, n);
    p.sx = &scale;
    finish_int8<4>(p, 0, n, sum, columns);
}

template <class T, int EPI>
hipError_t launch(const MmParams &p, hipStream_t st)
{
    const unsigned n = (p.n + 15) / 16;
    switch ((p.m + 15) / 16) {
    case 1: k_mm_few<T, EPI, 1, kFewWaves><<<n, kFewWaves * 64, 0, st>>>(p); break;
    case 2: k_mm_few<T, EPI, 2, kFewWaves><<<n, kFewWaves * 64, 0, st>>>(p); break;
    case 3: k_mm_few<T, EPI, 3, kFewWaves / 2><<<n, kFewWaves * 32, 0, st>>>(p); break;
    default: k_mm_few<T, EPI, 4, kFewWaves / 2><<<n, kFewWaves * 32, 0, st>>>(p); break;
    }
    return hipGetLastError();
}

}  // namespace

bool i8_fused(int64_t rows, int pitch) { return rows == 1 && pitch <= kFusedBytes; }

hipError_t launch_i8_fused(const MmParams &p, const QuantParams &q, hipStream_t st)
{
    const unsigned n = (p.n + 15) / 16, bytes = p.k;
    const auto run = [&](auto kernel) {
        const hipError_t e = allow_lds(reinterpret_cast<const void *>(kernel), kFusedBytes);
        if (e != hipSuccess)
            return e;
        kernel<<<n, kFewWaves * 64, bytes, st>>>(p, q);
        return hipGetLastError();
    };
    return q.dtype == ENOVA_F32 ? run(k_i8_fused<float>) : run(k_i8_fused<__bf16>);
}

hipError_t launch_mm_few(const MmParams &p, MmEpilogue epi, int dtype, hipStream_t st)
{
    if (p.m > kMmFewRows)
        return hipErrorInvalidValue;
    switch (epi) {
    case kMmGate: return dtype == ENOVA_F32 ? launch<float, kMmGate>(p, st) : launch<__bf16, kMmGate>(p, st);
    case kMmStore: return dtype == ENOVA_F32 ? launch<float, kMmStore>(p, st) : launch<__bf16, kMmStore>(p, st);
    case kMmInt8: return launch<int8_t, kMmInt8>(p, st);
    default: return hipErrorInvalidValue;
    }
}

}  // namespace enova
