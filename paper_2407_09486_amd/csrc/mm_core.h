// The matrix product that the gated block and the 8-bit product share: a tile of BM x BN outputs a block,
// operands staged through LDS by asynchronous 16-byte loads, 16x16 matrix operations on 64 bytes of the
// reduction at a time.
//
// A slab is 128 bytes of the reduction (64 bf16, 128 int8). Two LDS buffers hold one slab of both operands
// each: while the waves multiply one, the loads of the next are in flight. The matrix operation's first
// operand is W (so a lane's four results are neighbouring columns of C, stored together) and its second X.
//
// An operand is staged as it lies in memory and in one of two layouts:
//   rows (kMmRows): LDS rows of one output index, 128 bytes of the reduction each, in eight 16-byte pieces
//     that are exchanged by a key of the row (XOR), so that a fragment read (16 rows, one piece each) finds
//     every bank once;
//   columns (kMmCols): LDS rows of one reduction index, 2 B times the tile's width each, read with the
//     transposing load (four reduction indexes of 16 output indexes to 16 lanes at a time); 32-byte units
//     are exchanged by a key of the reduction index.
// The exchange is in the addresses that the loads to LDS read from (their LDS side is fixed: 16 bytes a lane).
//
// What it measured (bf16, random values): 16384 x 8192 -> 4096 in 790 us, 1.39 PFLOP/s (a library's product on the same
// card: 695 us), matrix cores busy 76% of cycles at the 1.75 GHz that the power limit leaves. Two buffers of 64 KiB and
// eight waves of 128 x 64 outputs (a 256-tile): four waves of 128 x 128 read a third less LDS, but have nothing to run
// while one waits (915 us). Fragments are read half a slab ahead of their use, and reads and loads are spread between the
// operations (all at once, after the barrier: 994 us). A 128-tile, two to a compute unit, serves smaller products.
// The 256-tile's 128 sums and two sets of fragments leave few of a thread's 256 registers: of its instances the one for
// two operands in columns keeps 52 bytes a thread in scratch memory, and the gate's for ragged reductions 20.
//
// The loads to LDS are written out as instructions: the compiler, which cannot tell the two buffers apart,
// waits for every load to LDS before the next LDS read. They write no register, and every wave waits for its
// own (vmcnt) before the barrier that hands a buffer over.
#pragma once

#include <type_traits>
#include <utility>

#include "block_internal.h"

namespace enova {

namespace {

typedef __bf16 mm_bf8 __attribute__((ext_vector_type(8)));
typedef short mm_s4 __attribute__((ext_vector_type(4)));
typedef float mm_f4 __attribute__((ext_vector_type(4)));
typedef int mm_i4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) char lds_char;

constexpr int kSlabBytes = 128;

// 16 zero bytes: where the loads of pieces past the end of the reduction point.
static __device__ const uint4 mm_zero = {0u, 0u, 0u, 0u};

struct Bf16Mm {
    typedef mm_f4 Acc;
    static constexpr int kElem = 2;
    static constexpr bool kExact = false;      // activations (gate_act)
    __device__ static Acc mma(uint4 a, uint4 b, Acc c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(mm_bf8, a), __builtin_bit_cast(mm_bf8, b), c, 0, 0, 0);
    }
};
struct PartsMm : Bf16Mm {              // of fp32 operands in three parts
    static constexpr bool kExact = true;
};
struct Int8Mm {
    typedef mm_i4 Acc;
    static constexpr int kElem = 1;
    __device__ static Acc mma(uint4 a, uint4 b, Acc c)
    {
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(mm_i4, a), __builtin_bit_cast(mm_i4, b), c, 0, 0, 0);
    }
};

// f(0), f(1), ... with compile-time numbers.
template <class F, int... I>
__device__ __forceinline__ void each(F f, std::integer_sequence<int, I...>)
{
    (f(std::integral_constant<int, I>()), ...);
}
template <int N, class F>
__device__ __forceinline__ void each(F f)
{
    each(f, std::make_integer_sequence<int, N>());
}

// Which column of a wave's 64 the first operand's row i of fragment t is: with rows in LDS, fragments
// interleave in fours so that a lane ends up with 16 neighbouring columns (8 of either projection for the
// gate); the transposing load gives neighbouring columns to neighbouring lanes.
enum WMap { kMapQuads, kMapHalves, kMapPlain };
template <WMap MAP>
__device__ __forceinline__ constexpr int w_row(int t, int i)
{
    return MAP == kMapQuads ? 64 * (t / 4) + 16 * (i / 4) + 4 * (t % 4) + i % 4
           : MAP == kMapHalves ? 32 * (t / 2) + 8 * (i / 4) + 4 * (t % 2) + i % 4
                               : 16 * t + i;
}
// The key of an LDS row, even over the 16 rows of any fragment (together with the row's parity, which
// chooses the half of the banks).
template <WMap MAP>
__device__ __forceinline__ int row_key(int r)
{
    return MAP == kMapQuads ? ((r >> 1) & 1) | ((r >> 3) & 6) : MAP == kMapHalves ? ((r >> 1) & 1) | ((r >> 2) & 6) : (r >> 1) & 7;
}
__device__ __forceinline__ int col_key(int k) { return (k & 3) | ((k >> 3) & 1) << 2; }

// The 16-byte pieces of one operand that a thread loads for every slab.
template <int LAYOUT, int TILE, int WAVES, WMap MAP, int ELEM>
struct Staged {
    static constexpr int kBytes = TILE * kSlabBytes;
    static constexpr int kLoads = kBytes / 1024 / WAVES;      // wave-wide loads of 1 KiB
    static constexpr int kPitch = TILE * ELEM;                // columns: bytes of an LDS row
    static constexpr int kPieces = kPitch / 16;               // columns: pieces of an LDS row
    unsigned off[kLoads];              // from the tile's first row (columns: from the slab's)
    int at[kLoads];                    // the piece's place along the reduction within a slab, in elements

    // first: the tile's first row (column); count: the rows (columns) there are
    __device__ void init(int wave, int lane, int64_t ld, int first, int count)
    {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int q = wave * kLoads + j;
            if constexpr (LAYOUT == kMmRows) {
                const int r = q * 8 + lane / 8, piece = (lane % 8) ^ row_key<MAP>(r);
                int from = r;
                if constexpr (MAP == kMapHalves)              // rows of both projections in turn, 32 of each
                    from = r / 64 * 32 + r % 32;
                from = min(from, count - 1 - first);
                off[j] = static_cast<unsigned>(from * ld) + piece * 16;
                at[j] = piece * 16 / ELEM;
            } else {
                const int b = q * 64 + lane, k = b / kPieces, piece = (b % kPieces) ^ (col_key(k) << 1);
                const int last = (count - 1) / (16 / ELEM) * (16 / ELEM);       // the last whole or padded piece
                const int col = min(first + piece * (16 / ELEM), last);
                off[j] = static_cast<unsigned>(k * ld) + col * ELEM;
                at[j] = k;
            }
        }
    }
    // base: the tile's first row (columns: row 0) at the slab's start; lds: LDS address of the operand's buffer
    template <bool TAIL>
    __device__ void load(int j, const char *base, unsigned lds, int wave, int left) const
    {
        const unsigned to = lds + (wave * kLoads + j) * 1024;
        if (TAIL) {
            const char *src = at[j] < left ? base + off[j] : reinterpret_cast<const char *>(&mm_zero);
            asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "s"(to) : "m0", "memory");
        } else {
            asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off[j]), "s"(base), "s"(to) : "m0", "memory");
        }
    }
};

// Fragments of one operand: 16 output indexes x 64 bytes of the reduction.
template <int LAYOUT, int TILE, WMap MAP, int ELEM, int N>
struct Fragments {
    unsigned a[LAYOUT == kMmRows ? 2 : N];
    __device__ void init(int first, int lane)
    {
        const int i = lane % 16, g = lane / 16;
        if constexpr (LAYOUT == kMmRows) {
            const int r = first + w_row<MAP>(0, i);
            a[0] = r * kSlabBytes + ((g ^ row_key<MAP>(r)) * 16);
            a[1] = a[0] ^ 64;
        } else {
            const int k = 8 * g + i / 4;
#pragma unroll
            for (int t = 0; t < N; ++t)
                a[t] = k * TILE * ELEM + ((((first / 16) + t) ^ col_key(k)) * 32) + (i % 4) * 8;
        }
    }
    __device__ uint4 read(const char *lds, int t, int s) const
    {
        if constexpr (LAYOUT == kMmRows) {
            return *reinterpret_cast<const uint4 *>(lds + a[s] + w_row<MAP>(t, 0) * kSlabBytes);
        } else {
            const char *p = lds + a[t] + s * 32 * TILE * ELEM;
            const mm_s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) mm_s4 *)(p));
            const mm_s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) mm_s4 *)(p + 4 * TILE * ELEM));
            const uint2 l = __builtin_bit_cast(uint2, lo), h = __builtin_bit_cast(uint2, hi);
            return make_uint4(l.x, l.y, h.x, h.y);
        }
    }
};

// act(g) and its derivative. EXACT (blocks of fp32): within a few ulp of the result, GELU with expf and erfcf. Else (bf16,
// whose next rounding is up to 2^-8, and 8-bit codes) the hardware's exponential and reciprocal, an ulp each, the former of a
// rounded product (a relative |g| 2^-24 more), and for GELU Phi from Abramowitz and Stegun's formula 7.1.26 for erf,
// sharing the exponential with the density: within 2.5e-7, which is no more than the order of the tail where g < -5.
// With expf, erff and division a tile of the bf16 hidden gradient spent as long on them as on memory
// (16384 x 4096 -> 8192: 1019 us, 996 us so).
template <int ACT, bool EXACT>
__device__ __forceinline__ void gate_act(float g, float &a, float &da)
{
    constexpr float kLog2e = 1.4426950408889634f, kLog2eRest = 1.4426950408889634 - kLog2e;
    if constexpr (ACT == ENOVA_GATE_RELU) {
        a = g < 0.0f ? 0.0f : g;
        da = g > 0.0f ? 1.0f : 0.0f;
    } else if constexpr (ACT == ENOVA_GATE_SILU && EXACT) {
        // e^-g as 2^t (1 + r ln 2), r what the product t lost; beyond |g| = 128 it is 0 or infinite all the same
        const float x = fminf(fmaxf(g, -128.0f), 128.0f), t = -kLog2e * x;
        const float r = __builtin_fmaf(-kLog2e, x, -t) - kLog2eRest * x, p = __builtin_amdgcn_exp2f(t);
        const float e = p < __builtin_inff() ? __builtin_fmaf(p, r * 0.6931471805599453f, p) : p;
        const float s = __builtin_amdgcn_rcpf(1.0f + e);
        a = g * s;
        da = s * (1.0f + g * (g < 0.0f ? 1.0f - s : e * s));
    } else if constexpr (ACT == ENOVA_GATE_SILU) {
        const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * g));
        a = g * s;
        da = s * (1.0f + g * (1.0f - s));
    } else if constexpr (EXACT) {
        const float cdf = 0.5f * erfcf(-0.70710678118654752f * g);
        a = g * cdf;
        da = cdf + g * expf(-0.5f * g * g) * 0.39894228040143268f;
    } else {
        const float t = __builtin_amdgcn_rcpf(1.0f + 0.3275911f * 0.70710678118654752f * fabsf(g));
        const float e = __builtin_amdgcn_exp2f(-0.5f * kLog2e * g * g);
        const float tail = 0.5f * e * t * (0.254829592f + t * (-0.284496736f + t * (1.421413741f + t * (-1.453152027f + t * 1.061405429f))));
        const float cdf = g < 0.0f ? tail : 1.0f - tail;
        a = g * cdf;
        da = cdf + g * e * 0.39894228040143268f;
    }
}
template <bool EXACT, int N>
__device__ __forceinline__ void gate_acts(int act, const float (&g)[N], float (&a)[N], float (&da)[N])
{
    const auto all = [&](auto which) {
#pragma unroll
        for (int e = 0; e < N; ++e)
            gate_act<decltype(which)::value, EXACT>(g[e], a[e], da[e]);
    };
    if (act == ENOVA_GATE_SILU)
        all(std::integral_constant<int, ENOVA_GATE_SILU>());
    else if (act == ENOVA_GATE_GELU)
        all(std::integral_constant<int, ENOVA_GATE_GELU>());
    else
        all(std::integral_constant<int, ENOVA_GATE_RELU>());
}

// N neighbouring values as bf16, or as three bf16 parts in planes of their own (an fp32 operand of a later
// product), where the whole run is inside the row and aligned.
template <int N>
__device__ __forceinline__ void store_operand(__bf16 *dst, int64_t plane, const float (&v)[N])
{
    __bf16 h[N];
#pragma unroll
    for (int e = 0; e < N; ++e)
        h[e] = static_cast<__bf16>(v[e]);
    typedef uint32_t pack __attribute__((ext_vector_type(N / 2)));
    *reinterpret_cast<pack *>(dst) = __builtin_bit_cast(pack, h);
    if (plane) {
        __bf16 mid[N], low[N];
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const float r = v[e] - static_cast<float>(h[e]);
            mid[e] = static_cast<__bf16>(r);
            low[e] = static_cast<__bf16>(r - static_cast<float>(mid[e]));
        }
        *reinterpret_cast<pack *>(dst + plane) = __builtin_bit_cast(pack, mid);
        *reinterpret_cast<pack *>(dst + 2 * plane) = __builtin_bit_cast(pack, low);
    }
}

__device__ __forceinline__ void load8(const float *src, float (&v)[8])
{
    const float4 a = reinterpret_cast<const float4 *>(src)[0], b = reinterpret_cast<const float4 *>(src)[1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void store8(float *dst, const float (&v)[8])
{
    reinterpret_cast<float4 *>(dst)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4 *>(dst)[1] = make_float4(v[4], v[5], v[6], v[7]);
}

// The bf16 block keeps g and u for its gradient as f16 with the exponent of the largest of eight neighbours: 11 bits of
// every value within 2^-29 of that, half of fp32's bytes. The gradient's own rounding to bf16 is eight times coarser
// (errors against 64 bits are the same 2.3e-3 as with fp32 g and u); bf16 would have added half as much again.
// e is that exponent (a row's values that are not finite have no part in it and stay what they are).
__device__ __forceinline__ int coded_exponent(float top)
{
    return max(static_cast<int>(__float_as_uint(top) >> 23) - 127, -110);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float(static_cast<unsigned>(127 + e) << 23); }
template <int N>
__device__ __forceinline__ float finite_top(const float (&v)[N])
{
    float top = 0.0f;
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float a = fabsf(v[e]);
        top = a < __builtin_inff() ? fmaxf(top, a) : top;
    }
    return top;
}
// N values under exponent e. SIGNED (g): a zero's sign bit says that the value was not positive. One that was, but is
// nothing beside its neighbours, comes back as the smallest normal number: ReLU's derivative is 1 there.
template <bool SIGNED, int N>
__device__ __forceinline__ void store_coded(void *dst, int64_t at, const float (&v)[N], int e)
{
    const float by = power_of_two(14 - e);
    _Float16 h[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        h[i] = static_cast<_Float16>(v[i] * by);
        if (SIGNED)
            h[i] = v[i] > 0.0f ? h[i] : -__builtin_fabsf16(h[i]);
    }
    typedef uint32_t pack __attribute__((ext_vector_type(N / 2)));
    *reinterpret_cast<pack *>(static_cast<_Float16 *>(dst) + at) = __builtin_bit_cast(pack, h);
}

// Eight saved values of g and of u as they lie in memory.
struct SavedPiece {
    uint4 q[4];
    int eg, eu;
    __device__ void load(const MmParams &p, int64_t m, int n)
    {
        const int64_t at = m * p.ldg + n;
        if (p.ge) {
            q[0] = *reinterpret_cast<const uint4 *>(static_cast<const _Float16 *>(p.g) + at);
            q[1] = *reinterpret_cast<const uint4 *>(static_cast<const _Float16 *>(p.u) + at);
            eg = p.ge[at / 8];
            eu = p.ue[at / 8];
        } else {
            const uint4 *const g = reinterpret_cast<const uint4 *>(static_cast<const float *>(p.g) + at);
            const uint4 *const u = reinterpret_cast<const uint4 *>(static_cast<const float *>(p.u) + at);
            q[0] = g[0], q[1] = g[1], q[2] = u[0], q[3] = u[1];
        }
    }
    __device__ void values(const MmParams &p, float (&g)[8], float (&u)[8]) const
    {
        if (p.ge) {
            typedef _Float16 half8 __attribute__((ext_vector_type(8)));
            typedef uint16_t bits8 __attribute__((ext_vector_type(8)));
            const half8 hg = __builtin_bit_cast(half8, q[0]), hu = __builtin_bit_cast(half8, q[1]);
            const bits8 bits = __builtin_bit_cast(bits8, q[0]);
            const float bg = power_of_two(eg - 14), bu = power_of_two(eu - 14);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                g[e] = bits[e] ? static_cast<float>(hg[e]) * bg : 0x1p-126f;
                u[e] = static_cast<float>(hu[e]) * bu;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const mm_f4 a = __builtin_bit_cast(mm_f4, q[i]), b = __builtin_bit_cast(mm_f4, q[2 + i]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    g[4 * i + e] = a[e];
                    u[4 * i + e] = b[e];
                }
            }
        }
    }
};

// What becomes of eight neighbouring columns n .. n + 7 of a finished row.
template <bool EXACT>
__device__ __forceinline__ void finish_gate(const MmParams &p, int64_t m, int n, float (&g)[8], float (&u)[8])
{
    float h[8], da[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        g[e] = n + e < p.n ? g[e] : 0.0f;
        u[e] = n + e < p.n ? u[e] : 0.0f;
    }
    gate_acts<EXACT>(p.act, g, h, da);
#pragma unroll
    for (int e = 0; e < 8; ++e)
        h[e] *= u[e];
    if (p.c)
        store_operand<8>(static_cast<__bf16 *>(p.c) + m * p.ldc + n, p.plane, h);
    if (p.h32)
        store8(p.h32 + m * p.ldg + n, h);
    if (p.ge) {
        const int64_t at = m * p.ldg + n;
        const int eg = coded_exponent(finite_top(g)), eu = coded_exponent(finite_top(u));
        store_coded<true>(p.g, at, g, eg);
        store_coded<false>(p.u, at, u, eu);
        p.ge[at / 8] = static_cast<int8_t>(eg);
        p.ue[at / 8] = static_cast<int8_t>(eu);
    } else if (p.g) {
        store8(static_cast<float *>(p.g) + m * p.ldg + n, g);
        store8(static_cast<float *>(p.u) + m * p.ldg + n, u);
    }
}
template <bool EXACT>
__device__ __forceinline__ void finish_gate_back(const MmParams &p, int64_t m, int n, const float (&dh)[8], const float (&g)[8],
                                                 const float (&u)[8])
{
    float dg[8], du[8], a[8], da[8];
    gate_acts<EXACT>(p.act, g, a, da);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float d = n + e < p.n ? dh[e] : 0.0f;
        dg[e] = d * u[e] * da[e];
        du[e] = d * a[e];
    }
    store_operand<8>(static_cast<__bf16 *>(p.c) + m * p.ldc + n, p.plane, dg);
    store_operand<8>(static_cast<__bf16 *>(p.c2) + m * p.ldc + n, p.plane, du);
}
// N neighbouring values of C (kMmStore, kMmInt8)
template <int N>
__device__ __forceinline__ void finish_store(const MmParams &p, int64_t m, int n, const float (&v)[N])
{
    void *to = p.c;
    if (p.m2 && m >= p.m1) {
        if (m < p.m2)
            return;
        to = p.c2;
        m -= p.m2;
    }
    if (p.f32) {
        float *const c = static_cast<float *>(to) + m * p.ldc + n;
        if (p.wide && n + N <= p.n) {
#pragma unroll
            for (int e = 0; e < N; e += 4)
                *reinterpret_cast<float4 *>(c + e) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (n + e < p.n)
                    c[e] = v[e];
        }
    } else {
        __bf16 *const c = static_cast<__bf16 *>(to) + m * p.ldc + n;
        if (p.wide && n + N <= p.n) {
            store_operand<N>(c, 0, v);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e)
                if (n + e < p.n)
                    c[e] = static_cast<__bf16>(v[e]);
        }
    }
}
// The scales and biases of columns n .. n + N - 1 (zeros past the last).
template <int N>
struct Int8Columns {
    float scale[N], bias[N];
    __device__ void load(const MmParams &p, int n)
    {
#pragma unroll
        for (int e = 0; e < N; ++e) {
            scale[e] = n + e < p.n ? p.sw[n + e] : 0.0f;
            bias[e] = p.bias && n + e < p.n ? p.bias[n + e] : 0.0f;
        }
    }
};
template <int N>
__device__ __forceinline__ void finish_int8(const MmParams &p, int64_t m, int n, const int (&sum)[N], const Int8Columns<N> &c)
{
    const float f = p.sx[m];
    float v[N];
#pragma unroll
    for (int e = 0; e < N; ++e)
        v[e] = static_cast<float>(sum[e]) * f * c.scale[e] + c.bias[e];
    finish_store<N>(p, m, n, v);
}

template <class MM, int EPI, int XL, int WL, int BM, int BN, int WM, int WN>
struct Mm {
    static constexpr int kWaves = WM * WN, kThreads = kWaves * 64;
    static constexpr int kTm = BM / WM / 16, kTn = BN / WN / 16;   // fragments of a wave
    static constexpr WMap kMap = EPI == kMmGate ? kMapHalves : WL == kMmRows ? kMapQuads : kMapPlain;
    static constexpr int kElem = MM::kElem;
    static constexpr int kSlab = kSlabBytes / kElem;
    static constexpr int kCols = EPI == kMmGate ? BN / 2 : BN;     // columns of C that a tile covers
    typedef Staged<XL, BM, kWaves, kMapPlain, kElem> StageX;
    typedef Staged<WL, BN, kWaves, kMap, kElem> StageW;
    static constexpr int kBufBytes = StageX::kBytes + StageW::kBytes;
    static constexpr int kPitch = BN + 4;      // of the LDS rows that results pass through: fragments' rows meet no bank twice
    static constexpr int kLds = BM / 2 * kPitch * 4 > 2 * kBufBytes ? BM / 2 * kPitch * 4 : 2 * kBufBytes;
    static constexpr int kWn = BN / WN;        // columns (rows of W) of a wave
    static_assert(kWn % 64 == 0, "a wave covers columns by 64");
};

// Tile of a block: blocks that run at the same time on one XCD (every eighth block) take neighbouring
// tiles, four tile rows deep, so that its L2 holds what they share (y of 16384 x 8192 -> 4096: 908, 888, 858,
// 914 us with 1, 2, 4, 8).
__device__ __forceinline__ void mm_tile(int b, int tiles_m, int tiles_n, int &tm, int &tn)
{
    const int total = tiles_m * tiles_n;
    const int per = total / 8, more = total % 8, x = b % 8;
    const int id = x * per + min(x, more) + b / 8;
    constexpr int kDeep = 4;
    const int group = id / (kDeep * tiles_n), first = group * kDeep;
    const int deep = min(kDeep, tiles_m - first), in = id - group * kDeep * tiles_n;
    tm = first + in % deep;
    tn = in / deep;
}

template <class MM, int EPI, int XL, int WL, int BM, int BN, int WM, int WN, bool TAIL>
__device__ __forceinline__ void mm_block(const MmParams &p, int block)
{
    typedef Mm<MM, EPI, XL, WL, BM, BN, WM, WN> C;
    typedef typename MM::Acc Acc;
    extern __shared__ __attribute__((aligned(1024))) char lds[];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int wm = wave / WN, wn = wave % WN;
    const int tiles = p.tiles_m * p.tiles_n;
    const int slice = block / tiles;
    int tile_m, tile_n;
    mm_tile(block - slice * tiles, p.tiles_m, p.tiles_n, tile_m, tile_n);
    const int m0 = tile_m * BM, n0 = tile_n * C::kCols;

    typename C::StageX sx;
    typename C::StageW sw;
    sx.init(wave, lane, p.ldx, m0, p.m);
    sw.init(wave, lane, p.ldw, n0, p.n);
    Fragments<XL, BM, kMapPlain, C::kElem, C::kTm> fx;
    Fragments<WL, BN, C::kMap, C::kElem, C::kTn> fw;
    fx.init(wm * (BM / WM), lane);
    fw.init(wn * C::kWn, lane);

    Acc acc[C::kTm][C::kTn];
#pragma unroll
    for (int i = 0; i < C::kTm; ++i)
#pragma unroll
        for (int j = 0; j < C::kTn; ++j)
            acc[i][j] = Acc{0, 0, 0, 0};

    // slabs of this slice, over all segments
    const int per = (p.k + C::kSlab - 1) / C::kSlab, all = per * p.segments;
    const int begin = static_cast<int>(static_cast<int64_t>(all) * slice / p.slices);
    const int end = static_cast<int>(static_cast<int64_t>(all) * (slice + 1) / p.slices);
    const int64_t step_x = XL == kMmRows ? kSlabBytes : C::kSlab * p.ldx;
    const int64_t step_w = WL == kMmRows ? kSlabBytes : C::kSlab * p.ldw;
    const int64_t tile_x = XL == kMmRows ? m0 * p.ldx : 0, tile_w = WL == kMmRows ? n0 * p.ldw : 0;
    // what is staged next: the operands' slab addresses, and how much of the segment's reduction is left
    int seg = begin / per;
    int left = p.k - (begin - seg * per) * C::kSlab;
    const char *next_x = nullptr, *next_w = nullptr, *next_w2 = nullptr;
    const auto enter = [&](int64_t slab) {
        next_x = static_cast<const char *>(p.x[seg]) + tile_x + slab * step_x;
        next_w = static_cast<const char *>(p.w[seg]) + tile_w + slab * step_w;
        if constexpr (EPI == kMmGate)
            next_w2 = static_cast<const char *>(p.w2[seg]) + tile_w + slab * step_w;
    };
    const unsigned lds0 = static_cast<unsigned>(reinterpret_cast<uintptr_t>((lds_char *)lds));
    constexpr int kLoads = C::StageX::kLoads + C::StageW::kLoads;
    const auto stage_one = [&](int j, unsigned buf) {
        if (j < C::StageX::kLoads)
            sx.template load<TAIL>(j, next_x, buf, wave, left);
        else {
            const int jw = j - C::StageX::kLoads;
            // the gate's LDS rows are 32 of one projection and 32 of the other in turn: four loads of each
            const bool second = EPI == kMmGate && ((wave * C::StageW::kLoads + jw) / 4) % 2;
            sw.template load<TAIL>(jw, second ? next_w2 : next_w, buf + C::StageX::kBytes, wave, left);
        }
    };
    const auto staged = [&] {
        left -= C::kSlab;
        next_x += step_x;
        next_w += step_w;
        if constexpr (EPI == kMmGate)
            next_w2 += step_w;
        if (left <= 0 && ++seg < p.segments) {
            left = p.k;
            enter(0);
        }
    };
    const auto stage = [&](int which) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
            stage_one(j, lds0 + which * C::kBufBytes);
        staged();
    };
    struct Set {
        uint4 f[C::kTn + C::kTm];      // W's fragments, then X's
    };
    const auto read_one = [&](Set &f, int j, int which, int s) {
        const char *const buf = lds + which * C::kBufBytes;
        f.f[j] = j < C::kTn ? fw.read(buf + C::StageX::kBytes, j, s) : fx.read(buf, j - C::kTn, s);
    };
    // The operations on one half of a slab, with the reads of the next half and the loads of a later slab spread
    // between them: issued in a row they would hold the operations behind them back.
    const auto half = [&](const Set &f, auto load, int load_to, auto read, Set &next, int which, int s) {
        constexpr int kReads = C::kTn + C::kTm, kReadsRow = (kReads + C::kTm - 3) / (C::kTm - 2);
        each<C::kTm>([&](auto row) {
            constexpr int i = decltype(row)::value;
            if constexpr (decltype(read)::value)
                each<kReadsRow>([&](auto n) {
                    constexpr int j = i * kReadsRow + decltype(n)::value;
                    if constexpr (j < kReads)
                        read_one(next, j, which, s);
                });
            if constexpr (decltype(load)::value) {
                constexpr int from = i * kLoads / C::kTm, to = (i + 1) * kLoads / C::kTm;
                each<to - from>([&](auto n) {
                    stage_one(from + decltype(n)::value, lds0 + load_to * C::kBufBytes);
                });
            }
#pragma unroll
            for (int j = 0; j < C::kTn; ++j)
                acc[i][j] = MM::mma(f.f[j], f.f[C::kTn + i], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (decltype(load)::value)
            staged();
    };
    const std::true_type yes;
    const std::false_type no;
    // A slab's two halves are read one half ahead of the operations on them. Between the halves the buffer has
    // been read by all (the barrier), and the slab after the next is loaded into it.
    if (begin < end) {
        enter(begin - seg * per);
        stage(0);
        if (begin + 1 < end) {
            stage(1);
            asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
        } else {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        }
        __syncthreads();
        Set even, odd;
#pragma unroll
        for (int j = 0; j < C::kTn + C::kTm; ++j)
            read_one(even, j, 0, 0);
        const auto handed_over = [] {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            __syncthreads();
        };
        int at = begin, cur = 0;
        for (; at + 2 < end; ++at, cur ^= 1) {
            half(even, no, 0, yes, odd, cur, 1);
            handed_over();
            half(odd, yes, cur, yes, even, cur ^ 1, 0);
        }
        if (at + 1 < end) {
            half(even, no, 0, yes, odd, cur, 1);
            handed_over();
            half(odd, no, 0, yes, even, cur ^ 1, 0);
            cur ^= 1;
        }
        half(even, no, 0, yes, odd, cur, 1);
        half(odd, no, 0, no, even, 0, 0);
    }

    // Results go through LDS, half the tile's rows at a time, so that a thread has eight neighbouring columns and
    // memory sees whole lines; and in a loop that is not unrolled: straight from the fragments the code was 60 KiB,
    // fetched once by every block (hidden gradient of 500 rows, 420 -> 1111: 32 us, 24 us so; of 8192
    // rows, 1024 -> 2816: 208 us, 104 us so).
    // Lane l of fragment (i, j) holds row 16 i + l % 16 and the wave's columns w_row(j, 4 (l / 16) + 0..3).
    constexpr int kPitch = C::kPitch, kHalf = C::kTm / 2, kPieces = C::kCols / 8;
    constexpr int kPer = BM / 2 * kPieces / C::kThreads;
    typedef decltype(Acc()[0] + Acc()[0]) Value;
    Value *const out = reinterpret_cast<Value *>(lds);
    const auto place = [&](int c, int h, int &r, int &col, int64_t &m, int &n) {
        const int at = c * C::kThreads + threadIdx.x, piece = at % kPieces;
        r = at / kPieces;
        col = EPI == kMmGate ? piece / 4 * 64 + piece % 4 * 8 : piece * 8;
        m = m0 + r / (kHalf * 16) * (BM / WM) + h * kHalf * 16 + r % (kHalf * 16);
        n = n0 + piece * 8;
    };
    // a thread's columns are the same in every piece of its rows
    static_assert(C::kThreads % kPieces == 0);
    Int8Columns<8> columns;
    if constexpr (EPI == kMmInt8)
        columns.load(p, n0 + static_cast<int>(threadIdx.x) % kPieces * 8);
    const auto lay_out = [&](auto part) {
        constexpr int h = decltype(part)::value;
        each<kHalf>([&](auto row) {
            constexpr int i = decltype(row)::value;
#pragma unroll
            for (int j = 0; j < C::kTn; ++j)
                *reinterpret_cast<Acc *>(out + (wm * kHalf * 16 + i * 16 + lane % 16) * kPitch + wn * C::kWn +
                                         w_row<C::kMap>(j, 4 * (lane / 16))) = acc[h * kHalf + i][j];
        });
    };
#pragma unroll 1
    for (int h = 0; h < 2; ++h) {
        __syncthreads();               // the readers of the fragments, or of the first half, are done
        if (h == 0)
            lay_out(std::integral_constant<int, 0>());
        else
            lay_out(std::integral_constant<int, 1>());
        __syncthreads();
        int r, col, n;
        int64_t m;
        // the gate's gradient needs g and u: the next piece's are on their way while one is worked on
        SavedPiece ahead = {};
        const auto fetch = [&](int c) {
            place(c, h, r, col, m, n);
            if (m < p.m && n < p.n8)
                ahead.load(p, m, n);
        };
        const bool whole = p.slices == 1;
        if (EPI == kMmGateBack && whole)
            fetch(0);
        constexpr int kUnroll = EPI == kMmGate || EPI == kMmGateBack ? 1 : 4;
#pragma unroll kUnroll
        for (int c = 0; c < kPer; ++c) {
            const SavedPiece saved = ahead;
            if (EPI == kMmGateBack && whole && c + 1 < kPer)
                fetch(c + 1);
            place(c, h, r, col, m, n);
            if (m >= p.m || n >= p.n8)
                continue;
            Value v[8], v2[8];
#pragma unroll
            for (int e = 0; e < 8; e += 4) {
                const Acc q = *reinterpret_cast<const Acc *>(out + r * kPitch + col + e);
                v[e] = q[0], v[e + 1] = q[1], v[e + 2] = q[2], v[e + 3] = q[3];
                if constexpr (EPI == kMmGate) {
                    const Acc q2 = *reinterpret_cast<const Acc *>(out + r * kPitch + col + 32 + e);
                    v2[e] = q2[0], v2[e + 1] = q2[1], v2[e + 2] = q2[2], v2[e + 3] = q2[3];
                }
            }
            if (!whole) {
                constexpr int kMats = EPI == kMmGate ? 2 : 1;
                Value *const to = static_cast<Value *>(p.part) + (static_cast<int64_t>(slice) * kMats * p.m + m) * p.n8 + n;
#pragma unroll
                for (int e = 0; e < 8; e += 4) {
                    *reinterpret_cast<Acc *>(to + e) = Acc{v[e], v[e + 1], v[e + 2], v[e + 3]};
                    if constexpr (EPI == kMmGate)
                        *reinterpret_cast<Acc *>(to + static_cast<int64_t>(p.m) * p.n8 + e) = Acc{v2[e], v2[e + 1], v2[e + 2], v2[e + 3]};
                }
            } else if constexpr (EPI == kMmGate) {
                finish_gate<MM::kExact>(p, m, n, v, v2);
            } else if constexpr (EPI == kMmGateBack) {
                float g[8], u[8];
                saved.values(p, g, u);
                finish_gate_back<MM::kExact>(p, m, n, v, g, u);
            } else if constexpr (EPI == kMmInt8) {
                finish_int8<8>(p, m, n, v, columns);
            } else {
                finish_store<8>(p, m, n, v);
            }
        }
    }
}

template <class MM, int EPI, int XL, int WL, int BM, int BN, int WM, int WN, bool TAIL>
__global__ void __launch_bounds__(WM *WN * 64) k_mm(MmParams p)
{
    mm_block<MM, EPI, XL, WL, BM, BN, WM, WN, TAIL>(p, blockIdx.x);
}
// Two products side by side.
template <class MM, int EPI, int XL, int WL, int BM, int BN, int WM, int WN, bool TAIL>
__global__ void __launch_bounds__(WM *WN * 64) k_mm_pair(MmPair pair)
{
    const int first = pair.blocks[0], second = static_cast<int>(blockIdx.x) >= first;
    mm_block<MM, EPI, XL, WL, BM, BN, WM, WN, TAIL>(pair.p[second], static_cast<int>(blockIdx.x) - (second ? first : 0));
}

template <class MM, int EPI, int XL, int WL, int BM, int BN, int WM, int WN, bool TAIL>
hipError_t launch_mm_tail(const MmParams &p, unsigned blocks, hipStream_t st)
{
    typedef Mm<MM, EPI, XL, WL, BM, BN, WM, WN> C;
    const auto kernel = k_mm<MM, EPI, XL, WL, BM, BN, WM, WN, TAIL>;
    const hipError_t ready = allow_lds(reinterpret_cast<const void *>(kernel), C::kLds);
    if (ready != hipSuccess)
        return ready;
    kernel<<<blocks, C::kThreads, C::kLds, st>>>(p);
    return hipGetLastError();
}

// Fills in p's tiles; the number of its blocks, or 0 where a launch does not hold them.
template <class C, int BM>
int mm_blocks(MmParams &p)
{
    p.tiles_m = (p.m + BM - 1) / BM;
    p.tiles_n = (p.n + C::kCols - 1) / C::kCols;
    const int64_t blocks = static_cast<int64_t>(p.tiles_m) * p.tiles_n * p.slices;
    return blocks * C::kThreads >= int64_t{1} << 32 ? 0 : static_cast<int>(blocks);
}

template <class MM, int EPI, int XL, int WL, int BM, int BN, int WM, int WN>
hipError_t launch_mm_tile(MmParams p, hipStream_t st)
{
    typedef Mm<MM, EPI, XL, WL, BM, BN, WM, WN> C;
    const int n = mm_blocks<C, BM>(p);
    if (n == 0)
        return hipErrorInvalidConfiguration;
    return p.k % C::kSlab ? launch_mm_tail<MM, EPI, XL, WL, BM, BN, WM, WN, true>(p, n, st)
                          : launch_mm_tail<MM, EPI, XL, WL, BM, BN, WM, WN, false>(p, n, st);
}

// Both products have one k.
template <class MM, int EPI, int XL, int WL, int BM, int BN, int WM, int WN>
hipError_t launch_mm_tile_pair(MmPair pair, hipStream_t st)
{
    typedef Mm<MM, EPI, XL, WL, BM, BN, WM, WN> C;
    for (int i = 0; i < 2; ++i)
        if ((pair.blocks[i] = mm_blocks<C, BM>(pair.p[i])) == 0)
            return hipErrorInvalidConfiguration;
    const auto run = [&](auto kernel) {
        const hipError_t ready = allow_lds(reinterpret_cast<const void *>(kernel), C::kLds);
        if (ready != hipSuccess)
            return ready;
        kernel<<<pair.blocks[0] + pair.blocks[1], C::kThreads, C::kLds, st>>>(pair);
        return hipGetLastError();
    };
    return pair.p[0].k % C::kSlab ? run(k_mm_pair<MM, EPI, XL, WL, BM, BN, WM, WN, true>)
                                  : run(k_mm_pair<MM, EPI, XL, WL, BM, BN, WM, WN, false>);
}

}  // namespace

}  // namespace enova
