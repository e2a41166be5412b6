// A row of x as 8-bit codes: q = rint(127 x / max |x|), scale = max |x| / 127.
#pragma once

#include "mm_core.h"

namespace enova {

namespace {

// Eight values of a row from column c on (zeros past the end): x, or act(g) u where gate >= 0.
template <class T>
__device__ __forceinline__ void load_x8(const T *row, int c, int cols, float (&v)[8])
{
    if (c + 8 <= cols) {
        T e[8];
#pragma unroll
        for (int i = 0; i < static_cast<int>(sizeof(e) / 16); ++i) {
            const uint4 q = reinterpret_cast<const Any16 *>(row + c)[i].v;
            __builtin_memcpy(e + i * (16 / sizeof(T)), &q, 16);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = static_cast<float>(e[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = c + i < cols ? static_cast<float>(row[c + i]) : 0.0f;
    }
}
template <class T>
__device__ __forceinline__ void quant_values(const T *row, int c, int cols, int gate, float (&v)[8])
{
    load_x8(row, c, cols, v);
    if (gate >= 0) {
        float a[8], da[8], u[8];
        load_x8(row + cols, c, cols, u);
        gate_acts<false>(gate, v, a, da);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = a[i] * u[i];
    }
}
// The largest |v|, infinity where one is not finite.
__device__ __forceinline__ float quant_top(const float (&v)[8], float top)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float a = fabsf(v[i]);
        top = a < __builtin_inff() ? fmaxf(top, a) : __builtin_inff();
    }
    return top;
}
__device__ __forceinline__ uint2 quant_codes(const float (&v)[8], float top)
{
    const bool good = top < __builtin_inff();
    const float by = good && top > 0.0f ? top : 1.0f;
    uint32_t q[2] = {0u, 0u};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (good)
            q[i / 4] |= static_cast<uint32_t>(static_cast<int>(rintf(v[i] / by * 127.0f)) & 255) << (8 * (i % 4));
    return make_uint2(q[0], q[1]);
}
__device__ __forceinline__ float quant_scale(float top)
{
    return top < __builtin_inff() ? top * (1.0f / 127) : __builtin_nanf("");
}

// The maximum over a block of THREADS; shared: a float a wave.
template <int THREADS>
__device__ __forceinline__ float block_top(float top, float *shared)
{
#pragma unroll
    for (int d = 32; d > 0; d >>= 1)
        top = fmaxf(top, __shfl_xor(top, d));
    if ((threadIdx.x & 63) == 0)
        shared[threadIdx.x >> 6] = top;
    __syncthreads();
    top = shared[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w)
        top = fmaxf(top, shared[w]);
    return top;
}

}  // namespace

}  // namespace enova
