// Product in 8-bit integers with a scale for each row of x and each output (mm_core.h), and the rows'
// quantisation.
#include "quantize.h"

namespace enova {

namespace {

// A block takes a row, eight neighbouring values a thread at a time. Rows of up to KEEP pieces a thread stay in
// registers between the maximum and the codes; wider ones (KEEP = 0) are read again, from the caches.
template <class T, int THREADS, int KEEP>
__global__ void __launch_bounds__(THREADS) k_quantize(const T *x, int64_t ld, int cols, int gate, int8_t *q, int pitch, float *scale)
{
    __shared__ float shared[THREADS / 64];
    const int64_t row = blockIdx.x;
    const T *const src = x + row * ld;
    float v[KEEP ? KEEP : 1][8];
    float top = 0.0f;
    if constexpr (KEEP) {
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
            quant_values(src, (i * THREADS + static_cast<int>(threadIdx.x)) * 8, cols, gate, v[i]);
#pragma unroll
        for (int i = 0; i < KEEP; ++i)
            top = quant_top(v[i], top);
    } else {
        for (int c = threadIdx.x * 8; c < cols; c += THREADS * 8) {
            quant_values(src, c, cols, gate, v[0]);
            top = quant_top(v[0], top);
        }
    }
    top = block_top<THREADS>(top, shared);
    if constexpr (KEEP) {
#pragma unroll
        for (int i = 0; i < KEEP; ++i) {
            const int c = (i * THREADS + static_cast<int>(threadIdx.x)) * 8;
            if (c < pitch)
                *reinterpret_cast<uint2 *>(q + row * pitch + c) = quant_codes(v[i], top);
        }
    } else {
        for (int c = threadIdx.x * 8; c < pitch; c += THREADS * 8) {
            quant_values(src, c, cols, gate, v[0]);
            *reinterpret_cast<uint2 *>(q + row * pitch + c) = quant_codes(v[0], top);
        }
    }
    if (threadIdx.x == 0)
        scale[row] = quant_scale(top);
}

template <class T>
hipError_t quantize(const T *x, int64_t ld, int64_t rows, int cols, int gate, int8_t *q, int pitch, float *scale, hipStream_t st)
{
    const auto run = [&](auto kernel, int threads) {
        return launch_in_runs(rows, threads, [&](int64_t from, unsigned n) {
            kernel<<<n, threads, 0, st>>>(x + from * ld, ld, cols, gate, q + from * pitch, pitch, scale + from);
        });
    };
    if (pitch <= 2048)
        return run(k_quantize<T, 256, 1>, 256);
    if (pitch <= 4096)
        return run(k_quantize<T, 512, 1>, 512);
    if (pitch <= 8192)
        return run(k_quantize<T, 512, 2>, 512);
    return run(k_quantize<T, 512, 0>, 512);
}

}  // namespace

hipError_t launch_quantize(const void *x, int dtype, int64_t ld, int64_t rows, int cols, int gate, int8_t *q, int pitch,
                           float *scale, hipStream_t st)
{
    return dtype == ENOVA_F32 ? quantize(static_cast<const float *>(x), ld, rows, cols, gate, q, pitch, scale, st)
                              : quantize(static_cast<const __bf16 *>(x), ld, rows, cols, gate, q, pitch, scale, st);
}

hipError_t launch_mm_int8(const MmParams &p, int tile, hipStream_t st)
{
    if (tile == 256)
        return launch_mm_tile<Int8Mm, kMmInt8, kMmRows, kMmRows, 256, 256, 2, 4>(p, st);
    return launch_mm_tile<Int8Mm, kMmInt8, kMmRows, kMmRows, 128, 128, 2, 2>(p, st);
}

}  // namespace enova
