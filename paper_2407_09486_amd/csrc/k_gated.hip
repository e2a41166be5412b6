// Products of the gated feed-forward block (mm_core.h), the finish of those cut into slices, and the bf16
// operands that products of fp32 or unaligned matrices are made from.
//
// An fp32 operand is three bf16 parts, which hold its 24 bits from 2^-110 up (below, the third ends under bf16's
// smallest number), and its product six products of parts, smallest first (a1 b3, a3 b1, a2 b2, a1 b2, a2 b1, a1 b1: what
// is left out is 2^-26 of it): errors against 64 bits are 5e-7 where the fp32 unit's product has 1.5e-6, at 1.3 times its
// rate (4096 rows, 1024 -> 2048, forward and gradients: 869 us). Two f16 parts under a power of two for each row or
// column, three products, took 707 us, but hold nothing below 2^-40 of the largest value along the reduction, where a
// small gradient may meet a large activation: not kept.
#include <algorithm>

#include "mm_core.h"

namespace enova {

namespace {

template <class MM, int EPI, int XL, int WL>
hipError_t launch_tile(const MmParams &p, int tile, hipStream_t st)
{
    if (tile == 256)
        return launch_mm_tile<MM, EPI, XL, WL, 256, 256, 2, 4>(p, st);
    return launch_mm_tile<MM, EPI, XL, WL, 128, 128, 2, 2>(p, st);
}
// An epilogue with activations has an instance for each type of block: both in one cost bf16 0.6 to 1.2% (minibatch 516
// -> 519 us, small batch 84.2 -> 85.2).
template <int EPI, int XL, int WL>
hipError_t launch_bf16(const MmParams &p, int tile, hipStream_t st)
{
    if constexpr (EPI == kMmGate || EPI == kMmGateBack)
        if (p.f32)
            return launch_tile<PartsMm, EPI, XL, WL>(p, tile, st);
    return launch_tile<Bf16Mm, EPI, XL, WL>(p, tile, st);
}

// Eight columns a thread.
template <int EPI, bool EXACT>
__device__ __forceinline__ void mm_finish(const MmParams &p, int64_t from)
{
    const int64_t i = (from + blockIdx.x) * 256 + threadIdx.x;
    const int per = p.n8 / 8;
    const int64_t m = i / per, plane = static_cast<int64_t>(p.m) * p.n8;
    const int n = static_cast<int>(i - m * per) * 8;
    if (m >= p.m)
        return;
    const int64_t at = m * p.n8 + n;
    if constexpr (EPI == kMmInt8) {
        const int *const part = static_cast<const int *>(p.part) + at;
        int v[8] = {};
#pragma unroll 4
        for (int s = 0; s < p.slices; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] += part[s * plane + e];
        Int8Columns<8> columns;
        columns.load(p, n);
        finish_int8<8>(p, m, n, v, columns);
    } else {
        constexpr int kMats = EPI == kMmGate ? 2 : 1;
        const float *const part = static_cast<const float *>(p.part) + at;
        float v[kMats][8] = {};
#pragma unroll 4
        for (int s = 0; s < p.slices; ++s)
#pragma unroll
            for (int k = 0; k < kMats; ++k) {
                float f[8];
                load8(part + (s * kMats + k) * plane, f);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    v[k][e] += f[e];
            }
        if constexpr (EPI == kMmGate) {
            finish_gate<EXACT>(p, m, n, v[0], v[1]);
        } else if constexpr (EPI == kMmGateBack) {
            float g[8], u[8];
            SavedPiece saved;
            saved.load(p, m, n);
            saved.values(p, g, u);
            finish_gate_back<EXACT>(p, m, n, v[0], g, u);
        } else {
            finish_store<8>(p, m, n, v[0]);
        }
    }
}

template <int EPI, bool EXACT>
__global__ void __launch_bounds__(256) k_mm_finish(MmParams p, int64_t from)
{
    mm_finish<EPI, EXACT>(p, from);
}
__global__ void __launch_bounds__(256) k_mm_finish_pair(MmPair pair)
{
    if (pair.p[blockIdx.y].slices > 1)
        mm_finish<kMmStore, false>(pair.p[blockIdx.y], 0);
}

__global__ void __launch_bounds__(256) k_zero(uint16_t *p, int64_t n)
{
    const int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x;
    if (i < n)
        p[i] = 0;
}

// Eight columns a thread; a block row for each matrix.
template <class T>
__global__ void __launch_bounds__(256) k_pack(PackJobs jobs, int64_t from)
{
    const PackJob j = jobs.job[blockIdx.y];
    const int64_t i = (from + blockIdx.x) * 256 + threadIdx.x;
    const int per = j.pitch / 8;
    const int64_t r = i / per;
    const int c = static_cast<int>(i - r * per) * 8;
    if (r >= j.rows)
        return;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] = c + e < j.cols ? static_cast<float>(static_cast<const T *>(j.src)[r * j.ld + c + e]) : 0.0f;
    store_operand<8>(static_cast<__bf16 *>(j.dst) + r * j.pitch + c, j.plane, v);
}

}  // namespace

// Time of a product by tile and slices, from what was measured for its parts (bf16, us): a slab of a 256-tile takes
// a compute unit 1.45; of a 128-tile 0.55 where the unit has one, 0.86 where it has two (both operands in columns:
// 0.75 and 1.15); a block's start and end 11 and 9; what a product moves beside its operands (`moves` bytes an output)
// at 5 TB/s, half hidden where two blocks share a unit; `alone`, what its finish takes longer in a tile's few waves than
// in the finishing launch; that launch 4, 0.12 a slice, and its traffic at 4 TB/s.
MmPlan mm_plan(int64_t m, int64_t n, int64_t slabs, bool columns, double moves, double alone)
{
    MmPlan best{128, 1, 0};
    double least = 1e30;
    for (const int tile : {256, 128}) {
        const int64_t tiles = ((m + tile - 1) / tile) * ((n + tile - 1) / tile), room = tile == 256 ? 256 : 512;
        for (int64_t slices = 1; slices <= 64 && slices * 2 <= std::max<int64_t>(slabs, 2); ++slices) {
            const int64_t blocks = tiles * slices, rounds = (blocks + room - 1) / room;
            if (blocks * (tile == 256 ? 512 : 256) >= int64_t{1} << 32)      // more threads than a launch holds
                break;
            const double one = tile == 256 ? 1.45 : (blocks <= 256 ? 0.55 : 0.86) * (columns ? 1.35 : 1.0);
            const double mn = static_cast<double>(m) * static_cast<double>(n), used = std::min<double>(1.0, blocks / 256.0);
            double us = static_cast<double>(rounds) * (static_cast<double>((slabs + slices - 1) / slices) * one + (tile == 256 ? 11.0 : 9.0));
            const int64_t part = slices > 1 ? slices * m * ((n + 15) / 16 * 16) : 0;
            if (slices > 1)
                us += 4.0 + 0.12 * static_cast<double>(slices) + (static_cast<double>(part) * 8 + mn * moves) / 4e6;
            else
                us += mn * moves / (5e6 * used) * (tile == 256 || blocks <= 256 ? 1.0 : 0.5) + (rounds == 1 ? alone : 0.0);
            if (us < least) {
                least = us;
                best = {tile, static_cast<int>(slices), part};
            }
        }
    }
    return best;
}

hipError_t launch_mm_bf16(const MmParams &p, MmEpilogue epi, int x_layout, int w_layout, int tile, hipStream_t st)
{
    if (epi == kMmGate && x_layout == kMmRows && w_layout == kMmRows)
        return launch_bf16<kMmGate, kMmRows, kMmRows>(p, tile, st);
    if (epi == kMmGateBack && x_layout == kMmRows && w_layout == kMmCols)
        return launch_bf16<kMmGateBack, kMmRows, kMmCols>(p, tile, st);
    if (epi == kMmStore && x_layout == kMmRows && w_layout == kMmRows)
        return launch_bf16<kMmStore, kMmRows, kMmRows>(p, tile, st);
    if (epi == kMmStore && x_layout == kMmRows && w_layout == kMmCols)
        return launch_bf16<kMmStore, kMmRows, kMmCols>(p, tile, st);
    if (epi == kMmStore && x_layout == kMmCols && w_layout == kMmCols)
        return launch_bf16<kMmStore, kMmCols, kMmCols>(p, tile, st);
    return hipErrorInvalidValue;
}

static int64_t mm_plan_blocks(const MmParams &p, const MmPlan &plan)
{
    return static_cast<int64_t>((p.m + plan.tile - 1) / plan.tile) * ((p.n + plan.tile - 1) / plan.tile) * plan.slices;
}

bool mm_pairs(const MmParams &a, const MmPlan &pa, const MmParams &b, const MmPlan &pb)
{
    return pa.tile == pb.tile && a.k == b.k && a.segments == b.segments &&
           mm_plan_blocks(a, pa) + mm_plan_blocks(b, pb) <= (pa.tile == 256 ? 256 : 512);
}

hipError_t launch_mm_pair(const MmPair &pair, int tile, hipStream_t st)
{
    const hipError_t e = tile == 256 ? launch_mm_tile_pair<Bf16Mm, kMmStore, kMmCols, kMmCols, 256, 256, 2, 4>(pair, st)
                                     : launch_mm_tile_pair<Bf16Mm, kMmStore, kMmCols, kMmCols, 128, 128, 2, 2>(pair, st);
    int64_t pieces = 0;
    for (const MmParams &p : pair.p)
        if (p.slices > 1)
            pieces = std::max(pieces, static_cast<int64_t>(p.m) * (p.n8 / 8));
    if (e != hipSuccess || pieces == 0)
        return e;
    k_mm_finish_pair<<<dim3(static_cast<unsigned>((pieces + 255) / 256), 2), 256, 0, st>>>(pair);
    return hipGetLastError();
}

hipError_t launch_mm_finish(const MmParams &p, MmEpilogue epi, hipStream_t st)
{
    const auto run = [&](auto kernel) {
        return launch_in_runs((static_cast<int64_t>(p.m) * (p.n8 / 8) + 255) / 256, 256, [&](int64_t from, unsigned n) {
            kernel<<<n, 256, 0, st>>>(p, from);
        });
    };
    switch (epi) {
    case kMmGate: return p.f32 ? run(k_mm_finish<kMmGate, true>) : run(k_mm_finish<kMmGate, false>);
    case kMmGateBack: return p.f32 ? run(k_mm_finish<kMmGateBack, true>) : run(k_mm_finish<kMmGateBack, false>);
    case kMmInt8: return run(k_mm_finish<kMmInt8, false>);
    default: return run(k_mm_finish<kMmStore, false>);
    }
}

hipError_t launch_zero(void *p, int64_t bytes, hipStream_t st)
{
    return launch_in_runs((bytes / 2 + 255) / 256, 256, [&](int64_t from, unsigned n) {
        k_zero<<<n, 256, 0, st>>>(static_cast<uint16_t *>(p) + from * 256, bytes / 2 - from * 256);
    });
}

hipError_t launch_pack(const PackJobs &jobs, int dtype, hipStream_t st)
{
    int64_t most = 0;
    for (int i = 0; i < jobs.n; ++i)
        most = std::max(most, (jobs.job[i].rows * (jobs.job[i].pitch / 8) + 255) / 256);
    return launch_in_runs(most, 256, [&](int64_t from, unsigned n) {
        if (dtype == ENOVA_F32)
            k_pack<float><<<dim3(n, jobs.n), 256, 0, st>>>(jobs, from);
        else
            k_pack<__bf16><<<dim3(n, jobs.n), 256, 0, st>>>(jobs, from);
    });
}

}  // namespace enova
