// Internal declarations of the residual gated block's operators (include/enova_block.h).
#pragma once

#include "enova_block.h"
#include "internal.h"

namespace enova {

// A launch holds fewer than 2^32 threads: a longer grid goes in runs of 2^31, launch(first block, blocks) each.
template <class F>
hipError_t launch_in_runs(int64_t blocks, int threads, F launch)
{
    const int64_t run = (int64_t{1} << 31) / threads;
    for (int64_t from = 0; from < blocks; from += run) {
        launch(from, static_cast<unsigned>(blocks - from < run ? blocks - from : run));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess)
            return e;
    }
    return hipSuccess;
}

// 16 bytes at any address: the hardware's loads and stores take it.
struct __attribute__((packed, aligned(1))) Any16 {
    uint4 v;
};

// ---------------------------------------------------------------------------------------------
// AdamW
// ---------------------------------------------------------------------------------------------
constexpr int kAdamThreads = 256;
constexpr int kAdamBlock = 256;        // elements that share the scales of 8-bit states: a wave's four a lane
constexpr int kAdamChunk = 4096;       // elements of a thread block

struct AdamTensor {
    void *param;
    const void *grad;
    void *copy, *m, *v;
    float *m_scale, *v_scale;
    int64_t numel;
    int32_t wide;                      // every buffer is aligned for four elements at a time
};
struct AdamChunk {
    int32_t tensor, index;
};
struct AdamValues {
    float *m, *v;
    int32_t wide;
};
struct AdamArgs {
    float b1, b1c, b2, b2c;            // b and 1 - b
    float keep, lr, root, eps;         // 1 - lr decay, lr / (1 - b1^n), 1 / sqrt(1 - b2^n)
    float grad_scale;
    uint32_t step;
};
hipError_t launch_adamw(int bits, int param_dtype, int grad_dtype, const AdamTensor *t, const AdamChunk *c, int n,
                        const AdamArgs &a, hipStream_t st);
// New pointers of up to kAdamPointers entries of a table, as arguments of a launch: nothing of the host's is read
// after the call.
constexpr int kAdamPointers = 64;
struct AdamPointers {
    int from, n;
    uint64_t wide;                     // a bit an entry
    const void *a[kAdamPointers];
    void *b[kAdamPointers];
};
hipError_t launch_adamw_grads(AdamTensor *t, const AdamPointers &p, hipStream_t st);     // a: gradients
hipError_t launch_adamw_values(AdamValues *v, const AdamPointers &p, hipStream_t st);    // a, b: m and v
hipError_t launch_adamw_states(const AdamTensor *t, const AdamChunk *c, int n, const AdamValues *v, hipStream_t st);

// ---------------------------------------------------------------------------------------------
// Norms, gate and residual scale
// ---------------------------------------------------------------------------------------------
struct NormParams {
    const void *residual, *branch;
    int64_t rows;
    int model;
    int layer;
    float eps, keep, scale;
    int64_t group;                     // rows that share a gate row (gate != NULL)
    const float *post, *post_bias, *pre, *pre_bias, *gate;
    float *stats;                      // [rows][4]: mean and factor of the branch, mean and factor of res
    // forward
    void *res, *out;
    // backward
    const void *dres, *dout;
    void *dresidual, *dbranch;
    // Sums over rows. The rows are cut into items of at most item_rows (an item never crosses a gate
    // row), a team of threads takes a run of consecutive items, and a block leaves its teams' sums in
    // part [blocks][kNormSums][model]; gate sums are left per item (gate_part: dgate itself where an item is
    // a whole group; NULL: not asked for).
    int item_rows;
    int64_t items_per_group, items, items_per_team;
    float *part;
    float *gate_part;
    unsigned want;                     // bit i: sum i of kNormSums is asked for
};
constexpr int kNormSums = 4;           // post, post_bias, pre, pre_bias
constexpr int kNormWidest = 16384;
// How many threads take a row of this width: a wave or a part of one (256 threads a block), or a block.
int norm_team(int model);
hipError_t launch_resnorm_forward(const NormParams &p, int dtype, hipStream_t st);
hipError_t launch_resnorm_backward(const NormParams &p, int dtype, int64_t blocks, hipStream_t st);
// n > 1: out[i][c] = sum over j < total of src[i][j * stride + c]. n = 1: out[0][y * model + c] = sum over
// y per <= j < min((y + 1) per, total) of src[0][j * stride + c] for y < rows.
struct NormSumJobs {
    int n = 0;
    const float *src[kNormSums] = {};
    float *out[kNormSums] = {};
};
hipError_t launch_norm_sums(const NormSumJobs &jobs, int64_t stride, int64_t per, int64_t total, int64_t rows, int model,
                            hipStream_t st);

// ---------------------------------------------------------------------------------------------
// Matrix products (mm_core.h): C(m, n) = sum over segments s, k < K of X_s(m, k) W_s(n, k)
// ---------------------------------------------------------------------------------------------
// A product whose operands are several matrices one behind the other along the reduction: the two halves
// of the gated block's input gradient, and the six products of three bf16 parts that stand for an fp32 one.
constexpr int kMmSegments = 12;
enum MmEpilogue {
    kMmStore = 0,        // C
    kMmGate,             // h = act(g) u from both projections at once (and g, u)
    kMmGateBack,         // C is dh: dg and du from it and the saved g and u
    kMmInt8,             // C sx[m] sw[n] + bias[n] from 32-bit integers
};
struct MmParams {
    const void *x[kMmSegments], *w[kMmSegments];
    const void *w2[kMmSegments];       // kMmGate: the second projection (w: the first)
    int segments;
    int64_t ldx, ldw;                  // bytes between rows as they are stored
    int m, n, k;                       // k: of a segment, in elements. kMmGate: n columns of either projection
    int n8;                            // n rounded up to 8: kMmGate and kMmGateBack write the columns past n as zeros
    int tiles_m, tiles_n;
    // The reduction's slices. More than one: the product leaves 32-bit partial sums in
    // part [slices][kMmGate: 2][m][n8], and launch_mm_finish does the rest.
    int slices;
    void *part;
    int act;
    // outputs. kMmGate: c = h; kMmGateBack: c = dg, c2 = du; kMmStore: rows from m2 on go to c2 (0: none do)
    void *c, *c2;
    int64_t ldc;                       // elements
    int m2, m1;                        // kMmStore: rows m1 .. m2 - 1 are padding and written nowhere
    int64_t plane;                     // elements between the three bf16 parts of an fp32 operand (0: bf16)
    float *h32;                        // kMmGate of few rows of fp32: h in fp32, pitch ldg (c may then be NULL)
    int f32;                           // the handle's type, and c's (kMmStore, kMmInt8): fp32 instead of bf16
    int wide;                          // rows of c are aligned for eight elements at a time
    // saved projections, pitch ldg, zeros past n: fp32, or where ge and ue are there f16 with an exponent for every
    // eight neighbouring columns (pitch ldg / 8)
    void *g, *u;
    int8_t *ge, *ue;
    int64_t ldg;
    const float *sx, *sw, *bias;
};
struct MmPair {
    MmParams p[2];
    int blocks[2];
};
// Layout of an operand: its rows hold the reduction (as stored for y = x W^T), or its columns do.
enum { kMmRows = 0, kMmCols = 1 };
// A product's tile and how many slices its reduction is cut into; n counts both projections of a gate.
struct MmPlan {
    int tile;                          // 256 or 128, both ways
    int slices;
    int64_t part;                      // 32-bit words of partial sums
};
MmPlan mm_plan(int64_t m, int64_t n, int64_t slabs, bool columns, double moves, double alone);
// Lets a kernel use so much dynamic LDS on the current device (asked for once a kernel and device).
hipError_t allow_lds(const void *kernel, int bytes);
hipError_t launch_mm_bf16(const MmParams &p, MmEpilogue epi, int x_layout, int w_layout, int tile, hipStream_t st);
hipError_t launch_mm_int8(const MmParams &p, int tile, hipStream_t st);
// Two stored products of one reduction over operands in columns, in one launch (and one to finish them), where their
// blocks, of one tile, run side by side in one round: mm_pairs.
bool mm_pairs(const MmParams &a, const MmPlan &pa, const MmParams &b, const MmPlan &pb);
hipError_t launch_mm_pair(const MmPair &pair, int tile, hipStream_t st);
// The sum of a product's slices in their order, and what the product itself would have done with it.
hipError_t launch_mm_finish(const MmParams &p, MmEpilogue epi, hipStream_t st);
// The same products for few rows (p.m <= kMmFewRows, both operands in rows, one segment of the caller's own
// matrices in any alignment; fp32 ones are taken apart in registers). dtype: of the operands.
constexpr int kMmFewRows = 64;
hipError_t launch_mm_few(const MmParams &p, MmEpilogue epi, int dtype, hipStream_t st);
// Zeros (a kernel: a caller's graph may hold it).
hipError_t launch_zero(void *p, int64_t bytes, hipStream_t st);
// dst [parts][rows][pitch] bf16 from src [rows][cols] (pitch ld): bf16 copied, fp32 in three parts `plane`
// elements apart; columns cols .. pitch - 1 are zero. pitch is a multiple of 8. All jobs in one launch.
struct PackJob {
    const void *src;
    int64_t ld, rows;
    int cols, pitch;
    void *dst;
    int64_t plane;
};
constexpr int kPackJobs = 5;
struct PackJobs {
    int n = 0;
    PackJob job[kPackJobs];
};
hipError_t launch_pack(const PackJobs &jobs, int dtype, hipStream_t st);
// The 8-bit product of a row that takes x as it is (every block makes the codes itself), where
// i8_fused(rows, pitch) says so.
bool i8_fused(int64_t rows, int pitch);
struct QuantParams {
    const void *x;
    int64_t ld;
    int cols, gate, dtype;
};
hipError_t launch_i8_fused(const MmParams &p, const QuantParams &q, hipStream_t st);
// 8-bit operands: q [rows][pitch] (zero past cols) and the scales of x [rows][ld], or of act(g) u from its halves.
hipError_t launch_quantize(const void *x, int dtype, int64_t ld, int64_t rows, int cols, int gate, int8_t *q, int pitch,
                           float *scale, hipStream_t st);

}  // namespace enova
