// Host side of the residual gated block's operators: argument checks, workspaces and launch sequences.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstring>
#include <limits>
#include <new>
#include <vector>

#include "block_internal.h"

using namespace enova;

namespace enova {

hipError_t allow_lds(const void *kernel, int bytes)
{
    // a small table without locks: an entry says which kernel, on which device, was asked for last in its place
    static std::atomic<uintptr_t> asked[512];
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess)
        return e;
    const uintptr_t key = reinterpret_cast<uintptr_t>(kernel) * 64 + static_cast<uintptr_t>(dev & 63) + 1;
    const size_t at = static_cast<size_t>(key * 0x9e3779b97f4a7c15ull >> 55);
    if (asked[at].load(std::memory_order_acquire) == key)
        return hipSuccess;
    e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == hipSuccess)
        asked[at].store(key, std::memory_order_release);      // two that share a place take turns asking again
    return e;
}

}  // namespace enova

namespace {

// Up to how many rows a product is taken by the kernels for few rows, whose blocks of 16 weight rows read all of x
// each: 64 where the tiles would need their operands packed first (fp32: 197 us for 64 rows through 4096 -> 8192,
// 437 for 65) or where the weights, one matrix's, are less than 8 MiB (8-bit, 1000 -> 8000: 11 us, tiles 14); 48 from
// there to 16 MiB, and 16 beyond, where x's traffic weighs more than a tile's launch (bf16, 4096 -> 8192: 46 us for 16
// rows, 57 for 32, 47 by tiles).
int few_rows(bool packed, int64_t weight_bytes)
{
    constexpr int64_t kMiB = int64_t{1} << 20;
    return packed || weight_bytes < 8 * kMiB ? kMmFewRows : weight_bytes <= 16 * kMiB ? 48 : 16;
}

constexpr int kWidest = 262144;
constexpr int64_t kMostRows = int64_t{1} << 30;

// A handle's device workspace: grows on demand, and is handed out in 256-byte aligned pieces. Launches that a graph
// captured hold its address, so a buffer that a captured call was given stays allocated until the handle goes.
struct Workspace {
    char *p = nullptr;
    size_t cap = 0;
    bool captured = false;             // by a call that was given p
    std::vector<char *> outgrown;

    ~Workspace()
    {
        (void)hipFree(p);
        for (char *q : outgrown)
            (void)hipFree(q);
    }
    enova_status need(size_t bytes, hipStream_t stream)
    {
        hipStreamCaptureStatus capturing = hipStreamCaptureStatusNone;
        if (hipStreamIsCapturing(stream, &capturing) != hipSuccess)
            (void)hipGetLastError();
        if (bytes <= cap) {
            captured |= capturing != hipStreamCaptureStatusNone;
            return ENOVA_OK;
        }
        if (capturing != hipStreamCaptureStatusNone)
            return fail(ENOVA_EINVAL, "the workspace has to grow to %zu bytes, which a stream under capture cannot: make one such call before", bytes);
        if (captured) {
            try {
                outgrown.push_back(p);
            } catch (const std::bad_alloc &) {
                return fail(ENOVA_ENOMEM, "host memory");
            }
        } else {
            (void)hipFree(p);          // waits for the work that uses it
        }
        p = nullptr;
        cap = 0;
        captured = false;
        const hipError_t e = hipMalloc(reinterpret_cast<void **>(&p), bytes);
        if (e != hipSuccess) {
            p = nullptr;
            (void)hipGetLastError();
            return fail(ENOVA_ENOMEM, "hipMalloc(%zu): %s", bytes, hipGetErrorString(e));
        }
        cap = bytes;
        return ENOVA_OK;
    }
};
// Lays pieces out first (base NULL: only sizes), then again over the workspace.
struct Carve {
    char *base = nullptr;
    size_t at = 0;
    template <class T>
    T *take(int64_t n)
    {
        T *q = base ? reinterpret_cast<T *>(base + at) : nullptr;
        at += (static_cast<size_t>(n) * sizeof(T) + 255) / 256 * 256;
        return q;
    }
};

bool aligned(const void *p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
int64_t up(int64_t n, int64_t to) { return (n + to - 1) / to * to; }

}  // namespace

#define ENOVA_TRY(expr, what)                    \
    do {                                         \
        const hipError_t e_ = (expr);            \
        if (e_ != hipSuccess)                    \
            return hip_fail(e_, what);           \
    } while (0)

struct enova_gated_s {
    int device = 0;
    enova_gated_config c{};
    Workspace ws;
};
struct enova_resnorm_s {
    int device = 0;
    enova_resnorm_config c{};
    Workspace ws;
};
struct enova_adamw_s {
    int device = 0;
    enova_adamw_config c{};
    std::vector<AdamTensor> host;
    int chunks = 0;
    char *table = nullptr;             // tensors, chunks, and the destinations of a states call
    AdamTensor *d_tensors = nullptr;
    AdamChunk *d_chunks = nullptr;
    AdamValues *d_values = nullptr;
};
struct enova_i8_s {
    int device = 0;
    enova_i8_config c{};
    const int8_t *w = nullptr;
    int64_t ldw = 0;
    const float *w_scale = nullptr, *bias = nullptr;
    Workspace ws;
};

// ------------------------------------------------------------------------------ gated block
namespace {

// A matrix as the products read it: bf16, rows of whole 16 bytes, `parts` planes for fp32.
struct Operand {
    const __bf16 *p = nullptr;
    int64_t ld = 0;                    // elements
    int64_t plane = 0;
};

// What a forward call keeps for the backward call, [rows][pitch] each: h as the products read it, and g and u, in fp32
// for fp32 blocks, else in f16 with an exponent for every eight columns.
struct Kept {
    __bf16 *h = nullptr;
    void *g = nullptr, *u = nullptr;
    int8_t *ge = nullptr, *ue = nullptr;
    static int64_t bytes(int64_t rows, int64_t pitch, bool f32) { return up(rows * pitch * (f32 ? 14 : 6) + (f32 ? 0 : rows * pitch / 4), 16); }
    Kept(void *base, int64_t rows, int64_t pitch, bool f32)
    {
        if (!base)
            return;
        const int64_t n = rows * pitch;
        char *at = static_cast<char *>(base);
        g = at;
        u = at + n * (f32 ? 4 : 2);
        h = reinterpret_cast<__bf16 *>(at + n * (f32 ? 8 : 4));
        if (!f32) {
            ge = reinterpret_cast<int8_t *>(at + n * 6);
            ue = ge + n / 8;
        }
    }
    void tell(MmParams &p, int64_t pitch) const
    {
        p.g = g;
        p.u = u;
        p.ge = ge;
        p.ue = ue;
        p.ldg = pitch;
    }
};

// The six products of three bf16 parts (largest first) that make an fp32 product, smallest first.
constexpr int kPartX[6] = {2, 0, 1, 1, 0, 0}, kPartW[6] = {0, 2, 1, 0, 1, 0};

struct GatedCall {
    enova_gated op;
    hipStream_t st;
    int T, D, F, D8, F8;
    bool f32;
    Carve carve;
    PackJobs jobs;

    GatedCall(enova_gated o, int64_t rows, hipStream_t s)
        : op(o), st(s), T(static_cast<int>(rows)), D(o->c.model), F(o->c.hidden), D8(static_cast<int>(up(D, 8))),
          F8(static_cast<int>(up(F, 8))), f32(o->c.dtype == ENOVA_F32)
    {
    }
    int parts() const { return f32 ? 3 : 1; }
    // (a tile's rows have to lie within 2^31 bytes)
    bool packs(const void *src, int64_t ld, int cols) const
    {
        return f32 || ld % 8 || cols % 8 || !aligned(src, 16) || ld > (int64_t{1} << 22);
    }
    // src [rows][cols] as an operand, packed (by pack()) where the products cannot read it
    Operand operand(const void *src, int64_t ld, int64_t rows, int cols)
    {
        if (!packs(src, ld, cols))
            return {static_cast<const __bf16 *>(src), ld, 0};
        const int pitch = static_cast<int>(up(cols, 8));
        __bf16 *dst = carve.take<__bf16>(parts() * rows * pitch);
        const int64_t plane = f32 ? rows * pitch : 0;
        jobs.job[jobs.n++] = {src, ld, rows, cols, pitch, dst, plane};
        return {dst, pitch, plane};
    }
    // Queues the packing (on the second pass over the workspace).
    hipError_t pack()
    {
        const hipError_t e = carve.base ? launch_pack(jobs, op->c.dtype, st) : hipSuccess;
        jobs.n = 0;
        return e;
    }
    Operand own(int64_t rows, int64_t pitch)
    {
        Operand o{carve.take<__bf16>(parts() * rows * pitch), pitch, f32 ? rows * pitch : 0};
        return o;
    }
    // Adds X W's products to p's segments.
    void segments(MmParams &p, const Operand &x, const Operand &w, const Operand *w2 = nullptr) const
    {
        for (int i = f32 ? 0 : 5; i < 6; ++i) {
            p.x[p.segments] = x.p + kPartX[i] * x.plane;
            p.w[p.segments] = w.p + kPartW[i] * w.plane;
            p.w2[p.segments] = w2 ? w2->p + kPartW[i] * w2->plane : nullptr;
            ++p.segments;
        }
        p.ldx = x.ld * 2;
        p.ldw = w.ld * 2;
    }
    MmParams params(int m, int n, int k) const
    {
        MmParams p{};
        p.m = m;
        p.n = n;
        p.k = k;
        p.n8 = static_cast<int>(up(n, 8));
        p.slices = 1;
        p.act = op->c.act;
        p.f32 = f32;
        return p;
    }
    void output(MmParams &p, void *c, int64_t ldc) const
    {
        p.c = c;
        p.ldc = ldc;
        p.wide = ldc % 8 == 0 && aligned(c, 16);
    }
    int64_t slabs(const MmParams &p) const { return up(p.k, 64) / 64 * p.segments; }

    // Bytes a product moves for each of its outputs beside its operands (kMmGate: an output of either projection).
    double moved(const MmParams &p, MmEpilogue epi) const
    {
        const double operand = 2.0 * parts();
        const double kept = f32 ? 8.0 : 4.25;
        return epi == kMmGate ? (operand + (p.g ? kept : 0.0)) / 2 : epi == kMmGateBack ? kept + 2 * operand : f32 ? 4.0 : 2.0;
    }
    // The next product's plan: made in the first pass over the workspace, kept for the second.
    const MmPlan &next_plan(const MmParams &p, MmEpilogue epi, int x_layout)
    {
        MmPlan &plan = plans[products++];
        if (!carve.base)
            plan = mm_plan(p.m, epi == kMmGate ? 2 * static_cast<int64_t>(p.n8) : p.n, slabs(p), x_layout == kMmCols,
                           moved(p, epi), epi == kMmGateBack ? 6.0 : epi == kMmGate ? 2.0 : 0.0);
        return plan;
    }
    // Queues a product (on the second pass), whole or in slices. Products run one after the other: they share the
    // partial sums' place.
    hipError_t product(MmParams p, MmEpilogue epi, int x_layout, int w_layout)
    {
        const MmPlan plan = next_plan(p, epi, x_layout);
        p.slices = plan.slices;
        const size_t mark = carve.at;
        p.part = plan.part ? carve.take<float>(plan.part) : nullptr;
        most = std::max(most, carve.at);
        carve.at = mark;
        if (!carve.base)
            return hipSuccess;
        const hipError_t e = launch_mm_bf16(p, epi, x_layout, w_layout, plan.tile, st);
        return e == hipSuccess && p.slices > 1 ? launch_mm_finish(p, epi, st) : e;
    }
    // Two stored products of operands in columns, together where they fit.
    hipError_t pair(MmParams a, MmParams b)
    {
        const MmPlan pa = next_plan(a, kMmStore, kMmCols), pb = next_plan(b, kMmStore, kMmCols);
        if (!mm_pairs(a, pa, b, pb)) {
            products -= 2;
            const hipError_t e = product(a, kMmStore, kMmCols, kMmCols);
            return e == hipSuccess ? product(b, kMmStore, kMmCols, kMmCols) : e;
        }
        const size_t mark = carve.at;
        a.slices = pa.slices;
        b.slices = pb.slices;
        a.part = pa.part ? carve.take<float>(pa.part) : nullptr;
        b.part = pb.part ? carve.take<float>(pb.part) : nullptr;
        most = std::max(most, carve.at);
        carve.at = mark;
        return carve.base ? launch_mm_pair(MmPair{{a, b}, {0, 0}}, pa.tile, st) : hipSuccess;
    }
    // h (and g, u where they are asked for) from x
    hipError_t gate(const Operand &x, const Operand &wg, const Operand &wu, const Operand &h, const Kept &kept)
    {
        MmParams p = params(T, F, D);
        segments(p, x, wg, &wu);
        p.c = const_cast<__bf16 *>(h.p);
        p.ldc = h.ld;
        p.plane = h.plane;
        kept.tell(p, F8);
        return product(p, kMmGate, kMmRows, kMmRows);
    }
    // Ends the first pass: the workspace is there, and the products' plans are known.
    enova_status lay_out()
    {
        const enova_status s = op->ws.need(std::max<size_t>(most, 256), st);
        carve = {op->ws.p, 0};
        products = 0;
        return s;
    }
    size_t most = 0;
    MmPlan plans[5] = {};              // of the first pass, in the second's order
    int products = 0;
};

// The launches of a backward call; over no workspace yet, what they need of one.
struct GatedBackward {
    const void *x;
    int64_t ldx;
    const void *wg, *wu, *wd;
    const float *saved;
    const void *dy;
    int64_t lddy;
    void *dx;
    int64_t lddx;
    void *dwg, *dwu, *dwd;

    enova_status queue(GatedCall &g) const
    {
        const int64_t rows = g.T;
        const Operand ox = g.operand(x, ldx, rows, g.D), oy = g.operand(dy, lddy, rows, g.D),
                      og = g.operand(wg, g.D, g.F, g.D), ou = g.operand(wu, g.D, g.F, g.D),
                      od = g.operand(wd, g.F, g.D, g.F);
        ENOVA_TRY(g.pack(), "pack");
        const Operand dgu = g.own(rows, 2 * g.F8);     // [dg | du]
        Operand dg = dgu, du = dgu;
        du.p += g.F8;
        const Kept kept(saved ? const_cast<float *>(saved) : reinterpret_cast<float *>(g.carve.take<char>(Kept::bytes(rows, g.F8, g.f32))),
                        rows, g.F8, g.f32);
        const Operand h{kept.h, g.F8, g.f32 ? rows * g.F8 : 0};
        g.most = std::max(g.most, g.carve.at);
        if (!saved)
            ENOVA_TRY(g.gate(ox, og, ou, h, kept), "gate product");
        {
            MmParams p = g.params(g.T, g.F, g.D);
            g.segments(p, oy, od);
            p.c = const_cast<__bf16 *>(dg.p);
            p.c2 = const_cast<__bf16 *>(du.p);
            p.ldc = dgu.ld;
            p.plane = dgu.plane;
            kept.tell(p, g.F8);
            ENOVA_TRY(g.product(p, kMmGateBack, kMmRows, kMmCols), "hidden gradient");
        }
        if (dx) {
            MmParams p = g.params(g.T, g.D, g.F);
            g.segments(p, dg, og);
            g.segments(p, du, ou);
            g.output(p, dx, lddx);
            ENOVA_TRY(g.product(p, kMmStore, kMmRows, kMmCols), "input gradient");
        }
        // The weights' gradients: [dg | du]'s columns are the rows of both projections'. They are small products over one
        // long reduction, and share a launch where one round holds both (500 rows, 420 x 1111: 95 -> 84 us a
        // training pass).
        MmParams up = g.params(g.F8 + g.F, g.D, g.T), down = g.params(g.D, g.F, g.T);
        g.segments(up, dgu, ox);
        g.output(up, dwg, g.D);
        up.c2 = dwu;
        up.wide = up.wide && aligned(dwu, 16);
        up.m1 = g.F;
        up.m2 = g.F8;
        g.segments(down, oy, h);
        g.output(down, dwd, g.F);
        if (dwg && dwd)
            ENOVA_TRY(g.pair(up, down), "weights' gradients");
        else if (dwg)
            ENOVA_TRY(g.product(up, kMmStore, kMmCols, kMmCols), "projections' gradients");
        else if (dwd)
            ENOVA_TRY(g.product(down, kMmStore, kMmCols, kMmCols), "output weights' gradient");
        return ENOVA_OK;
    }
};

enova_status gated_checked(enova_gated op, const void *x, int64_t ldx, int64_t rows, const void *wg, const void *wu,
                           const void *wd)
{
    if (!op)
        return fail(ENOVA_EINVAL, "NULL handle");
    if (rows < 0 || rows > kMostRows)
        return fail(ENOVA_EINVAL, "rows = %lld: need 0 .. 2^30", static_cast<long long>(rows));
    if (!wg || !wu || !wd || (rows && !x))
        return fail(ENOVA_EINVAL, "NULL matrix");
    if (ldx < op->c.model)
        return fail(ENOVA_EINVAL, "a row pitch of %lld is less than the %d columns", static_cast<long long>(ldx), op->c.model);
    return ENOVA_OK;
}

}  // namespace

extern "C" {

enova_status enova_gated_init(const enova_gated_config *config, enova_gated *out)
{
    if (!config || !out)
        return fail(ENOVA_EINVAL, "NULL argument");
    *out = nullptr;
    if (config->model < 1 || config->model > kWidest || config->hidden < 1 || config->hidden > kWidest)
        return fail(ENOVA_EINVAL, "need 1 <= model, hidden <= %d", kWidest);
    if (config->dtype != ENOVA_F32 && config->dtype != ENOVA_BF16)
        return fail(ENOVA_EINVAL, "unknown dtype %d", config->dtype);
    if (config->act < ENOVA_GATE_SILU || config->act > ENOVA_GATE_RELU)
        return fail(ENOVA_EINVAL, "unknown activation %d", config->act);
    int dev = 0;
    ENOVA_TRY(hipGetDevice(&dev), "hipGetDevice");
    enova_gated op = new (std::nothrow) enova_gated_s;
    if (!op)
        return fail(ENOVA_ENOMEM, "host memory");
    op->device = dev;
    op->c = *config;
    *out = op;
    return ENOVA_OK;
}

enova_status enova_gated_destroy(enova_gated op)
{
    if (op) {
        DeviceGuard guard(op->device);
        delete op;
    }
    return ENOVA_OK;
}

enova_status enova_gated_saved_floats(enova_gated op, int64_t rows, int64_t *floats)
{
    if (!op || !floats || rows < 0 || rows > kMostRows)
        return fail(ENOVA_EINVAL, "NULL argument, or rows out of range");
    *floats = Kept::bytes(rows, up(op->c.hidden, 8), op->c.dtype == ENOVA_F32) / 4;
    return ENOVA_OK;
}

enova_status enova_gated_forward(enova_gated op, const void *x, int64_t ldx, int64_t rows, const void *wg,
                                 const void *wu, const void *wd, void *y, int64_t ldy, float *saved, hipStream_t stream)
{
    enova_status s = gated_checked(op, x, ldx, rows, wg, wu, wd);
    if (s != ENOVA_OK)
        return s;
    if ((rows && !y) || ldy < op->c.model || !aligned(saved, 16))
        return fail(ENOVA_EINVAL, "y is NULL, its row pitch is less than its columns, or saved is not on a 16-byte boundary");
    if (rows == 0)
        return ENOVA_OK;
    DeviceGuard guard(op->device);
    if (!guard.ok)
        return fail(ENOVA_EHIP, "hipSetDevice(%d)", op->device);
    GatedCall g(op, rows, stream);
    const Kept kept(saved, rows, g.F8, g.f32);
    const int64_t h_plane = g.f32 ? rows * g.F8 : 0;
    if (rows <= few_rows(g.packs(x, ldx, g.D) || g.packs(wg, g.D, g.D) || g.packs(wd, g.F, g.F), static_cast<int64_t>(g.D) * g.F * 2)) {
        const int64_t size = g.f32 ? 4 : 2;
        // in fp32 the second product reads h as it is, not its saved parts
        if ((s = op->ws.need(rows * g.F8 * size, stream)) != ENOVA_OK)
            return s;
        MmParams p = g.params(g.T, g.F, g.D);
        p.segments = 1;
        p.x[0] = x;
        p.w[0] = wg;
        p.w2[0] = wu;
        p.ldx = ldx * size;
        p.ldw = g.D * size;
        p.c = g.f32 || saved ? kept.h : reinterpret_cast<__bf16 *>(op->ws.p);
        p.ldc = g.F8;
        p.plane = h_plane;
        p.h32 = g.f32 ? reinterpret_cast<float *>(op->ws.p) : nullptr;
        kept.tell(p, g.F8);
        ENOVA_TRY(launch_mm_few(p, kMmGate, op->c.dtype, stream), "gate product");
        MmParams q = g.params(g.T, g.D, g.F);
        q.segments = 1;
        q.x[0] = g.f32 ? p.h32 : p.c;
        q.w[0] = wd;
        q.ldx = g.F8 * size;
        q.ldw = g.F * size;
        g.output(q, y, ldy);
        ENOVA_TRY(launch_mm_few(q, kMmStore, op->c.dtype, stream), "output product");
        return ENOVA_OK;
    }
    for (int pass = 0; pass < 2; ++pass) {
        const Operand ox = g.operand(x, ldx, rows, g.D), og = g.operand(wg, g.D, g.F, g.D),
                      ou = g.operand(wu, g.D, g.F, g.D), od = g.operand(wd, g.F, g.D, g.F);
        ENOVA_TRY(g.pack(), "pack");
        const Operand h = saved ? Operand{kept.h, g.F8, h_plane} : g.own(rows, g.F8);
        g.most = g.carve.at;
        ENOVA_TRY(g.gate(ox, og, ou, h, kept), "gate product");
        MmParams p = g.params(g.T, g.D, g.F);
        g.segments(p, h, od);
        g.output(p, y, ldy);
        ENOVA_TRY(g.product(p, kMmStore, kMmRows, kMmRows), "output product");
        if (pass == 0) {
            if (saved && g.most > op->ws.cap) {        // it grows: for the backward call that follows as well
                GatedCall later(op, rows, stream);
                const GatedBackward b{x, ldx, wg, wu, wd, saved, x, ldx, y, ldy, y, y, y};
                if ((s = b.queue(later)) != ENOVA_OK)
                    return s;
                g.most = std::max(g.most, later.most);
            }
            if ((s = g.lay_out()) != ENOVA_OK)
                return s;
        }
    }
    return ENOVA_OK;
}

enova_status enova_gated_backward(enova_gated op, const void *x, int64_t ldx, int64_t rows, const void *wg,
                                  const void *wu, const void *wd, const float *saved, const void *dy, int64_t lddy,
                                  void *dx, int64_t lddx, void *dwg, void *dwu, void *dwd, hipStream_t stream)
{
    enova_status s = gated_checked(op, x, ldx, rows, wg, wu, wd);
    if (s != ENOVA_OK)
        return s;
    if ((rows && !dy) || lddy < op->c.model || (dx && lddx < op->c.model) || !dwg != !dwu || !aligned(saved, 16))
        return fail(ENOVA_EINVAL, "dy is NULL, a row pitch is less than its columns, only one of dwg and dwu is given, or saved is not on a 16-byte boundary");
    DeviceGuard guard(op->device);
    if (!guard.ok)
        return fail(ENOVA_EHIP, "hipSetDevice(%d)", op->device);
    if (rows == 0) {
        const int64_t bytes = static_cast<int64_t>(op->c.model) * op->c.hidden * (op->c.dtype == ENOVA_F32 ? 4 : 2);
        for (void *q : {dwg, dwu, dwd})
            if (q)
                ENOVA_TRY(launch_zero(q, bytes, stream), "zero gradients");
        return ENOVA_OK;
    }
    GatedCall g(op, rows, stream);
    const GatedBackward b{x, ldx, wg, wu, wd, saved, dy, lddy, dx, lddx, dwg, dwu, dwd};
    for (int pass = 0; pass < 2; ++pass) {
        if ((s = b.queue(g)) != ENOVA_OK)
            return s;
        if (pass == 0 && (s = g.lay_out()) != ENOVA_OK)
            return s;
    }
    return ENOVA_OK;
}

// ------------------------------------------------------------------------------ norms
enova_status enova_resnorm_init(const enova_resnorm_config *config, enova_resnorm *out)
{
    if (!config || !out)
        return fail(ENOVA_EINVAL, "NULL argument");
    *out = nullptr;
    if (config->model < 1 || config->model > kNormWidest)
        return fail(ENOVA_EINVAL, "need 1 <= model <= %d", kNormWidest);
    if (config->dtype != ENOVA_F32 && config->dtype != ENOVA_BF16)
        return fail(ENOVA_EINVAL, "unknown dtype %d", config->dtype);
    if (config->norm != ENOVA_RMS_NORM && config->norm != ENOVA_LAYER_NORM)
        return fail(ENOVA_EINVAL, "unknown norm %d", config->norm);
    if (!(config->eps > 0.0f) || !std::isfinite(config->eps) || !std::isfinite(config->keep) || !std::isfinite(config->scale))
        return fail(ENOVA_EINVAL, "need eps > 0 and finite keep and scale");
    if (config->group < 0)
        return fail(ENOVA_EINVAL, "group = %lld", static_cast<long long>(config->group));
    int dev = 0;
    ENOVA_TRY(hipGetDevice(&dev), "hipGetDevice");
    enova_resnorm op = new (std::nothrow) enova_resnorm_s;
    if (!op)
        return fail(ENOVA_ENOMEM, "host memory");
    op->device = dev;
    op->c = *config;
    *out = op;
    return ENOVA_OK;
}

enova_status enova_resnorm_destroy(enova_resnorm op)
{
    if (op) {
        DeviceGuard guard(op->device);
        delete op;
    }
    return ENOVA_OK;
}

static enova_status resnorm_checked(enova_resnorm op, const void *residual, const void *branch, int64_t rows, const float *post,
                                    const float *post_bias, const float *pre, const float *gate)
{
    if (!op)
        return fail(ENOVA_EINVAL, "NULL handle");
    if (rows < 0 || rows > kMostRows)
        return fail(ENOVA_EINVAL, "rows = %lld: need 0 .. 2^30", static_cast<long long>(rows));
    if (!pre || (rows && (!residual || !branch)))
        return fail(ENOVA_EINVAL, "NULL matrix or weight");
    if (post_bias && !post)
        return fail(ENOVA_EINVAL, "post_bias without post");
    if (gate && op->c.group < 1)
        return fail(ENOVA_EINVAL, "a gate needs a group of 1 row or more");
    return ENOVA_OK;
}

static NormParams norm_params(const enova_resnorm_config &c, const void *residual, const void *branch, int64_t rows,
                              const float *post, const float *post_bias, const float *pre, const float *gate)
{
    NormParams p{};
    p.residual = residual;
    p.branch = branch;
    p.rows = rows;
    p.model = c.model;
    p.layer = c.norm == ENOVA_LAYER_NORM;
    p.eps = c.eps;
    p.keep = c.keep;
    p.scale = c.scale;
    p.group = gate ? std::min<int64_t>(c.group, std::max<int64_t>(rows, 1)) : 1;
    p.post = post;
    p.post_bias = post_bias;
    p.pre = pre;
    p.gate = gate;
    return p;
}

enova_status enova_resnorm_forward(enova_resnorm op, const void *residual, const void *branch, int64_t rows,
                                   const float *post, const float *post_bias, const float *pre, const float *pre_bias,
                                   const float *gate, void *res, void *out, float *stats, hipStream_t stream)
{
    const enova_status s = resnorm_checked(op, residual, branch, rows, post, post_bias, pre, gate);
    if (s != ENOVA_OK)
        return s;
    if ((rows && (!res || !out)) || !aligned(stats, 16))
        return fail(ENOVA_EINVAL, "NULL output, or stats not on a 16-byte boundary");
    if (rows == 0)
        return ENOVA_OK;
    DeviceGuard guard(op->device);
    if (!guard.ok)
        return fail(ENOVA_EHIP, "hipSetDevice(%d)", op->device);
    NormParams p = norm_params(op->c, residual, branch, rows, post, post_bias, pre, gate);
    p.pre_bias = pre_bias;
    p.res = res;
    p.out = out;
    p.stats = stats;
    ENOVA_TRY(launch_resnorm_forward(p, op->c.dtype, stream), "resnorm");
    return ENOVA_OK;
}

enova_status enova_resnorm_backward(enova_resnorm op, const void *residual, const void *branch, int64_t rows,
                                    const float *post, const float *post_bias, const float *pre, const float *gate,
                                    const float *stats, const void *dres, const void *dout, void *dresidual, void *dbranch,
                                    float *dpost, float *dpost_bias, float *dpre, float *dpre_bias, float *dgate,
                                    hipStream_t stream)
{
    enova_status s = resnorm_checked(op, residual, branch, rows, post, post_bias, pre, gate);
    if (s != ENOVA_OK)
        return s;
    if ((rows && (!stats || !dres || !dout || !dresidual || !dbranch)) || !aligned(stats, 16))
        return fail(ENOVA_EINVAL, "NULL argument, or stats not on a 16-byte boundary");
    if ((dpost && !post) || (dgate && !gate))
        return fail(ENOVA_EINVAL, "the gradient of a weight or gate that is not given");
    DeviceGuard guard(op->device);
    if (!guard.ok)
        return fail(ENOVA_EHIP, "hipSetDevice(%d)", op->device);
    NormParams p = norm_params(op->c, residual, branch, rows, post, post_bias, pre, gate);
    p.stats = const_cast<float *>(stats);
    p.dres = dres;
    p.dout = dout;
    p.dresidual = dresidual;
    p.dbranch = dbranch;
    float *const sums[kNormSums] = {dpost, dpost_bias, dpre, dpre_bias};
    for (int i = 0; i < kNormSums; ++i)
        p.want |= sums[i] ? 1u << i : 0u;
    // What a compute unit holds, 8 waves (`target` teams; 16 in two rounds: 6 to 14% slower), each walking the same number of items: runs of rows, of one
    // gate where there are gates, whose groups are cut where that evens the teams' shares out (half a row an item:
    // its gate and the sums it leaves).
    const int team = norm_team(p.model), per_block = team <= 64 ? 256 / team : 1;
    const int64_t target = 131072 / std::min(team, 512);
    const int64_t groups = gate ? (rows + p.group - 1) / p.group : 0;
    if (groups) {
        const int64_t most = std::min<int64_t>(p.group, std::max<int64_t>(1, 4 * target / groups));
        double best = 0.0;
        for (int64_t cut = 1; cut <= most; cut += std::max<int64_t>(1, cut / 8)) {
            const int64_t item_rows = (p.group + cut - 1) / cut, parts = (p.group + item_rows - 1) / item_rows;
            const double cost = (item_rows + 0.5) * ((groups * parts + target - 1) / target);
            if (cut == 1 || cost < best) {
                best = cost;
                p.item_rows = static_cast<int>(item_rows);
                p.items_per_group = parts;
            }
        }
        p.items = groups * p.items_per_group;
    } else {
        p.item_rows = static_cast<int>(std::max<int64_t>(1, (rows + target - 1) / target));
        p.items_per_group = 1;
        p.items = (rows + p.item_rows - 1) / p.item_rows;
    }
    p.items_per_team = std::max<int64_t>(1, (p.items + target - 1) / target);
    const int64_t teams = (p.items + p.items_per_team - 1) / p.items_per_team, blocks = (teams + per_block - 1) / per_block;
    Carve carve;
    float *gate_part = nullptr;
    for (int pass = 0; pass < 2; ++pass) {
        p.part = carve.take<float>(blocks * kNormSums * p.model);
        if (dgate && p.items_per_group > 1)
            gate_part = carve.take<float>(p.items * p.model);
        if (pass == 0) {
            if ((s = op->ws.need(std::max<size_t>(carve.at, 256), stream)) != ENOVA_OK)
                return s;
            carve = {op->ws.p, 0};
        }
    }
    p.gate_part = gate_part ? gate_part : dgate;
    if (rows)
        ENOVA_TRY(launch_resnorm_backward(p, op->c.dtype, blocks, stream), "resnorm gradients");
    NormSumJobs jobs;
    for (int i = 0; i < kNormSums; ++i)
        if (sums[i]) {
            jobs.src[jobs.n] = p.part + i * p.model;
            jobs.out[jobs.n++] = sums[i];
        }
    if (jobs.n)
        ENOVA_TRY(launch_norm_sums(jobs, kNormSums * static_cast<int64_t>(p.model), blocks, blocks, jobs.n, p.model, stream), "sums over rows");
    if (gate_part) {
        NormSumJobs gates;
        gates.n = 1;
        gates.src[0] = gate_part;
        gates.out[0] = dgate;
        ENOVA_TRY(launch_norm_sums(gates, p.model, p.items_per_group, p.items, groups, p.model, stream), "gate sums");
    }
    return ENOVA_OK;
}

// ------------------------------------------------------------------------------ AdamW
static void free_adamw(enova_adamw op)
{
    if (!op)
        return;
    (void)hipFree(op->table);
    delete op;
}

static bool adam_wide(const AdamTensor &t, int param_dtype, int grad_dtype, int bits)
{
    return aligned(t.param, param_dtype == ENOVA_F32 ? 16 : 8) && aligned(t.grad, grad_dtype == ENOVA_F32 ? 16 : 8) &&
           aligned(t.copy, 8) && aligned(t.m, bits == 8 ? 4 : 16) && aligned(t.v, bits == 8 ? 4 : 16);
}

enova_status enova_adamw_init(const enova_adamw_config *config, const enova_adamw_tensor *tensors, int32_t n_tensors,
                              enova_adamw *out)
{
    if (!config || !out || (n_tensors > 0 && !tensors))
        return fail(ENOVA_EINVAL, "NULL argument");
    *out = nullptr;
    const enova_adamw_config &c = *config;
    if (n_tensors < 0)
        return fail(ENOVA_EINVAL, "n_tensors = %d", n_tensors);
    if (c.bits != 32 && c.bits != 8)
        return fail(ENOVA_EINVAL, "states of %d bits: need 32 or 8", c.bits);
    for (int32_t d : {c.param_dtype, c.grad_dtype})
        if (d != ENOVA_F32 && d != ENOVA_BF16)
            return fail(ENOVA_EINVAL, "unknown dtype %d", d);
    if (!(c.b1 >= 0.0 && c.b1 < 1.0) || !(c.b2 >= 0.0 && c.b2 < 1.0) || !(c.eps > 0.0) || !(c.decay >= 0.0) ||
        !std::isfinite(c.eps) || !std::isfinite(c.decay))
        return fail(ENOVA_EINVAL, "need 0 <= b1, b2 < 1, eps > 0, decay >= 0");
    int64_t chunks = 0;
    for (int i = 0; i < n_tensors; ++i) {
        const enova_adamw_tensor &t = tensors[i];
        if (t.numel < 0)
            return fail(ENOVA_EINVAL, "tensor %d: numel = %lld", i, static_cast<long long>(t.numel));
        if (t.numel && (!t.param || !t.grad || !t.m || !t.v || (c.bits == 8 && (!t.m_scale || !t.v_scale))))
            return fail(ENOVA_EINVAL, "tensor %d: NULL buffer", i);
        if (t.copy && c.param_dtype != ENOVA_F32)
            return fail(ENOVA_EINVAL, "tensor %d: only fp32 parameters have bf16 copies", i);
        chunks += (t.numel + kAdamChunk - 1) / kAdamChunk;
    }
    if (chunks * kAdamThreads >= int64_t{1} << 32)         // one launch
        return fail(ENOVA_EINVAL, "too many elements for one step");
    int dev = 0;
    ENOVA_TRY(hipGetDevice(&dev), "hipGetDevice");
    enova_adamw op = new (std::nothrow) enova_adamw_s;
    if (!op)
        return fail(ENOVA_ENOMEM, "host memory");
    op->device = dev;
    op->c = c;
    op->chunks = static_cast<int>(chunks);
    std::vector<AdamChunk> list;
    try {
        op->host.resize(n_tensors);
        list.reserve(chunks);
        for (int i = 0; i < n_tensors; ++i) {
            const enova_adamw_tensor &t = tensors[i];
            op->host[i] = {t.param, t.grad, t.copy, t.m, t.v, t.m_scale, t.v_scale, t.numel, 0};
            op->host[i].wide = adam_wide(op->host[i], c.param_dtype, c.grad_dtype, c.bits);
            for (int64_t k = 0; k * kAdamChunk < t.numel; ++k)
                list.push_back({i, static_cast<int32_t>(k)});
        }
    } catch (const std::bad_alloc &) {
        free_adamw(op);
        return fail(ENOVA_ENOMEM, "host memory");
    }
    Carve carve;
    for (int pass = 0; pass < 2; ++pass) {
        op->d_tensors = carve.take<AdamTensor>(std::max(n_tensors, 1));
        op->d_chunks = carve.take<AdamChunk>(std::max<int64_t>(chunks, 1));
        const size_t copied = carve.at;
        op->d_values = carve.take<AdamValues>(std::max(n_tensors, 1));
        if (pass == 0) {
            hipError_t e = hipMalloc(reinterpret_cast<void **>(&op->table), carve.at);
            if (e != hipSuccess) {
                op->table = nullptr;
                (void)hipGetLastError();
                free_adamw(op);
                return fail(ENOVA_ENOMEM, "hipMalloc(%zu): %s", carve.at, hipGetErrorString(e));
            }
            // both lists in one copy
            const size_t from = (sizeof(AdamTensor) * std::max(n_tensors, 1) + 255) / 256 * 256;
            try {
                std::vector<char> both(copied);
                if (n_tensors)
                    std::memcpy(both.data(), op->host.data(), sizeof(AdamTensor) * n_tensors);
                if (chunks)
                    std::memcpy(both.data() + from, list.data(), sizeof(AdamChunk) * chunks);
                e = hipMemcpy(op->table, both.data(), copied, hipMemcpyHostToDevice);
            } catch (const std::bad_alloc &) {
                free_adamw(op);
                return fail(ENOVA_ENOMEM, "host memory");
            }
            if (e != hipSuccess) {
                free_adamw(op);
                return hip_fail(e, "hipMemcpy tensor list");
            }
            carve = {op->table, 0};
        }
    }
    *out = op;
    return ENOVA_OK;
}

enova_status enova_adamw_destroy(enova_adamw op)
{
    if (op) {
        DeviceGuard guard(op->device);
        free_adamw(op);
    }
    return ENOVA_OK;
}

static enova_status not_captured(hipStream_t stream)
{
    hipStreamCaptureStatus capturing = hipStreamCaptureStatusNone;
    (void)hipStreamIsCapturing(stream, &capturing);
    return capturing == hipStreamCaptureStatusNone ? ENOVA_OK : fail(ENOVA_EINVAL, "not on a stream under capture");
}

enova_status enova_adamw_set_grads(enova_adamw op, const void *const *grads, hipStream_t stream)
{
    if (!op || !grads)
        return fail(ENOVA_EINVAL, "NULL argument");
    const enova_status s = not_captured(stream);
    if (s != ENOVA_OK)
        return s;
    const int n = static_cast<int>(op->host.size());
    for (int i = 0; i < n; ++i)
        if (op->host[i].numel && !grads[i])
            return fail(ENOVA_EINVAL, "tensor %d: NULL gradient", i);
    DeviceGuard guard(op->device);
    if (!guard.ok)
        return fail(ENOVA_EHIP, "hipSetDevice(%d)", op->device);
    for (int from = 0; from < n; from += kAdamPointers) {
        AdamPointers p{};
        p.from = from;
        p.n = std::min(n - from, kAdamPointers);
        for (int i = 0; i < p.n; ++i) {
            AdamTensor &t = op->host[from + i];
            t.grad = grads[from + i];
            t.wide = adam_wide(t, op->c.param_dtype, op->c.grad_dtype, op->c.bits);
            p.a[i] = t.grad;
            p.wide |= static_cast<uint64_t>(t.wide) << i;
        }
        ENOVA_TRY(launch_adamw_grads(op->d_tensors, p, stream), "gradients' list");
    }
    return ENOVA_OK;
}

enova_status enova_adamw_step(enova_adamw op, int64_t n, double lr, float grad_scale, hipStream_t stream)
{
    if (!op)
        return fail(ENOVA_EINVAL, "NULL handle");
    if (n < 1 || !std::isfinite(lr) || !std::isfinite(grad_scale))
        return fail(ENOVA_EINVAL, "need a step number of 1 or more, and finite lr and grad_scale");
    if (op->chunks == 0)
        return ENOVA_OK;
    DeviceGuard guard(op->device);
    if (!guard.ok)
        return fail(ENOVA_EHIP, "hipSetDevice(%d)", op->device);
    const enova_adamw_config &c = op->c;
    AdamArgs a{};
    a.b1 = static_cast<float>(c.b1);
    a.b1c = static_cast<float>(1.0 - c.b1);
    a.b2 = static_cast<float>(c.b2);
    a.b2c = static_cast<float>(1.0 - c.b2);
    a.keep = static_cast<float>(1.0 - lr * c.decay);
    a.lr = static_cast<float>(lr * (1.0 / (1.0 - std::pow(c.b1, static_cast<double>(n)))));
    a.root = static_cast<float>(1.0 / std::sqrt(1.0 - std::pow(c.b2, static_cast<double>(n))));
    // the kernel's reciprocal takes no subnormal numbers; beside a root of v in fp32 (3.7e-23 at least) neither does eps show
    a.eps = std::max(static_cast<float>(c.eps), std::numeric_limits<float>::min());
    a.grad_scale = grad_scale;
    a.step = static_cast<uint32_t>(n);
    ENOVA_TRY(launch_adamw(c.bits, c.param_dtype, c.grad_dtype, op->d_tensors, op->d_chunks, op->chunks, a, stream), "AdamW step");
    return ENOVA_OK;
}

enova_status enova_adamw_states(enova_adamw op, float *const *m, float *const *v, hipStream_t stream)
{
    if (!op || !m || !v)
        return fail(ENOVA_EINVAL, "NULL argument");
    if (op->c.bits != 8)
        return fail(ENOVA_EINVAL, "the states are held in 32 bits");
    const enova_status s = not_captured(stream);
    if (s != ENOVA_OK)
        return s;
    const int n = static_cast<int>(op->host.size());
    for (int i = 0; i < n; ++i)
        if (op->host[i].numel && (!m[i] || !v[i]))
            return fail(ENOVA_EINVAL, "tensor %d: NULL destination", i);
    if (op->chunks == 0)
        return ENOVA_OK;
    DeviceGuard guard(op->device);
    if (!guard.ok)
        return fail(ENOVA_EHIP, "hipSetDevice(%d)", op->device);
    for (int from = 0; from < n; from += kAdamPointers) {
        AdamPointers p{};
        p.from = from;
        p.n = std::min(n - from, kAdamPointers);
        for (int i = 0; i < p.n; ++i) {
            p.a[i] = m[from + i];
            p.b[i] = v[from + i];
            p.wide |= static_cast<uint64_t>(aligned(p.a[i], 16) && aligned(p.b[i], 16)) << i;
        }
        ENOVA_TRY(launch_adamw_values(op->d_values, p, stream), "destinations' list");
    }
    ENOVA_TRY(launch_adamw_states(op->d_tensors, op->d_chunks, op->chunks, op->d_values, stream), "AdamW states");
    return ENOVA_OK;
}

// ------------------------------------------------------------------------------ 8-bit product
enova_status enova_i8_init(const enova_i8_config *config, const int8_t *w, int64_t ldw, const float *w_scale,
                           const float *bias, enova_i8 *out)
{
    if (!config || !out || !w || !w_scale)
        return fail(ENOVA_EINVAL, "NULL argument");
    *out = nullptr;
    if (config->inputs < 1 || config->inputs > kWidest / 2 || config->outputs < 1 || config->outputs > kWidest)
        return fail(ENOVA_EINVAL, "need 1 <= inputs <= %d, 1 <= outputs <= %d", kWidest / 2, kWidest);
    if (config->dtype != ENOVA_F32 && config->dtype != ENOVA_BF16)
        return fail(ENOVA_EINVAL, "unknown dtype %d", config->dtype);
    if (config->gate < -1 || config->gate > ENOVA_GATE_RELU)
        return fail(ENOVA_EINVAL, "unknown activation %d", config->gate);
    if (ldw < config->inputs || ldw % 16 || ldw > 4 * kWidest || !aligned(w, 16))
        return fail(ENOVA_EINVAL, "w's row pitch %lld: need a multiple of 16 of at least %d and at most %d, on a 16-byte boundary",
                    static_cast<long long>(ldw), config->inputs, 4 * kWidest);
    int dev = 0;
    ENOVA_TRY(hipGetDevice(&dev), "hipGetDevice");
    enova_i8 op = new (std::nothrow) enova_i8_s;
    if (!op)
        return fail(ENOVA_ENOMEM, "host memory");
    op->device = dev;
    op->c = *config;
    op->w = w;
    op->ldw = ldw;
    op->w_scale = w_scale;
    op->bias = bias;
    *out = op;
    return ENOVA_OK;
}

enova_status enova_i8_destroy(enova_i8 op)
{
    if (op) {
        DeviceGuard guard(op->device);
        delete op;
    }
    return ENOVA_OK;
}

enova_status enova_i8_forward(enova_i8 op, const void *x, int64_t ldx, int64_t rows, void *y, int64_t ldy, hipStream_t stream)
{
    if (!op)
        return fail(ENOVA_EINVAL, "NULL handle");
    const enova_i8_config &c = op->c;
    if (rows < 0 || rows > kMostRows || (rows && (!x || !y)))
        return fail(ENOVA_EINVAL, "rows out of 0 .. 2^30, or a NULL matrix");
    if (ldx < (c.gate < 0 ? 1 : 2) * static_cast<int64_t>(c.inputs) || ldy < c.outputs)
        return fail(ENOVA_EINVAL, "a row pitch is less than the columns");
    if (rows == 0)
        return ENOVA_OK;
    DeviceGuard guard(op->device);
    if (!guard.ok)
        return fail(ENOVA_EHIP, "hipSetDevice(%d)", op->device);
    const int pitch = static_cast<int>(up(c.inputs, 16));
    const bool few = rows <= few_rows(false, static_cast<int64_t>(pitch) * c.outputs);
    const MmPlan plan = few ? MmPlan{0, 1, 0} : mm_plan(rows, c.outputs, (pitch + 127) / 128, false, c.dtype == ENOVA_F32 ? 4.0 : 2.0, 0.0);
    const bool fused = i8_fused(rows, pitch);
    Carve carve;
    int8_t *q = nullptr;
    float *scale = nullptr;
    int *part = nullptr;
    for (int pass = 0; pass < 2 && !fused; ++pass) {
        q = carve.take<int8_t>(rows * pitch);
        scale = carve.take<float>(rows);
        part = plan.part ? carve.take<int>(plan.part) : nullptr;
        if (pass == 0) {
            const enova_status s = op->ws.need(carve.at, stream);
            if (s != ENOVA_OK)
                return s;
            carve = {op->ws.p, 0};
        }
    }
    MmParams p{};
    p.x[0] = q;
    p.w[0] = op->w;
    p.segments = 1;
    p.ldx = pitch;
    p.ldw = op->ldw;
    p.m = static_cast<int>(rows);
    p.n = c.outputs;
    p.n8 = static_cast<int>(up(p.n, 8));
    p.k = pitch;
    p.slices = plan.slices;
    p.part = part;
    p.c = y;
    p.ldc = ldy;
    p.f32 = c.dtype == ENOVA_F32;
    p.wide = ldy % 8 == 0 && aligned(y, 16);
    p.sx = scale;
    p.sw = op->w_scale;
    p.bias = op->bias;
    if (fused) {
        ENOVA_TRY(launch_i8_fused(p, QuantParams{x, ldx, c.inputs, c.gate, c.dtype}, stream), "8-bit product");
        return ENOVA_OK;
    }
    ENOVA_TRY(launch_quantize(x, c.dtype, ldx, rows, c.inputs, c.gate, q, pitch, scale, stream), "quantize");
    if (few)
        ENOVA_TRY(launch_mm_few(p, kMmInt8, ENOVA_BF16, stream), "8-bit product");
    else
        ENOVA_TRY(launch_mm_int8(p, plan.tile, stream), "8-bit product");
    if (p.slices > 1)
        ENOVA_TRY(launch_mm_finish(p, kMmInt8, stream), "8-bit product");
    return ENOVA_OK;
}

}  // extern "C"
