/*
 * enova_block.h -- C ABI of the operators of a residual gated block (MI355X, gfx950).
 *
 * A deeper window encoder than the detector's one hidden layer (enova_detect.h) is a stack of blocks
 * over flattened windows, one row a window:
 *
 *     res = keep * residual + scale * gate * N(branch; post)      norms, gate and residual scale:
 *     out = N(res; pre)                                           enova_resnorm_*
 *     branch' = (act(out Wg^T) * (out Wu^T)) Wd^T                 gated feed-forward block: enova_gated_*
 *
 * with the gradients of both, an AdamW step over all of a stack's tensors (enova_adamw_*), and the
 * product in 8-bit integers that serves a trained projection (enova_i8_*).
 *
 * Conventions are those of enova_detect.h: every function returns an enova_status and none aborts or
 * throws; arguments are checked on the host before any launch, and a failing call writes no output;
 * pointers are device memory unless they are said to be the host's; calls are asynchronous on `stream`,
 * those on one handle must not overlap, and a handle's workspace grows on demand (a growing call waits
 * for the device, and is refused while `stream` is being captured into a graph). A graph that captured
 * calls holds the workspace that they were given: a handle keeps it when a later call needs a larger one,
 * has to outlive the graph, and a replay counts as a call on it. Matrices are row-major
 * with the row pitch ("ld", in elements) given where one is; `rows` may be 0. Types: ENOVA_F32 or
 * ENOVA_BF16 for a handle's matrices; sums and norms are formed in 32 bits. Buffers of one call must not
 * overlap unless it is said that they may.
 */
#ifndef ENOVA_BLOCK_H
#define ENOVA_BLOCK_H

#include "enova_detect.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct enova_gated_s *enova_gated;       /* opaque; owned by the library */
typedef struct enova_resnorm_s *enova_resnorm;
typedef struct enova_adamw_s *enova_adamw;
typedef struct enova_i8_s *enova_i8;

/* ---------------------------------------------------------------- gated feed-forward block
 * y = h Wd^T, h = act(g) * u, g = x Wg^T, u = x Wu^T for x [rows][model], Wg and Wu [hidden][model],
 * Wd [model][hidden] (contiguous, as torch.nn.Linear stores them).
 * act: SiLU g / (1 + e^-g), GELU g Phi(g) (with erf), or ReLU (derivative 0 at 0).
 * bf16: products of bf16 with fp32 accumulation; h and the gradients of g and u are rounded to bf16
 * once, as operands of the next product, and g and u between the forward and the backward call to 11 bits
 * (and to 2^-39 of the largest of eight neighbours: a smaller one is 0 but for the sign ReLU needs).
 * f32: operands in three bf16 parts (24 bits, fewer below 2^-110), six products, activations within a few
 * ulp; values that are not finite, or past bf16's largest (3.39e38), make NaN of what they reach. */
typedef enum { ENOVA_GATE_SILU = 0, ENOVA_GATE_GELU = 1, ENOVA_GATE_RELU = 2 } enova_gate_act;

typedef struct {
    int32_t model, hidden;   /* 1 .. 262144 each */
    int32_t dtype;           /* enova_dtype of every matrix */
    int32_t act;             /* enova_gate_act */
} enova_gated_config;

/* Create the block's handle on the current device. Errors: EINVAL, ENOMEM, EHIP. */
enova_status enova_gated_init(const enova_gated_config *config, enova_gated *out);
enova_status enova_gated_destroy(enova_gated op);

/* Floats of the buffer that a forward call leaves g, u and h in for the backward call. Errors: EINVAL. */
enova_status enova_gated_saved_floats(enova_gated op, int64_t rows, int64_t *floats_host);

/* y [rows][model]. saved: NULL (serving), or enova_gated_saved_floats floats. Errors: EINVAL, ENOMEM, EHIP. */
enova_status enova_gated_forward(enova_gated op, const void *x, int64_t ldx, int64_t rows, const void *wg,
                                 const void *wu, const void *wd, void *y, int64_t ldy, float *saved,
                                 hipStream_t stream);

/* The gradients for dy [rows][model]: dx [rows][model] (or NULL), dwg, dwu [hidden][model] (both or
 * neither NULL) and dwd [model][hidden] (or NULL), overwritten. saved: the forward call's, or NULL: g and
 * u are computed again. The order of every sum is fixed, so equal inputs give equal bits.
 * Errors: EINVAL, ENOMEM, EHIP. */
enova_status enova_gated_backward(enova_gated op, const void *x, int64_t ldx, int64_t rows, const void *wg,
                                  const void *wu, const void *wd, const float *saved, const void *dy,
                                  int64_t lddy, void *dx, int64_t lddx, void *dwg, void *dwu, void *dwd,
                                  hipStream_t stream);

/* ---------------------------------------------------------------- norms, gate and residual scale
 * res = keep * residual + scale * gate * b, b = N(branch; post, post_bias) (or b = branch where post is
 * NULL); out = N(res; pre, pre_bias), formed from res before it is rounded to the handle's type.
 * N(v; w, c) = v / sqrt(mean(v^2) + eps) * w + c (RMS) or (v - mean v) / sqrt(var v + eps) * w + c
 * (LAYER, population variance); biases may be NULL. gate: NULL (1), or [ceil(rows/group)][model], row r
 * taking gate row r / group (group >= 1; one gate for all rows is group >= rows). Matrices [rows][model]
 * are contiguous; norm weights, biases and gates are fp32. */
typedef enum { ENOVA_RMS_NORM = 0, ENOVA_LAYER_NORM = 1 } enova_norm_kind;

typedef struct {
    int32_t model;           /* 1 .. 16384 */
    int32_t dtype;           /* enova_dtype of the matrices */
    int32_t norm;            /* enova_norm_kind */
    float eps, keep, scale;  /* eps > 0 */
    int64_t group;           /* rows that share a gate row; read where a gate is given */
} enova_resnorm_config;

enova_status enova_resnorm_init(const enova_resnorm_config *config, enova_resnorm *out);
enova_status enova_resnorm_destroy(enova_resnorm op);

/* stats: NULL, or [rows][4] floats for the backward call. res may be residual. Errors: EINVAL, EHIP. */
enova_status enova_resnorm_forward(enova_resnorm op, const void *residual, const void *branch, int64_t rows,
                                   const float *post, const float *post_bias, const float *pre,
                                   const float *pre_bias, const float *gate, void *res, void *out, float *stats,
                                   hipStream_t stream);

/* Gradients for dres and dout (of res and out): dresidual and dbranch [rows][model], dpost, dpost_bias,
 * dpre, dpre_bias [model] and dgate (the gate's shape) in fp32, overwritten; each may be NULL but
 * dresidual and dbranch. The order of every sum is fixed. Errors: EINVAL, ENOMEM, EHIP. */
enova_status enova_resnorm_backward(enova_resnorm op, const void *residual, const void *branch, int64_t rows,
                                    const float *post, const float *post_bias, const float *pre,
                                    const float *gate, const float *stats, const void *dres,
                                    const void *dout, void *dresidual, void *dbranch, float *dpost,
                                    float *dpost_bias, float *dpre, float *dpre_bias, float *dgate,
                                    hipStream_t stream);

/* ---------------------------------------------------------------- AdamW over many tensors
 *   m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2,
 *   p = p (1 - lr decay) - (m lr / (1 - b1^n)) / (sqrt(v) / sqrt(1 - b2^n) + eps)
 * at step n = 1, 2, ..., for every tensor of the handle in one launch. Parameters and gradients are fp32
 * or bf16; an fp32 parameter may have a bf16 copy, which receives its rounded value.
 * bits = 32: m and v are fp32. bits = 8: each 256 consecutive elements of a tensor share two fp32 scales,
 *   m = m_scale sign(c) (c / 127)^2, c int8;   sqrt(v) = v_scale (c / 255)^2, c uint8,
 * the scales being the largest |m| and sqrt(v) of the 256. Codes are rounded down after a dither in
 * [0, 1) is added that takes every value evenly over the steps (an average that moves by less than a
 * code's distance each step still moves), and a positive v has a code of 1 at least. Where an m or v of the 256
 * is not finite, all of them stand for NaN from then on. eps is taken as at least the smallest normal fp32. */
typedef struct {
    void *param;             /* [numel] */
    const void *grad;        /* [numel] */
    void *copy;              /* bf16 [numel] or NULL */
    void *m, *v;             /* fp32, or int8 and uint8 */
    float *m_scale, *v_scale;/* [ceil(numel/256)] each; bits = 8 only */
    int64_t numel;           /* >= 0 */
} enova_adamw_tensor;

typedef struct {
    int32_t bits;            /* 32 or 8 */
    int32_t param_dtype, grad_dtype;   /* enova_dtype */
    double b1, b2, eps, decay;         /* 0 <= b < 1, eps > 0, decay >= 0 */
} enova_adamw_config;

/* The handle keeps the list (host array of n_tensors; the device buffers stay the caller's, and have to
 * outlive the handle). States start as the caller left them (zero for a first step). Errors: EINVAL, ENOMEM, EHIP. */
enova_status enova_adamw_init(const enova_adamw_config *config, const enova_adamw_tensor *tensors,
                              int32_t n_tensors, enova_adamw *out);
enova_status enova_adamw_destroy(enova_adamw op);

/* New gradient buffers (host array of n_tensors device pointers) for later steps, in the stream's order; not while
 * `stream` is being captured. Errors: EINVAL, EHIP. */
enova_status enova_adamw_set_grads(enova_adamw op, const void *const *grads, hipStream_t stream);

/* Step number n >= 1 with gradients multiplied by grad_scale. n and lr are arguments of the launch: a captured step
 * replays with those. Errors: EINVAL, EHIP. */
enova_status enova_adamw_step(enova_adamw op, int64_t n, double lr, float grad_scale, hipStream_t stream);

/* The values that 8-bit states stand for, in fp32 (host arrays of n_tensors device pointers, each [numel]).
 * Not while `stream` is being captured. Errors: EINVAL (32-bit states among them), EHIP. */
enova_status enova_adamw_states(enova_adamw op, float *const *m, float *const *v, hipStream_t stream);

/* ---------------------------------------------------------------- product in 8-bit integers
 * y[r][o] = sx[r] w_scale[o] sum_k q[r][k] w[o][k] + bias[o] with q = rint(127 x / max |x|) and
 * sx = max |x| / 127 of each row (a row of zeros gives the bias; a row that is not finite throughout gives
 * NaN), sums in 32-bit integers. w [outputs][ldw] int8, ldw a multiple of 16 and at least inputs; w_scale,
 * bias (or NULL) fp32 [outputs]: the caller's, and have to outlive the handle.
 * gate >= 0 (an enova_gate_act): x has 2 * inputs columns [g | u], and act(g) * u (in fp32) is what is
 * multiplied. */
typedef struct {
    int32_t inputs, outputs; /* 1 .. 262144 each, inputs at most 131072 */
    int32_t dtype;           /* enova_dtype of x and y */
    int32_t gate;            /* -1, or an enova_gate_act */
} enova_i8_config;

enova_status enova_i8_init(const enova_i8_config *config, const int8_t *w, int64_t ldw, const float *w_scale,
                           const float *bias, enova_i8 *out);
enova_status enova_i8_destroy(enova_i8 op);

/* y [rows][outputs] from x [rows][inputs]. Errors: EINVAL, ENOMEM, EHIP. */
enova_status enova_i8_forward(enova_i8 op, const void *x, int64_t ldx, int64_t rows, void *y, int64_t ldy,
                              hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* ENOVA_BLOCK_H */
