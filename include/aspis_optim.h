/*
 * aspis_optim.h -- the end of a training step over a model's many tensors:
 * the global norm of the gradients, their clipping by it, and the AdamW
 * update.  The gradients are those that a round aggregated (views of
 * aspis_aggregate's out, cut at any coordinate) or those of a backward pass.
 *
 *   norm     ||g|| = s * sqrt( sum over tensors t, elements i of g_t[i]^2 )   aspis_grad_norm
 *   clip     g_t[i] <- c * s * g_t[i],  c = min(1, max_norm / (||g|| + 1e-6)) aspis_clip_grads
 *   update   AdamW on c * s * g without writing the clipped gradient          aspis_adamw
 *
 * s is a scale that the gradients have yet to be multiplied by (1 / loss scale,
 * 1 / micro-batches; 1 for none).
 *
 * Conventions, beside those of aspis.h:
 *   - A list is a host object made once for a set of tensors; it holds their
 *     addresses, lengths and types, and no device memory.  The tensors stay the
 *     caller's and have to stay where they are while the list is in use.  Calls
 *     on one list may come from several threads.
 *   - A tensor is `numel` elements without gaps, of fp32, bf16 or fp16, at any
 *     address that is a multiple of the element's size.  numel 0 is allowed (data
 *     may then be NULL).  One list may mix types, lengths and alignments.
 *   - Sums, norms and moments are held in 32 bits or more.  Up to 64 squares are
 *     added in fp32, and such sums as pairs of fp32 numbers (48 bits), or in fp64
 *     where they leave [1e-30, 1e24]: a norm neither overflows nor vanishes while
 *     it is within fp32's range itself.  The order depends on the call, the list
 *     (lengths, types, addresses modulo 32) and the device, so the same call gives
 *     the same bits each time.  Other calls on the same values (with and without
 *     tensor_norms, norm and clipping, copies elsewhere) may differ in the last bits.
 *   - NaN and infinity follow IEEE-754 through the formulas: an infinite norm
 *     makes c = 0 (finite gradients become 0, infinite ones NaN), a NaN makes
 *     everything NaN.  aspis_adamw can leave everything as it was instead.  An
 *     infinite max_norm clips nothing: c = 1, whatever the norm.
 *   - work is ASPIS_NORM_WORKSPACE_BYTES of device memory, 16-byte aligned,
 *     zeroed once by the caller; every call leaves it ready for the next.  Calls
 *     that may overlap on the GPU need a workspace (and a norm) each.
 *   - Clipping takes small lists in one cooperative kernel, whose blocks wait for one another.  The
 *     wait is bounded: were it ever to run out (after seconds), the norm and the gradients are
 *     undefined, and the workspace has to be zeroed again.
 *   - No call allocates, copies from the host or waits; all can be captured in a
 *     graph (with the arguments of the captured call, aspis_adamw's step too).
 */
#ifndef ASPIS_OPTIM_H
#define ASPIS_OPTIM_H

#include "aspis.h"

#ifdef __cplusplus
extern "C" {
#endif

#define ASPIS_NORM_WORKSPACE_BYTES 40960
#define ASPIS_CLIP_EPS 1e-6f          /* added to the norm in the clipping quotient */

typedef enum { ASPIS_F32 = 0, ASPIS_BF16 = 1, ASPIS_F16 = 2 } aspis_dtype;

/* One tensor of gradients, and where its clipped values go. */
typedef struct {
    void *data;                  /* device [numel] */
    void *out;                   /* device [numel], or NULL: clipped in place */
    int64_t numel;
    int32_t type;                /* aspis_dtype of data */
    int32_t out_type;            /* aspis_dtype of out; ignored where out is NULL */
} aspis_tensor;

typedef struct aspis_tensors aspis_tensors;

/* Checks n tensors and makes a list of them in *out.  Host only.
 * ASPIS_E_INVAL: a NULL pointer, a negative length or count, an unknown type;
 * ASPIS_E_ALIGN: an address that is no multiple of its element's size;
 * ASPIS_E_RANGE: more than 2^38 elements in a tensor, more than 2^24 tensors, or no
 * memory for the list.
 * Tensors may overlap for the norm; aspis_clip_grads refuses a list in which a
 * range that it writes overlaps another range (out may be data itself). */
aspis_status aspis_tensors_create(const aspis_tensor *tensors, int64_t n, aspis_tensors **out);
void aspis_tensors_destroy(aspis_tensors *list);

/* The global norm, and optionally that of every tensor.
 *   scale         s, finite and > 0
 *   norm          device fp32, out
 *   tensor_norms  device [n] fp32, out (0 for empty tensors), or NULL
 *   work          workspace
 * An empty list has norm 0.  Reads every element once. */
aspis_status aspis_grad_norm(const aspis_tensors *grads, float scale, float *norm,
                             float *tensor_norms, void *work, void *stream);

/* Clips the gradients: out_t[i] (or data_t[i]) = RN(g_t[i] * (s * c)), rounded once
 * to the output's type.
 *   max_norm  >= 0, may be infinite (NaN or negative: ASPIS_E_INVAL)
 *   norm      device fp32: written where work is given; with work NULL it is
 *             read, and is the norm to clip by (of the scaled gradients: that of
 *             a larger model, or of the other lists of this one)
 *   work      workspace, or NULL
 * In place nothing is written where s * c is 1: below the bound the call only
 * reads. */
aspis_status aspis_clip_grads(const aspis_tensors *grads, float max_norm, float scale,
                              float *norm, void *work, void *stream);

/* One tensor of parameters with its gradient and its moments. */
typedef struct {
    void *param;                 /* device [numel], in/out */
    float *master;               /* device [numel] fp32, in/out: the weights that the step is
                                    made on, param being their rounding; NULL: param itself */
    const void *grad;            /* device [numel] */
    float *exp_avg;              /* device [numel] fp32, in/out: first moment m */
    float *exp_avg_sq;           /* device [numel] fp32, in/out: second moment v */
    int64_t numel;
    int32_t param_type;          /* aspis_dtype; fp32 parameters take no master */
    int32_t grad_type;           /* aspis_dtype */
    float weight_decay;          /* of this tensor, >= 0 and finite */
    int32_t reserved;            /* 0 */
} aspis_param;

typedef struct aspis_params aspis_params;

/* Checks n parameters and makes a list of them in *out.  Host only.  Errors as for
 * aspis_tensors_create; ASPIS_E_INVAL too where any two of the arrays overlap,
 * except gradients among themselves. */
aspis_status aspis_params_create(const aspis_param *params, int64_t n, aspis_params **out);
void aspis_params_destroy(aspis_params *list);

typedef struct {
    double lr;                   /* finite in fp32 */
    double beta1, beta2;         /* in [0, 1) */
    double eps;                  /* >= 0, finite in fp32, which it is used in */
    int64_t step;                /* this step's number, from 1: bias corrections 1 - beta^step */
    float max_norm;              /* >= 0: clip to it (INFINITY: only the norm is taken);
                                    negative: no norm, no clipping */
    float scale;                 /* s, finite and > 0 */
    int32_t skip_nonfinite;      /* 1: change nothing where the norm is not finite */
    int32_t reserved;            /* 0 */
} aspis_adamw_args;

/* One AdamW step on every tensor, with h = g * (s * c) (c = 1 without clipping):
 *     m <- beta1 m + (1 - beta1) h
 *     v <- beta2 v + (1 - beta2) h^2
 *     x <- x (1 - lr * weight_decay)
 *          - lr / (1 - beta1^step) * m / ( sqrt(v / (1 - beta2^step)) + eps )
 * in fp32, x being master, or else param (of a 16-bit type: read as fp32 and
 * rounded to nearest once).  With a master, param = RN(x).
 *   norm  device fp32: as for aspis_clip_grads, of all the list's gradients; NULL
 *         with max_norm < 0 (then work is NULL and skip_nonfinite 0 too)
 *   work  workspace, or NULL: norm is given
 * Parameters that follow other schedules go in lists of their own: take the norm of
 * all gradients once with aspis_grad_norm and give it to each list's call. */
aspis_status aspis_adamw(const aspis_params *params, const aspis_adamw_args *args, float *norm,
                         void *work, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* ASPIS_OPTIM_H */
