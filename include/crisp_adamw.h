/*
 * libcrisp, the step of fine-tuning (Alg. 1 line 11): one AdamW step over all tensors of a model, with the moments in 32 or
 * in 8 bits and the pruned positions held, and the bit mask of the hybrid pattern that it (and crisp_fp8_quant) takes.
 *
 * The conventions of crisp.h hold: status codes, arguments checked on the host before any device call, no allocation and
 * no synchronisation, work enqueued on `stream`.
 */
#ifndef CRISP_ADAMW_H
#define CRISP_ADAMW_H

#include "crisp.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { CRISP_P_F32 = 0, CRISP_P_BF16 = 1 };           /* element type of weights and of gradients */
enum { CRISP_MOMENTS_32 = 0, CRISP_MOMENTS_8 = 1 };

/*
 * One tensor of a step, its elements contiguous.  Device pointers, 16-byte aligned unless noted.
 * Moments in 32 bits: m and v are fp32, numel each.  In 8 bits, for blocks of 128 consecutive elements (the last one may be
 * short): m holds e4m3 values that stand for m[i] * m_scale[i / 128], v holds e4m3 values whose v[i] * v_scale[i / 128] is
 * the square root of the second moment.  Zeros in all four are the moments before the first step.
 */
typedef struct {
    void *w;                 /* weights, fp32 or bf16 per w_type; updated                                              */
    const void *g;           /* gradients, fp32 or bf16 per g_type                                                     */
    void *m, *v;             /* first and second moment; updated                                                       */
    float *m_scale, *v_scale;/* MOMENTS_8: ceil(numel/128) each, 4-byte aligned; updated.  NULL with MOMENTS_32        */
    uint16_t *w_copy;        /* optional, w_type F32 only: the new weights rounded to bf16                             */
    const uint32_t *mask;    /* optional: numel/row_len rows of ceil(row_len/32) words, bit k%32 of word k/32 set for  */
                             /* the kept columns of a row (as crisp_hybrid_mask writes it, or an nm_mask); 4-byte aligned */
    int64_t numel;           /* 0 .. 2^35; 0: nothing to do, no pointer is looked at                                   */
    int64_t row_len;         /* mask given: columns of a row, numel a multiple of it, both below 2^31; else ignored    */
    int32_t w_type, g_type;  /* CRISP_P_*                                                                              */
    int32_t moments;         /* CRISP_MOMENTS_*                                                                        */
    float weight_decay;      /* of this tensor, >= 0                                                                   */
} crisp_adamw_tensor;

/* Values of a step that are read on the device when it runs: a captured step replays with the values of the moment. */
typedef struct {
    float lr, grad_scale;
    int32_t step;            /* >= 1 (less counts as 1)                                        */
    int32_t skip;            /* not 0: the step changes nothing (gradients that overflowed)    */
} crisp_adamw_live;

typedef struct {
    double lr, beta1, beta2, eps;  /* lr >= 0, 0 <= beta < 1, eps > 0 also when rounded to fp32 (more than 2^-150) */
    double grad_scale;             /* gradients are multiplied by this first (clipping, a loss's scale)            */
    int64_t step;                  /* 1 .. 2^31 - 1: number of this step, for the correction of the moments' start */
    const crisp_adamw_live *live;  /* device, 4-byte aligned, or NULL: given, its lr, grad_scale and step replace  */
                                   /* the three above, which are then not looked at                                */
} crisp_adamw_hyper;

/*
 * One step of all tensors, in launches of up to 40 tensors of the same types.  Per element, in fp32, each operation rounded once:
 *   g' = g * grad_scale
 *   m  = beta1 * m + (1 - beta1) * g'
 *   v  = beta2 * v + (1 - beta2) * (g' * g')
 *   w  = w * (1 - lr * weight_decay) - (m / (sqrt(v) * (1 / sqrt(1 - beta2^step)) + eps)) * (lr / (1 - beta1^step))
 * (the scalars in parentheses are computed in fp64 and rounded to fp32), w rounded to its type.  The update uses the new
 * moments before they are rounded to 8 bits.  8-bit moments are rounded to nearest even with a block's scale
 * max(largest value / 448, 2^-126), except that a second moment that is not zero never becomes zero: the smallest code
 * stands for it, since the update would divide by eps alone in the next step.
 * A pruned position (mask bit not set) keeps its weight, its moments become zero, its gradient is not looked at; with
 * w_copy, the copy there has to hold the rounded weight already.
 * Without `live` a captured step replays with the lr, grad_scale and step that it was captured with.
 * The tensors' buffers must not overlap, and a tensor comes once.  tensors: host array of n_tensors elements (1 .. 2^20); everything is checked
 * before anything is enqueued.  Errors: EINVAL, ESHAPE, EALIGN, EDEVICE.
 */
CRISP_API crisp_status crisp_adamw_batch(int32_t n_tensors, const crisp_adamw_tensor *tensors,
                                         const crisp_adamw_hyper *hyper, void *stream);

/*
 * The hybrid pattern of a layer as one bit mask (Sec. 3.1: block sparsity AND N:M): mask is S x ceil(K/32) uint32, a bit set
 * where nm_mask has it and the block that holds it is in row_ptr / col_idx (outputs of crisp_select_mask).  mask may be
 * nm_mask itself.  All pointers device.  Errors: EINVAL, ESHAPE, EALIGN, EDEVICE.
 */
CRISP_API crisp_status crisp_hybrid_mask(const crisp_layer_desc *desc, const uint32_t *nm_mask, const int32_t *row_ptr,
                                         const int32_t *col_idx, uint32_t *mask, void *stream);

#ifdef __cplusplus
}
#endif
#endif
