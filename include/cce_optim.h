/*
 * libcce, optimizer entry points over many tensors at once, for AMD MI355X (gfx950): the steps that
 * include/cce_aux.h has for one tensor (gradient norm with its clipping coefficient, AdamW), for all
 * tensors of a model in a few launches, with moments in 32 or in 8 bits.
 *
 * Conventions are those of cce.h: tensor pointers are DEVICE pointers owned by the caller; `stream` is
 * a hipStream_t as void*; nothing is allocated, freed or synchronised: the calls consist of kernel
 * launches only, and a stream under HIP graph capture may make them once each has been made once on
 * the device outside a capture (a replay repeats the captured step: its tensors, its bias
 * corrections, its random numbers); CCE_OK or a negative CCE_ERR_* code is returned and nothing is
 * enqueued on an error (CCE_ERR_HIP: as in cce.h).
 *
 * `tensors` is a HOST array, read before the call returns and not kept: addresses may change from
 * call to call.  count >= 1.  A tensor of n = 0 values takes no part and its pointers are not looked
 * at; n is at most 2^33, all together 2^40 (CCE_ERR_UNSUPPORTED beyond).  The memory of no two entries
 * may overlap.
 */
#ifndef CCE_OPTIM_H_
#define CCE_OPTIM_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { CCE_STATE8_BLOCK = 128 };   /* values that share a scale in 8-bit moments */

typedef struct cce_optim_tensor {
    float* param;         /* i/o fp32 [n]  master parameters                                    16-byte aligned */
    void* param_bf16;     /* out bf16 [n]  their rounded copy; may be NULL                      16-byte aligned */
    const void* grad;     /* in  fp32 or bf16 [n]                                               16-byte aligned */
    void* m;              /* i/o first moment: fp32 [n], or uint8 [n] codes                     16-byte aligned */
    void* v;              /* i/o second moment: fp32 [n], or uint8 [n] codes of its square root 16-byte aligned */
    uint8_t* m_scale;     /* i/o [ceil(n / 128)]  NULL with moments in fp32 */
    uint8_t* v_scale;     /* i/o [ceil(n / 128)]  NULL with moments in fp32 */
    int64_t n;
    float lr_scale;       /* this tensor's learning rate is lr * lr_scale */
    float weight_decay;
    int32_t grad_bf16;    /* 0: grad is fp32, 1: bf16 */
    int32_t state8;       /* 0: moments in fp32, 1: in 8 bits */
} cce_optim_tensor;

/* Bytes of device workspace cce_grad_sumsq_multi needs for `count` tensors; 0 for count <= 0.  Host only. */
size_t cce_sumsq_multi_workspace_bytes(int64_t count);

/*
 * Sum of squares of all gradients and the clipping coefficient of their global norm (gradient-clipping
 * strategies).  Of `tensors` it reads grad, n and grad_bf16.
 *   sumsq      i/o fp64 [1] device, 8-byte aligned: accumulate == 0: set, != 0: added to (not finite if a
 *              gradient is not; the coefficient of a NaN is 1, as cce_clip_coef's)
 *   clip_coef  out fp32 [1] device, may be NULL: min(1, max_norm / (sqrt(sumsq) + eps_norm)) of the new
 *              sumsq; max_norm > 0 and eps_norm >= 0 are looked at only then
 *   workspace  at least cce_sumsq_multi_workspace_bytes(count) bytes, 256-byte aligned; calls that may
 *              run at the same time need one each
 * Squares and sums in fp64, in an order that the sizes alone decide.
 */
int cce_grad_sumsq_multi(const cce_optim_tensor* tensors, int64_t count, double* sumsq, int accumulate,
                         float max_norm, float eps_norm, float* clip_coef,
                         void* workspace, size_t workspace_bytes, void* stream);

/*
 * One AdamW step over all tensors: the formula of cce_adamw_step (include/cce_aux.h) with each tensor's
 * own learning rate and decay.  clip_coef in fp32 [1] device, may be NULL (= 1); step >= 1.
 *
 * Moments in 8 bits: a block of 128 values (the last one may be short) has codes c and a scale byte s:
 *   m  = e4m3(c) 2^(s - 127)     OCP E4M3: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7f, 0xff NaN
 *   v  = (u(c) 2^(s - 127))^2    unsigned: 4 exponent bits (bias 7), 4 mantissa bits; 0xff NaN, largest 480
 * Tensors of zero bytes are the moments before the first step.  A step forms the new moments in fp64 from
 * what the codes stand for, takes the update of param from them as they are, and rounds them to codes:
 * 2^(s - 127) is the smallest power of two, from 2^-100 to 2^120, with which the block's largest finite
 * |m| (sqrt(v)) is at most 448 (480), 1 for a block of zeros; a value between two codes goes up with the
 * probability of its place between them, in steps of 2^-17 (2^-16), and a sqrt(v) > 0 never to 0.  NaN,
 * infinite values and those beyond 448 (480) times 2^120 get a NaN code.  sqrt(v / bias correction) + eps is at least 2^-126 in the update.
 * Rounded to nearest, v could not follow a beta2 near 1: 0.1 % of it a step is far below half the
 * distance of two codes.
 * The random numbers are a hash of `seed`, `step` and the value's place in its tensor: the same call gives
 * the same bits.  `seed` is not used for moments in fp32, whose arithmetic is fp32 as in cce_adamw_step.
 */
int cce_adamw_multi_step(const cce_optim_tensor* tensors, int64_t count, float lr, float beta1, float beta2,
                         float eps, int64_t step, const float* clip_coef, uint32_t seed, void* stream);

/*
 * What 8-bit moments stand for, in fp32 (a checkpoint, an inspection).  n >= 1.
 *   codes   in  uint8 [n]               8-byte aligned
 *   scales  in  uint8 [ceil(n / 128)]
 *   second  0: the first moment; 1: the second moment (the squares)
 *   out     out fp32 [n]                16-byte aligned
 */
int cce_adamw_state8_read(const void* codes, const uint8_t* scales, int64_t n, int second, float* out, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* CCE_OPTIM_H_ */
