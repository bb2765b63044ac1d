/*
 * libcce, optimizer entry points for matrices, for AMD MI355X (gfx950): updates orthogonalised by
 * Newton-Schulz products (the Muon optimizer), for all matrices of a model in a few launches.  The tensors
 * that are no matrices (embedding, head, norms) go through include/cce_optim.h.
 *
 *   G of m x n, r = min(m, n):   X = G / (|G|_F + eps), transposed where m > n
 *   each step s:                 A = X X^T,   X = a_s X + (b_s A + c_s A A) X
 *   result:                      X, transposed back: the singular values of G moved towards 1
 *
 * Products take operands of 16 bits (fp16, power-of-two scales) and add in fp32; the diagonals of A and of b A + c A A
 * and what X loses by its rounding are held beside them.  With the coefficients 3.4445, -4.7750, 2.0315 and five steps the result, before it is
 * rounded to bf16, is off by 0.6 to 1.4e-3 of its 2-norm as a rule (what bf16's rounding adds is 1.7e-3), of low rank too, and by less than 2^-9 of it
 * unless roundings do not even out: where a few rows and columns hold nearly all of a few directions it is up to 2^-7 (5e-3 where it was tried, 6e-3
 * from 512 rows and 2.5 columns a row on, where two steps are taken as one), and of values that all round the same way, as a matrix of ones, 8e-3.
 * Coefficients and steps that amplify the smallest singular values more than those do (485 times) amplify what is rounded
 * along them as well.  Matrices with a side of up to 16, and thin ones (up to 64, the other side beyond 768 to 1024) take 64-bit products,
 * those with a side of up to 32 products of 22-bit operands: within 2^-13.
 *
 * Conventions are those of cce.h: matrix pointers are DEVICE pointers owned by the caller, dense row-major, aligned
 * to their elements; `stream` is a hipStream_t as void*; nothing is allocated, freed or synchronised: the
 * calls consist of kernel launches only, and a stream under HIP graph capture may make them once each has been
 * made once on the device outside a capture; CCE_OK or a negative CCE_ERR_* code is returned and nothing is
 * enqueued on an error (CCE_ERR_HIP: as in cce.h).
 *
 * Results do not depend on the run, but in their last bits on the list: the products of a list share their launches, and which tiles they take and
 * which sums are split goes by all of them.
 *
 * `matrices` is a HOST array, read before the call returns and not kept.  count >= 1.  A matrix with rows = 0 or
 * cols = 0 takes no part and its pointers are not looked at.  CCE_ERR_UNSUPPORTED: rows * cols, both rounded up to multiples
 * of 64, beyond 2^30, or the smaller side beyond 16384.  The memory of no two entries may overlap, nor the workspace any of it.
 */
#ifndef CCE_MUON_H_
#define CCE_MUON_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { CCE_NS_MAX_STEPS = 16 };

typedef struct cce_matrix {
    float* param;         /* i/o fp32 [rows, cols]  master parameters */
    void* out_bf16;       /* out bf16 [rows, cols]  cce_orthogonalize_multi: the result; cce_muon_multi_step: the
                             rounded copy of param, may be NULL */
    const void* grad;     /* in  fp32 or bf16 [rows, cols] */
    float* momentum;      /* i/o fp32 [rows, cols]  zeros before the first step */
    int64_t rows, cols;
    float lr_scale;       /* this matrix's learning rate is lr * lr_scale */
    float weight_decay;   /* param decays by 1 - lr * lr_scale * weight_decay, see cce_muon_multi_step */
    int32_t grad_bf16;    /* 0: grad is fp32, 1: bf16 */
    int32_t reserved;     /* 0 */
} cce_matrix;

/* Bytes of device workspace both calls need for these matrices (rows and cols are read); at least 256; 0 where a call would
 * refuse the sizes.  Host only.  A part of the list is worked on at a time, in at most 3 GB, or what the largest matrix needs: 5
 * bytes a value and 4 for each of the square of its smaller side; 64 MB of it for parts of long sums. */
size_t cce_muon_workspace_bytes(const cce_matrix* matrices, int64_t count);

/*
 * out_bf16 = the orthogonalised grad.  Of `matrices` it reads grad, rows, cols and grad_bf16.
 *   coefficients  HOST fp32 [steps][3]: a, b, c of each step; 1 <= steps <= CCE_NS_MAX_STEPS.  CCE_ERR_UNSUPPORTED where they
 *                 let a singular value grow beyond 2.5, or |b| x^2 + |c| x^4 beyond 60 for it: the 16-bit operands' range
 *   eps           >= 0; with 0 a matrix of zeros gives NaN
 *   workspace     at least cce_muon_workspace_bytes(matrices, count) bytes, 256-byte aligned; calls that may run at
 *                 the same time need one each
 * A matrix that holds a NaN or an infinity gives NaN in all of its values, and in no other matrix.
 */
int cce_orthogonalize_multi(const cce_matrix* matrices, int64_t count, const float* coefficients, int32_t steps, float eps,
                            void* workspace, size_t workspace_bytes, void* stream);

/*
 * One step of momentum, orthogonalisation and update over all matrices:
 *   g        = clip_coef * grad
 *   momentum = mu momentum + (1 - mu) g
 *   G        = mu momentum + (1 - mu) g (nesterov != 0) or momentum
 *   param    = (1 - lr lr_scale weight_decay) param - lr lr_scale orthogonalised(G);   out_bf16 = its rounded copy
 *   clip_coef  in fp32 [1] device, may be NULL (= 1);   0 <= mu < 1;   lr, lr_scale, weight_decay >= 0
 * Decay goes with the matrix's own learning rate, as in cce_optim.h.  The optimizer as published decays every matrix by 1 - lr * wd, its shape's
 * factor in the update alone: weight_decay = wd / lr_scale is that.  (With wd itself and lr_scale = 0.2 sqrt(max(rows, cols)) a matrix of 14336
 * rows decays 24 times as fast.)
 * Everything beside the products in fp32; the orthogonalised G goes into param without being rounded to 16 bits.
 */
int cce_muon_multi_step(const cce_matrix* matrices, int64_t count, float lr, float mu, int32_t nesterov,
                        const float* coefficients, int32_t steps, float eps, const float* clip_coef,
                        void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* CCE_MUON_H_ */
