/*
 * libcce, embedding entry points: the lookup at the other end of the model from the LM head of
 * include/cce.h, and its gradient, for AMD MI355X (gfx950).
 *
 *   lookup    y_i = scale * W[t_i]            the rows of the (usually tied) LM-head matrix
 *   gradient  dW[v] (+)= scale * sum over {i : t_i = v} of dy_i
 *
 * With tied embeddings the gradient is added to the dW that cce_backward left (accumulate_dW != 0),
 * so that one tensor goes on to the gradient norm and the optimizer.
 *
 * Conventions are those of cce.h: DEVICE pointers owned by the caller, dense row-major, 16-byte
 * aligned (tokens, status: 4-byte); bf16 tensors are raw 16-bit patterns (void*); `stream` is a
 * hipStream_t as void*; nothing is allocated, freed or synchronised: the calls consist of kernel
 * launches only, and a stream under HIP graph capture may make them once each has been made once on
 * the device outside a capture; CCE_OK or a negative CCE_ERR_* code is returned and nothing is
 * enqueued on an error (CCE_ERR_HIP: as in cce.h).
 *
 * Sizes: N >= 1 tokens (below 2^31), V >= 1 rows (at most 2^24), D a positive multiple of 8 (at
 * most 65536), V * D at most 2^37: CCE_ERR_INVALID for sizes <= 0, CCE_ERR_UNSUPPORTED for the
 * other limits.
 *
 * A token equal to `ignore_index` (padding) or outside [0, V) takes no part: its row of y is zero,
 * its row of dy is never read (it may hold NaN) and no row of dW changes by it.  A token outside
 * [0, V) that is not `ignore_index` also sets CCE_STATUS_BAD_TOKEN in `status`.
 *   status  i/o int32 [1]  device, may be NULL: the bit is OR-ed in and nothing is ever cleared, so
 *           that one word can serve all calls of a step; the caller clears it
 */
#ifndef CCE_EMBED_H_
#define CCE_EMBED_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Lookup.
 *   tokens  in  int32 [N]
 *   weight  in  bf16 [V, D]
 *   out     out bf16 [N, D]   scale * weight row, formed in fp32 and rounded once (scale = 1: the row)
 */
int cce_embedding_forward(const int32_t* tokens, const void* weight, int64_t N, int64_t D, int64_t V,
                          int32_t ignore_index, float scale, void* out, int32_t* status, void* stream);

/* Bytes of device workspace cce_embedding_backward needs; 0 for invalid shapes.  A workspace of this
 * size also serves every smaller N at the same D and V.  Host only. */
size_t cce_embedding_workspace_bytes(int64_t N, int64_t D, int64_t V);

/*
 * Gradient of the lookup with respect to the matrix.
 *   tokens  in  int32 [N]
 *   d_out   in  bf16 [N, D]   gradient of `out`
 *   dW      out fp32 [V, D]   accumulate_dW == 0: overwritten, rows that no token names with zeros;
 *                             accumulate_dW != 0: added to, other rows are neither read nor written
 *   workspace  at least cce_embedding_workspace_bytes(N, D, V) bytes, 256-byte aligned; calls that may
 *              run at the same time need one each
 * Sums are fp32 in an order that the arguments decide: the same call gives the same bits.
 */
int cce_embedding_backward(const int32_t* tokens, const void* d_out, int64_t N, int64_t D, int64_t V,
                           int32_t ignore_index, float scale, float* dW, int accumulate_dW, int32_t* status,
                           void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* CCE_EMBED_H_ */
