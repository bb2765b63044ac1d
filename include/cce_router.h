/*
 * libcce, router of a mixture-of-experts layer, for AMD MI355X (gfx950): from each row's logits its top-k experts with
 * their weights, and what is added to the loss of include/cce.h in training -- the balance loss and the router's z
 * loss -- with their gradients.
 *
 *   p_ie  = softmax of row i's E logits          lse_i = log sum_e exp(logit_ie)
 *   chosen(i)  the top_k experts of the largest logits, equal ones by the lowest index
 *   weight     p of the chosen expert; with renormalize != 0 divided by the sum of the row's chosen ones
 *   c_e   = rows that chose expert e             P_e = sum_i p_ie             n = rows that take part
 *   losses[0] = E / (top_k n^2) sum_e c_e P_e    the balance loss: 1 where all experts get the same
 *   losses[1] = 1 / n sum_i lse_i^2              the z loss
 * Both are 0 for n = 0.  A caller adds them to its loss with coefficients of its own.
 *
 * A logit of -inf keeps an expert from a row: its p is 0 and it is never chosen; places of a row without an expert get index
 * -1 and weight 0.  A row whose label is ignore_index (padding) or that may use no expert takes no part: indices -1,
 * weights 0, lse 0, a gradient of 0; its logits may hold anything if the label says so.  Labels here mark rows that nothing reads: those of
 * the head's loss will not do where they ignore tokens that later ones attend to, as a prompt's in fine-tuning, which need their experts.  A NaN ranks before all numbers and +inf
 * next; both make NaN of the row's weights and lse, and so of P and both losses.
 *
 * Conventions are those of cce.h: DEVICE pointers owned by the caller, dense row-major, aligned to their elements; `stream`
 * is a hipStream_t as void*; nothing is allocated, freed or synchronised: the calls consist of kernel launches only, and a
 * stream under HIP graph capture may make them once each has been made once on the device outside a capture; CCE_OK or a
 * negative CCE_ERR_* code is returned and nothing is enqueued on an error (CCE_ERR_HIP: as in cce.h).  Outputs may not overlap
 * each other, an input or the workspace; in the backward pass d_logits may be logits' own memory.
 *
 * Sizes: N >= 1 rows (below 2^31), 1 <= top_k <= E; CCE_ERR_UNSUPPORTED for E beyond CCE_ROUTER_MAX_EXPERTS or top_k beyond
 * CCE_ROUTER_MAX_TOP_K.  Results do not depend on the run, and a row's own not on the other rows:
 * sums are taken in an order that the sizes, the type and the alignment of logits decide.
 */
#ifndef CCE_ROUTER_H_
#define CCE_ROUTER_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum { CCE_ROUTER_MAX_EXPERTS = 1024, CCE_ROUTER_MAX_TOP_K = 32 };

/* Bytes of device workspace cce_router_forward needs; 0 for sizes it refuses.  Host only. */
size_t cce_router_workspace_bytes(int64_t N, int64_t E);

/*
 *   logits      in  bf16 (logits_bf16 = 1) or fp32 (0) [N, E]
 *   labels      in  int32 [N], may be NULL: every row takes part
 *   indices     out int32 [N, top_k]    the likeliest expert first
 *   weights     out fp32 [N, top_k]
 *   lse         out fp32 [N]
 *   counts      out int32 [E + 1]       c, and behind it n
 *   prob_sums   out fp32 [E]            P
 *   losses      out fp32 [2]
 *   workspace   at least cce_router_workspace_bytes(N, E) bytes, 256-byte aligned; calls that may run at the same time need
 *               one each
 */
int cce_router_forward(const void* logits, int32_t logits_bf16, const int32_t* labels, int64_t N, int64_t E, int32_t top_k,
                       int32_t renormalize, int32_t ignore_index, int32_t* indices, float* weights, float* lse, int32_t* counts,
                       float* prob_sums, float* losses, void* workspace, size_t workspace_bytes, void* stream);

/*
 * d_logits (of logits' type) for the gradients of weights and losses; counts are constants, as in every balance loss.
 *   indices, lse, counts   in  what the forward pass left; counts may have been summed over the ranks of a job, for losses over
 *               the rows of all ranks.  A row whose first index is negative gets zeros and its logits are not read; another
 *               index outside [0, E) is passed over; the others of a row differ from each other.
 *   d_weights   in  fp32 [N, top_k], may be NULL (0); not read where there is no expert
 *   d_losses    in  fp32 [2] device, may be NULL (0)
 */
int cce_router_backward(const void* logits, int32_t logits_bf16, const int32_t* indices, const float* lse, const int32_t* counts,
                        const float* d_weights, const float* d_losses, int64_t N, int64_t E, int32_t top_k, int32_t renormalize,
                        void* d_logits, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* CCE_ROUTER_H_ */
