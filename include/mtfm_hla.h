/*
 * mtfm_hla.h -- C ABI of hybrid linear attention with a decay for each head of libmtfm_hta.so, hand-written for AMD gfx950
 * (MI355X).
 *
 * The attention of mtfm_hta.h for jagged samples (a user's history tokens, followed by candidates that see the history and
 * themselves) with a state in place of the keys: cost linear in the history, and what a user's history amounts to is a
 * d x d matrix per query head, which serving keeps and brings up to date token by token.  With the decay
 * l = exp(log_decay[h]) of query head h and the keys and values of head h / (Hq / Hkv):
 *   history token i = 0 .. L-1   S_(i+1) = l S_i + k_i v_i^T        o_i = scale q_i S_(i+1)
 *   candidate t                  o_t = scale (l q_t S_L + <q_t, k_t> v_t)          (leaves no trace in the state)
 * S_0 is given (`state`) or zero, S_L is returned on request.  There is no softmax and no denominator: a normalization
 * (mtfm_rms.h, mtfm_gln.h) belongs behind it.
 * Backward: dq, dk, dv, and dstate, the gradient of S_0, from dout and (optionally) the gradient of S_L.  With
 * m_ij = l^(i-j) for a history key j that row i sees (candidates stand at i = L), 1 for a row's own key and 0 otherwise,
 * m_i0 = l^(i+1), w_j = l^(L-1-j):
 *   dq = scale [(dout v^T) m] k + scale m0 dout S_0^T            dk = scale [(dout v^T) m]^T q + w v dS_L^T
 *   dv = scale [(q k^T) m]^T dout + w k dS_L                     dS_0 = scale (m0 q)^T dout + l^L dS_L
 * The decay is a constant of the layer and has no gradient.  log_decay above 0 and NaN are taken as 0 (no decay).
 *
 * Layout: q, k, v, out and their gradients, offsets, hist_len, n_targets, layers and alignment as in mtfm_hta.h, element type
 * MTFM_HTA_BF16, head_dim 32, 64 or 128, Hq a multiple of Hkv.  States: [batch][Hq][head_dim (of k)][head_dim (of v)]
 * float32, 16-byte aligned.  final_state may be `state` itself, and dstate dfinal_state; other outputs overlap nothing.
 * Products take bf16 operands with float32 sums; the running state is float32, and what enters it is rounded no further than
 * to 16 bits of significand, and no further than to 24 where the caller gets the state.  Rows that belong to no user (behind the last one's, or beyond hist_len + n_targets) are not
 * touched.  What a row may not see does not reach it, whatever it holds; what sees an infinity or a NaN is not finite (and may be
 * NaN where the formula gives an infinity).  max_hist and max_targets bound what is looked at: a longer history or list is cut there.
 * Hq * head_dim at most 2^22, total_q and total_kv at most 2^30, batch * Hq * max(4 head_dim, 256) less than 2^32 - 2^27.
 *
 * Pointers are DEVICE pointers owned by the caller; `stream` is a hipStream_t passed as void* (NULL = the default stream).  The
 * calls validate their scalar arguments on the host, enqueue kernels and return; they never allocate, copy to the host or
 * synchronise, and may be captured.  Status codes, mtfm_hta_last_error() and mtfm_hta_validate_host() (for the offsets) are
 * those of mtfm_hta.h; on a non-zero status other than MTFM_HTA_ERR_LAUNCH nothing has been enqueued.  batch = 0 is valid.
 */
#ifndef MTFM_HLA_H
#define MTFM_HLA_H

#include "mtfm_hta.h"

#ifdef __cplusplus
extern "C" {
#endif

/* kernel kinds of this header for mtfm_hta_timing_read() */
enum { MTFM_HLA_KERNEL_FWD = 10,    /* forward, outputs */
       MTFM_HLA_KERNEL_STATES = 11, /* states of the pieces of long histories, either direction */
       MTFM_HLA_KERNEL_BWD = 12,    /* dq; dk, dv and dstate (two launches) */
       MTFM_HLA_KERNEL_SUM = 13,    /* dk, dv summed over the query heads of a group that one workgroup does not hold */
       MTFM_HLA_KERNEL_STEP = 14    /* single tokens */ };

/* Bytes of device workspace (0: none needed, workspace may be NULL; (size_t)-1: invalid or unsupported arguments). */
MTFM_HTA_API size_t mtfm_hla_workspace_bytes(int layer, int dtype, int is_bwd, int32_t batch, int64_t total_q, int64_t total_kv,
                 int32_t max_hist, int32_t max_targets, int32_t Hq, int32_t Hkv, int32_t head_dim);

/* Forward.  state: S_0 or NULL (zero); final_state: receives S_L, or NULL. */
MTFM_HTA_API int mtfm_hla_fwd(const void* q, const void* k, const void* v, const float* log_decay, const float* state, void* out,
                 float* final_state, const int32_t* q_offsets, const int32_t* kv_offsets, const int32_t* hist_len,
                 const int32_t* n_targets, int32_t batch, int64_t total_q, int64_t total_kv, int32_t max_hist,
                 int32_t max_targets, int32_t Hq, int32_t Hkv, int32_t head_dim, float scale, int dtype, int layer,
                 void* workspace, size_t workspace_bytes, void* stream);

/* Backward.  state: the forward pass's; dfinal_state: gradient of S_L or NULL (zero); dstate: receives the gradient of S_0,
 * or NULL.  dk and dv are sums over the query heads of a group, formed in float32 in a fixed order. */
MTFM_HTA_API int mtfm_hla_bwd(const void* dout, const void* q, const void* k, const void* v, const float* log_decay,
                 const float* state, const float* dfinal_state, void* dq, void* dk, void* dv, float* dstate,
                 const int32_t* q_offsets, const int32_t* kv_offsets, const int32_t* hist_len, const int32_t* n_targets,
                 int32_t batch, int64_t total_q, int64_t total_kv, int32_t max_hist, int32_t max_targets, int32_t Hq,
                 int32_t Hkv, int32_t head_dim, float scale, int dtype, int layer, void* workspace, size_t workspace_bytes,
                 void* stream);

/*
 * One history token for each of n_rows rows: q [n_rows][Hq][head_dim], k, v [n_rows][Hkv][head_dim], out like q; all in
 * float32 arithmetic.  state, new_state: pools [n_slots][Hq][head_dim][head_dim]; row i takes its state from slot slots[i]
 * (i itself if slots is NULL) of `state` and puts what follows into that slot of `new_state`, which may be `state` itself (else
 * they do not overlap); slots that no row names are not touched.  Rows that name the same slot are tokens of one user, in the
 * order of the rows.  A row whose slot is outside [0, n_slots) is padding: its output is zero.  `out` overlaps no input; n_rows * Hq
 * is less than 2^24 - 2^19.
 */
MTFM_HTA_API int mtfm_hla_step(const void* q, const void* k, const void* v, const float* log_decay, const float* state,
                 float* new_state, const int32_t* slots, void* out, int32_t n_rows, int32_t n_slots, int32_t Hq, int32_t Hkv,
                 int32_t head_dim, float scale, int dtype, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MTFM_HLA_H */
