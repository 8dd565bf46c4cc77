/*
 * ditpolicy.h -- the operators a policy update adds to the rollout of ditstep.h, in the same library
 * (libditstep.so) and under the same conventions: caller-owned device tensors, scratch from a caller's
 * workspace, asynchronous on `stream`, arguments checked before any launch, no device allocation.
 *
 *   packed_attention(_backward)  attention over packed sequences of different lengths, with grouped
 *                                heads and a causal mask, and its gradients: joint_attention for a batch
 *                                whose samples differ in text length or image size, the attention of a
 *                                causal text encoder, and one new token against a cache
 *   gated_norm(_backward)        the boundary between two sublayers of a block: residual + gate * branch,
 *                                with norms after the branch and before the next one, and its gradients
 *   flow_policy_loss             the clipped policy loss of one SDE step (flow_logprob's density, the
 *                                advantages of group_reward_stats) and its gradient for the velocity
 *
 * Packed rows. The rows of sequence i of a packed tensor are [off[i], off[i+1]), off a device array of
 * sequences + 1 int32. NULL offsets mean equal lengths: rows / sequences each, which has to be whole. The
 * host does not read device offsets: the kernels clamp them to the tensor's rows and take a sequence whose
 * end is before its start as empty, so bad offsets give wrong results but touch no other memory.
 * Output rows that belong to no sequence are left as they were.
 *
 * A call whose largest launch would take 2^32 threads or more is refused with DIT_ERR_UNSUPPORTED (attention: 256 to a tile of 16 to
 * 128 rows or keys of a head, one tile a sequence at least; norm: about hidden, to 8 rows; loss: 256 to a sample at least).
 *
 * Every result is the same from run to run: sums are taken in a fixed order, with no atomics.
 * Output tensors must not overlap inputs or each other, except where it is said below.
 */
#ifndef DITPOLICY_H
#define DITPOLICY_H

#include <stddef.h>
#include <stdint.h>

#include "ditstep.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ------------------------------------------------------------------ */
/* packed attention                                                     */
/* ------------------------------------------------------------------ */
/* Element (row, head, e) of a tensor is at base + row * X_row + head * X_head + e (strides in ELEMENTS,
 * 0 <= e < head_dim), so tensors may be slices of one packed projection [rows][heads + 2 kv_heads][d]. */
typedef struct {
  int32_t sequences;  /* >= 0 */
  int32_t heads;      /* query heads, a multiple of kv_heads */
  int32_t kv_heads;   /* query head j reads key/value head j / (heads / kv_heads) */
  int32_t head_dim;   /* 64 or 128 */
  int32_t total_q;    /* rows of q, o, lse */
  int32_t total_k;    /* rows of k, v */
  int32_t max_q;      /* no sequence has more queries than this (0: not known). It chooses the kernel and
                         its split of long keys; queries past it are not computed */
  int32_t causal;     /* nonzero: query i of m sees key j of n where j <= i + n - m (the last query sees
                         every key) */
  int32_t dtype;      /* dit_dtype of q, k, v, o and their gradients */
  float scale;        /* factor of q k^T, positive */
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;
} dit_packed_config;

/* Workspace bytes of the two calls (0 where none is needed, and for an invalid config). */
size_t packed_attention_workspace_bytes(const dit_packed_config* cfg);
size_t packed_attention_backward_workspace_bytes(const dit_packed_config* cfg);

/* o[i][h] = sum_j p_ij v_j, p_ij = exp(scale q_i.k_j - lse_i), lse_i = log sum_j exp(scale q_i.k_j), over the
 * visible keys j of the query's sequence; a query that sees none gets o = 0 and lse = -inf.
 * Scores are fp32, of any size; a query whose visible ones are all -inf (q k^T past the range of fp32) gets NaN in o, -inf in lse.
 *   q_offsets, k_offsets  rows of each sequence (device, or NULL)
 *   k_lengths  device [sequences] or NULL: only the first k_lengths[i] rows of sequence i's keys are used
 *              (a cache with room to grow); clamped to those rows
 *   lse        device [total_q][heads] fp32, or NULL
 * Keys outside the sequence are never read. A NaN or infinity in a key or value that the causal mask hides
 * from a query, but not from a later query of the same sequence, may still reach that query, if it sees any key.
 * Pointers and strides must keep 16-byte alignment of every (row, head); row strides are at least head_dim,
 * and o's (row, head) pieces must not overlap. DIT_ERR_UNSUPPORTED for a row stride of 2^24 elements or more
 * or a head stride of 2^40. */
dit_status packed_attention(const dit_packed_config* cfg, const void* q, const void* k, const void* v,
                            const int32_t* q_offsets, const int32_t* k_offsets, const int32_t* k_lengths,
                            void* o, float* lse, void* workspace, size_t workspace_bytes, dit_stream stream);

/* Gradients of packed_attention: d_o is the gradient of o, laid out like o; o and lse are the forward
 * call's. dq, dk and dv are laid out like q, k and v (whose (row, head) pieces must not overlap here). With p as
 * above, dv = p^T d_o, ds = p (d_o v^T - rowsum(d_o o)) scale, dq = ds k, dk = ds^T q; heads that share keys
 * add up. Key rows past k_lengths are left as they were; keys that no query sees get zeros. p comes from lse, of which fp32 holds
 * 2^-24 of its size: where |lse| is past 2^16 that is more than the rounding of bf16, and past 2^28 p may be any number. As forward, a NaN or infinity in a
 * row of a sequence may reach the gradients of rows that the causal mask sets apart from it, but dq of a query that sees no key is 0. */
dit_status packed_attention_backward(const dit_packed_config* cfg, const void* q, const void* k, const void* v,
                                     const void* o, const float* lse, const void* d_o,
                                     const int32_t* q_offsets, const int32_t* k_offsets, const int32_t* k_lengths,
                                     void* dq, void* dk, void* dv, void* workspace, size_t workspace_bytes,
                                     dit_stream stream);

/* ------------------------------------------------------------------ */
/* gated norm                                                           */
/* ------------------------------------------------------------------ */
typedef enum { DIT_NORM_NONE = 0, DIT_NORM_LAYER = 1, DIT_NORM_RMS = 2 } dit_norm_kind;

typedef struct {
  int32_t sequences;     /* >= 1 where rows > 0; each has its own gate, scale and shift */
  int32_t rows;          /* rows of x, y, h and their gradients: at most 2^28 */
  int32_t hidden;        /* 1..8192 */
  int32_t dtype;         /* dit_dtype of the row tensors and of the norm weights */
  int32_t post_norm;     /* dit_norm_kind of the branch y */
  int32_t pre_norm;      /* dit_norm_kind of h */
  float eps;             /* > 0 */
  float residual_scale;  /* factor of x, finite */
  int64_t x_row, y_row, h_row;  /* row strides in elements, at least hidden: of x, x_out and their gradients;
                                   of y and dy; of h and dh */
  int64_t mod_row;       /* row stride (floats) of gate, scale, shift and their gradients, at least hidden */
} dit_gated_norm_config;

/* x_out = residual_scale x + gate[s] u, u = post(y) post_w;  h = pre(x_out) pre_w (1 + scale[s]) + shift[s]
 * for the rows of sequence s, where layer(r) = (r - mean r) / sqrt(var r + eps), rms(r) = r / sqrt(mean r^2 +
 * eps) and none(r) = r. Statistics and sums are fp32; h is computed from x_out before its rounding.
 *   y NULL: x_out = residual_scale x (the first norm of a network)
 *   gate, scale, shift: device fp32 [sequences][hidden] at mod_row, each may be NULL (1, 0, 0)
 *   post_w, pre_w: [hidden], each may be NULL (1)
 *   x_out may be x (in place) and may be NULL; h may be NULL */
dit_status gated_norm(const dit_gated_norm_config* cfg, const void* x, const void* y, const void* post_w,
                      const void* pre_w, const float* gate, const float* scale, const float* shift,
                      const int32_t* offsets, void* x_out, void* h, dit_stream stream);

/* Workspace bytes of gated_norm_backward (0 for an invalid config). */
size_t gated_norm_backward_workspace_bytes(const dit_gated_norm_config* cfg);

/* Gradients of gated_norm at its output x_out, given those of x_out (dx_out, NULL: zero) and of h (dh, NULL:
 * zero, h unused). Row gradients dx (which may be dx_out) and dy, each may be NULL (not wanted); dy must be NULL
 * where y is. Vector gradients, fp32, each may be NULL: dgate, dscale, dshift [sequences][hidden] at mod_row (zeros for
 * an empty sequence), dpost_w, dpre_w [hidden]. Those of an input that was NULL in the forward call are the
 * gradients at its default. dgate and dpost_w must be NULL where y is. */
dit_status gated_norm_backward(const dit_gated_norm_config* cfg, const void* x_out, const void* y,
                               const void* post_w, const void* pre_w, const float* gate, const float* scale,
                               const int32_t* offsets, const void* dx_out, const void* dh, void* dx, void* dy,
                               float* dgate, float* dscale, float* dshift, float* dpost_w, float* dpre_w,
                               void* workspace, size_t workspace_bytes, dit_stream stream);

/* ------------------------------------------------------------------ */
/* policy loss of an SDE step                                           */
/* ------------------------------------------------------------------ */
size_t flow_policy_loss_workspace_bytes(int32_t batch, int64_t n_per_sample);

/* The clipped policy objective over the samples of one SDE step, and its gradient for the velocity. With mean, var
 * and logp as in flow_logprob (x, v, x_next [batch][n_per_sample] fp32),
 *   ratio[b] = exp(logp_scale (logp[b] - logp_old[b]))
 *   loss = 1/batch sum_b ( -min(ratio adv, clamp(ratio, 1 - clip_low, 1 + clip_high) adv)
 *                          + kl_weight logp_scale sum_i (mean - mean_ref)^2 / (2 var) )
 *   dv = d loss / d v   (a clipped sample has none from the first term; where both terms are equal the
 *                        unclipped one counts)
 * mean_ref is mean at the reference policy's velocity v_ref (NULL: no such term). logp_scale = 1 / n_per_sample
 * takes the density per element. t, t_next and noise_level are doubles (flow_logprob's are fp32: for a logp_old of its
 * making pass the values it was given, rounded to fp32). logp_old (fp64) and adv (fp32) are device [batch]. A sample with adv = 0 adds nothing, whatever its ratio.
 * Outputs (device), each may be NULL but one: loss [1], logp, ratio [batch], all fp64; dv [batch][n_per_sample]
 * fp32, which may be v. Sums are fp64. batch == 0 or n_per_sample == 0 writes nothing.
 * Errors: as flow_logprob; DIT_ERR_DOMAIN unless 0 <= clip_low <= 1, 0 <= clip_high, 0 <= kl_weight,
 * 0 < logp_scale, all finite; DIT_ERR_WORKSPACE. */
dit_status flow_policy_loss(const float* x, const float* v, const float* x_next, const float* v_ref, int32_t batch,
                            int64_t n_per_sample, double t, double t_next, double noise_level, const double* logp_old,
                            const float* adv, double logp_scale, double clip_low, double clip_high, double kl_weight,
                            double* loss, double* logp, double* ratio, float* dv, void* workspace,
                            size_t workspace_bytes, dit_stream stream);

#ifdef __cplusplus
}
#endif
#endif /* DITPOLICY_H */
