/*
 * bgpo_train.h -- C ABI of the token-level policy step on an LM head (GB300, sm_103a).
 *
 * bgpo.h takes hidden states to a sequence-level objective. These calls are for
 * objectives on the log-probability of each token, or on each Monte Carlo sample's
 * l, and for what follows a backward pass:
 *
 *   bgpo_token_logp_fwd   log p(y_i) of selected response tokens through the LM head
 *   bgpo_token_logp_bwd   their gradient: dL/dlogp -> dX, dW (bf16)
 *   bgpo_policy_loss      clipped policy loss with a KL term, and its gradient
 *   bgpo_preference_loss  loss on paired log ratios, and its gradient
 *   bgpo_grad_norm        global norm of many gradients
 *   bgpo_grad_clip        the gradients scaled to a largest norm
 *
 * The conventions of bgpo.h hold: device pointers on the current device, asynchronous
 * launches on `stream`, no allocation, host-side checks before any launch, a status
 * for each call, device-detected faults in the error word of the workspace
 * (bgpo_get_device_error, bgpo_clear_device_error). Results are deterministic: sums
 * have a fixed order and no atomic decides one. The sums of the losses and of the norm
 * are fp32 in trees of a bounded depth; where a chain grows with the sizes it carries what
 * its roundings leave out, so that their error does not grow with the batch.
 */
#ifndef BGPO_TRAIN_H_
#define BGPO_TRAIN_H_

#include "bgpo.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * A 2-D array given by strides: element (i, t) lies at data + i * row + t * col
 * (strides in elements, >= 0; 0 repeats an input along that axis). A transposed
 * [n_t, B] array of l is a [B, n_t] view with row = 1, col = B. data is aligned to
 * its element; NULL stands for an absent optional array. The last element lies at most
 * 2^42 elements after the first (BGPO_ERR_SHAPE otherwise). Fastest are arrays that run
 * along memory (col = 1), with one row stride and one alignment modulo 32 bytes (8 of a mask).
 */
typedef struct bgpo_view {
  const void* data;
  int64_t row;
  int64_t col;
} bgpo_view;

/* ---- token log-probabilities through the LM head ------------------------------------ */

/*
 * logp[b, i] = log softmax(W x_{b, P + i})[Y[b, i]] for the selected response positions, 0
 * for the others. Selected: mask[b, i] nonzero (every position where mask is NULL) and
 * i < resp_len[b] (where prob->resp_len is given). Logits are bf16 products summed in fp32
 * and never stored (with BGPO_FLAG_KEEP_LOGITS they stay in the workspace for the
 * backward). Of `prob`, the sizes, resp_len, flags, vocab_chunk and trace matter;
 * BGPO_FLAG_PAIR_DW is refused (BGPO_ERR_INVALID_ARG). ws is a workspace of
 * bgpo_workspace_bytes(prob), also one that held MC samples before: it then holds the
 * selected tokens, until the next bgpo_sample_mask. (A sample left pending under dW
 * pairing is dropped, which sets the error word to BGPO_ERR_INVALID_ARG.)
 *   mask      device uint8 [B, R] or NULL;  X, W, Y as for bgpo_elbo_fwd (a selected
 *             target outside [0, V) gives NaN; others are not looked at)
 *   logp_out  device float [B, R], written whole
 */
bgpo_status bgpo_token_logp_fwd(const bgpo_problem* prob, const uint8_t* mask, const void* X,
                                const void* W, const int32_t* Y, void* ws, size_t ws_bytes,
                                float* logp_out, void* stream);

/*
 * Gradient of sum dlogp[b, i] logp[b, i] over the tokens that the preceding
 * bgpo_token_logp_fwd on this workspace selected (same prob, X, W and Y):
 *   dz_r = dlogp_r (onehot(y_r) - softmax(W x_r))
 *   dX[b, i] = W^T dz_r (0 where not selected),  dW = sum_r dz_r x_r^T
 * Both are sums in fp32 rounded once to bf16, the type of X and W: what a bf16 network's
 * backward takes. dz is rounded to bf16 before the two products, as their tensor cores
 * take it (like W and X): beyond 128 selected tokens dX and dW are 0.0024 of their norm off,
 * of which bf16 outputs alone make 0.0017. Up to 128 tokens, where one entry's rounding
 * would show, what it leaves out goes through the products too, and only the outputs'
 * rounding is left. They are written whole, not accumulated; dlogp of positions that were
 * not selected is not read. May be repeated with another dlogp.
 *   dlogp device float [B, R];  dX device bf16 [B, R, H], dW device bf16 [V, H], 16-byte
 *   aligned
 * Without a preceding bgpo_token_logp_fwd of a problem of the same B, P, R, H, V, chunk width
 * and BGPO_FLAG_KEEP_LOGITS, the error word is set to BGPO_ERR_INVALID_ARG and dX and dW are
 * not written.
 */
bgpo_status bgpo_token_logp_bwd(const bgpo_problem* prob, const void* W, const float* dlogp,
                                void* ws, size_t ws_bytes, void* dX, void* dW, void* stream);

/* ---- workspace of the losses and of the gradient norm ---------------------------- */

/*
 * Bytes of device workspace the losses and the gradient norm need, whatever their sizes.
 * One workspace serves calls of different kinds, one after the other on one stream.
 */
size_t bgpo_train_workspace_bytes(void);

/* Clears the workspace's error word and counters (asynchronous on `stream`). Clear a
 * new workspace before its first call, and one whose last call returned BGPO_ERR_CUDA. */
bgpo_status bgpo_train_workspace_clear(void* ws, size_t ws_bytes, void* stream);

/* ---- clipped policy loss with a KL term ------------------------------------------- */

/* Ratio of the policies: per token, or one per row from the mean log ratio. */
#define BGPO_RATIO_TOKEN 0     /* r_{b,i} = e^{d_{b,i}},  d = logp - logp_old */
#define BGPO_RATIO_SEQUENCE 1  /* r_b = e^{(1 / n_b) sum_i m_{b,i} d_{b,i}} */

/* Weight w_b of a token of row b (n_b tokens of row b count, m = 1). */
#define BGPO_NORM_ROWS 0    /* scale / (N n_b): the mean over rows of their tokens' mean */
#define BGPO_NORM_TOKENS 1  /* scale / sum_b n_b: the mean over all tokens */
#define BGPO_NORM_SUM 2     /* scale: a plain sum */

/*
 * For tokens (b, i), 0 <= b < N, 0 <= i < T, with m = 1:
 *   u   = -min(r A, clip(r, 1 - clip_low, 1 + clip_high) A)
 *   k   = logp_ref - logp,  q = e^k - 1 - k  (an estimate of KL(policy || reference))
 *   L   = sum_{b,i} w_b m (u + beta q)
 *   dlogp = dL/dlogp = w_b m (-A r [not clipped] + beta (1 - e^k))
 * A token is clipped when A > 0 and r > 1 + clip_high, or A < 0 and r < 1 - clip_low.
 * With BGPO_RATIO_SEQUENCE the gradient flows through the row's ratio; since r_b is a
 * mean, each of the row's tokens gets -w_b A_b r_b as above. A row without tokens
 * contributes nothing. Values of masked-out tokens are never used, and their dlogp is 0; they
 * may be loaded beside tokens that count, so that all N T elements have to be readable (and
 * not being written meanwhile).
 *   logp, logp_old, logp_ref, adv   float; logp_ref optional (then beta must be 0);
 *       adv with col = 0 is one advantage a row, which BGPO_RATIO_SEQUENCE requires
 *   mask    uint8, nonzero = the token counts; optional (every token counts)
 *   dlogp   float, written whole (zeros included); optional (the loss alone). It must
 *       not overlap itself or an input.
 *   out     device float [6]: L, sum w m u, sum w m q, and over the tokens that count
 *       the share clipped below, the share clipped above and the mean ratio
 *       (0 when no token counts)
 *   clip_low, clip_high >= 0 (clip_high may be infinite); beta, scale finite
 * A non-finite L sets the device error word to BGPO_ERR_NONFINITE (values are written).
 * Sizes: N, T >= 1, N <= 2^28, T <= 2^30, N T <= 2^38.
 */
typedef struct bgpo_policy_loss_args {
  int32_t N, T;
  int32_t ratio, norm;
  float clip_low, clip_high, beta, scale;
  bgpo_view logp, logp_old, logp_ref, adv, mask, dlogp;
  float* out;
  bgpo_trace* trace; /* optional, as in bgpo_problem */
} bgpo_policy_loss_args;

bgpo_status bgpo_policy_loss(const bgpo_policy_loss_args* args, void* ws, size_t ws_bytes,
                             void* stream);

/* ---- preference loss on paired log ratios ------------------------------------------ */

#define BGPO_PREF_SIGMOID 0  /* -(1 - smoothing) log s(h) - smoothing log s(-h), s the sigmoid */
#define BGPO_PREF_HINGE 1    /* max(0, 1 - h) */
#define BGPO_PREF_IPO 2      /* (h - 1/2)^2 / beta^2 */

/*
 * Pair k of K holds row k of the chosen and row k of the rejected arrays:
 *   S   = sum_i m (logp - ref) over a row, divided by its token count if `average`
 *   h_k = beta (S_chosen - S_rejected) - margin
 *   L   = scale / K sum_k loss(h_k)
 *   d_chosen = dL/dlogp = m loss'(h) beta scale / K (/ n),  d_rejected = the negative
 *       with the rejected row's m and n
 * A row without tokens has S = 0. Values of masked-out tokens are never used but may be
 * loaded, as in bgpo_policy_loss; their gradients are 0.
 *   chosen, rejected           float [K, T_chosen], [K, T_rejected]
 *   ref_*                      float, both or neither (then S = sum m logp)
 *   mask_*                     uint8, nonzero = the token counts; each optional
 *   d_chosen, d_rejected       float, written whole, both or neither; they must overlap
 *                              neither themselves, each other nor an input
 *   margins                    device float [K] or NULL: h
 *   out                        device float [5]: L, the share of pairs with h > 0, and the
 *                              means of h, of beta S_chosen and of beta S_rejected
 *   beta, margin, scale finite (beta != 0 for BGPO_PREF_IPO), 0 <= smoothing <= 1 (0
 *   unless BGPO_PREF_SIGMOID)
 * A non-finite L sets the device error word to BGPO_ERR_NONFINITE (values are written).
 * Sizes: K, T_chosen, T_rejected >= 1, 2 K <= 2^28, T <= 2^30, 2 K T <= 2^38.
 */
typedef struct bgpo_preference_loss_args {
  int32_t K, T_chosen, T_rejected;
  int32_t kind, average;
  float beta, margin, smoothing, scale;
  bgpo_view chosen, ref_chosen, mask_chosen, d_chosen;
  bgpo_view rejected, ref_rejected, mask_rejected, d_rejected;
  float* margins;
  float* out;
  bgpo_trace* trace; /* optional, as in bgpo_problem */
} bgpo_preference_loss_args;

bgpo_status bgpo_preference_loss(const bgpo_preference_loss_args* args, void* ws, size_t ws_bytes,
                                 void* stream);

/* ---- global gradient norm and clipping ----------------------------------------------- */

#define BGPO_F32 0
#define BGPO_BF16 1
#define BGPO_F16 2

/*
 * One gradient of a list (host struct): n contiguous elements of `type` at `data`. `out`
 * receives the clipped gradient as n elements of `out_type`; out = data (and the same
 * type) clips in place. Pointers aligned to their elements; fastest where data and out lie
 * equally many elements past a boundary of eight. A tensor of n = 0 elements is skipped (its
 * pointers may be NULL).
 */
typedef struct bgpo_grad {
  const void* data;
  void* out;
  int64_t n;
  int32_t type, out_type;
} bgpo_grad;

/*
 * norm_out = sqrt(sum of the squares of all elements of all gradients): the Euclidean
 * norm, as one device float. Squares and their sums within a unit of 8,192 elements are
 * fp32; sums of those carry what their roundings leave out. A norm beyond 1.8e19 comes out
 * infinite; squares below 1e-38 (elements below 1e-19) lose bits, and elements below 2e-23
 * count as zero. An empty
 * list has norm 0. A non-finite norm sets the device error word to BGPO_ERR_NONFINITE (the
 * value is still written).
 * `out` and `out_type` are not used; trace is optional. n of a tensor at most 2^40, of the
 * list 2^44.
 */
bgpo_status bgpo_grad_norm(const bgpo_grad* grads, int32_t count, float* norm_out,
                           bgpo_trace* trace, void* ws, size_t ws_bytes, void* stream);

/*
 * out = f x for every gradient, f = min(1, max_norm / (norm + 1e-6)), with norm a device
 * float: bgpo_grad_norm's, or that of a larger set this one is a part of. Where norm is
 * not finite, f = 1 and the error word of ws (optional) is set to BGPO_ERR_NONFINITE: the
 * caller decides whether to step. Products are fp32, rounded once to the output's type.
 * Gradients clipped in place with f = 1 are neither read nor written. max_norm >= 0 and
 * finite. An output overlaps no other gradient or output, and its own gradient only in
 * place: list a tensor once.
 */
bgpo_status bgpo_grad_clip(const bgpo_grad* grads, int32_t count, const float* norm,
                           float max_norm, bgpo_trace* trace, void* ws, size_t ws_bytes,
                           void* stream);

#ifdef __cplusplus
}
#endif

#endif /* BGPO_TRAIN_H_ */
