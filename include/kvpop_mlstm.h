/*
 * kvpop_mlstm.h -- C ABI of the recurrence of KVpop's delayed mLSTM scorer (gfx950 / MI355X):
 * the read-outs that the scores of kvpop_running_topk and kvpop_retain_step are made of
 * (KVpop Sec. 3.2 eqs. delayed_mlstm_readout and mlstm_score, App. E.3-E.5), for prompts and
 * training, its backward pass, and one token at a time. kvpop.h's conventions (streams,
 * ownership, status codes, threads) hold here too.
 *
 * Per sequence and head, with f_t = sigmoid(fg_t) and i_t = exp(ig_t), a matrix and a vector
 *   C_t = f_t C_{t-1} + i_t k_t v_t^T,   z_t = f_t z_{t-1} + i_t k_t
 * are held, and query t reads them delay tokens later (when token t leaves the protected
 * window): with x = scale q_t and t + delay below the sequence's length,
 *   o_t = x^T C_{t + delay} / (x . z_{t + delay})     normalize = 1 (scale cancels; for positive
 *                                                     features: o_t = 0 where x . z is not > 0)
 *   o_t = x^T C_{t + delay}                           normalize = 0.
 *
 * What is held keeps a common factor apart, so that no gate overflows it:
 *   m_t = max(m_{t-1} + log f_t, ig_t),  C = C_t e^-m_t,  z = z_t e^-m_t;  empty: C = z = 0, m = -inf.
 * m is fp32: kvpop_mlstm_fwd rounds it once, at its end (2^-25 |m| at most); kvpop_mlstm_step, which would lose a
 * slow decay with every token, makes C and z those of the rounded m.
 *
 * Gates: ig = -inf masks a token (its k and v do not matter then, NaN included), fg = -inf forgets
 * everything exactly (where a packed sequence begins), and so does any fg below -2^24, where an fp32 m or lse
 * has no bits left for another token's gate; fg = +inf forgets nothing. NaN, ig = +inf and
 * elements of the other inputs that are not finite reach the results of their sequence and head only (of all
 * that is packed into one of B). normalize = 0: a read-out's and a gradient's weights exp(b_u - b_t + ig_t) are fp32
 * numbers; above 2^127 they are infinite, and NaN where they meet a zero.
 */
#ifndef KVPOP_MLSTM_H
#define KVPOP_MLSTM_H

#include "kvpop_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct kvpop_mlstm {
  int32_t batch;     /* B >= 1 */
  int32_t n_heads;   /* H >= 1 */
  int32_t seq_len;   /* T >= 1 */
  int32_t head_dim;  /* D in {64, 128}: of q, k and v */
  int32_t delay;     /* w >= 0 */
  int32_t normalize; /* 1 or 0 */
  float scale;       /* finite, > 0 */
  kvpop_rows q;      /* bf16 [B, H, T, D] */
  kvpop_rows k;
  kvpop_rows v;
  kvpop_rows ig;     /* bf16 [B, H, T]: strides >= 0 of any size, ptr 2-byte aligned */
  kvpop_rows fg;
  const int32_t* lens; /* [B] or NULL (T): sequences' lengths, taken into [0, T] */
} kvpop_mlstm;

/* What is held, updated in place: C fp32 [B, H, D, D] (C[d][e] of k_d v_e), z fp32 [B, H, D],
 * m fp32 [B, H]. */
typedef struct kvpop_mlstm_state {
  float* C;
  float* z;
  float* m;
} kvpop_mlstm_state;

/* The read-outs of whole sequences. state NULL: from nothing held. Else what is held before the first
 * token goes in, what is held after the last comes out (a sequence of length 0 keeps it). Queries of tokens before
 * the call that are read in it: delay = 0, and q moved by the delay, theirs first.
 * o: bf16 [B, H, T, D] contiguous; rows that are not read (t + delay >= lens[b]) are 0.
 * lse: fp32 [B, H, T] or NULL: log of x . z (normalize = 1; -inf where that is not > 0) or 0
 * (normalize = 0); -inf for rows that are not read. kvpop_mlstm_bwd takes it.
 * Products are of bf16 operands with fp32 sums: within a chunk of 64 tokens a weight times its <x, k>, a
 * read state's element and o are each rounded to bf16 once. What is held adds a token's weight times v to
 * 16 bits, in fp32 sums. lse is of an x . z that is not rounded to bf16; o is divided by the sum of the weights that it is made
 * with, rounded, unless one of them is negative (features of either sign: x . z may cancel), then by x . z.
 * workspace: kvpop_mlstm_fwd_workspace_size bytes of device memory, 16-byte aligned (may be NULL
 * if that is 0); its contents on entry do not matter. Calls that may run at the same time, and
 * graphs, need workspaces of their own.
 * KVPOP_EINVAL: a missing pointer, sizes < 1, delay < 0, normalize not 0 or 1, scale not finite and
 * > 0, strides < 0, too small a workspace, or an output over an input or another one.
 * KVPOP_EUNSUPPORTED: head_dim, strides of q, k, v not multiples of 8, alignment (q, k, v, o, C, z
 * 16 bytes, the others that of their type), T > KVPOP_MAX_SEQ_LEN, or more than a launch takes
 * (2^32 - 1 threads; 1024 per head and 64 tokens). */
int kvpop_mlstm_fwd(const kvpop_mlstm* a, const kvpop_mlstm_state* state, void* o, float* lse, void* workspace,
                    size_t workspace_bytes, void* stream);
size_t kvpop_mlstm_fwd_workspace_size(const kvpop_mlstm* a);

/* The gradients of kvpop_mlstm_fwd without a state, from its o and lse: with b_t the sum of log f up to
 * t, W(u, t) = exp(b_u - b_t + ig_t - lse_u) for the query x_u that reads at time u >= t, and
 * d_u = -do_u . o_u (0 with normalize = 0):
 *   dx_u = sum_t W (do_u . v_t + d_u) k_t,   dk_t = sum_u W (do_u . v_t + d_u) x_u,
 *   dv_t = sum_u W (x_u . k_t) do_u,   dig_t = k_t . dk_t,
 *   dfg_t = sigmoid(-fg_t) sum_{s < t <= u} W(u, s) (x_u . k_s) (do_u . v_s + d_u).
 * Rows with lse = -inf give nothing. All are bf16 and contiguous: dq (scale dx), dk, dv [B, H, T, D];
 * dig, dfg [B, H, T]; 0 for tokens and queries that take no part. do_: bf16 [B, H, T, D] (strided),
 * o: bf16 [B, H, T, D] contiguous, lse: fp32 [B, H, T].
 * Roundings are those of kvpop_mlstm_fwd; for dq the read state's elements keep 16 bits. With normalize = 1, the
 * rounding of o is taken out of d_u (x . dx = 0 tells it). dfg is a running sum of differences: its error is
 * relative to the largest of a sequence's partial sums, not to each element, and about 2^-16 of the terms with
 * u = s, which cancel in it.
 * Nothing depends on the order of workgroups. workspace as above (kvpop_mlstm_bwd_workspace_size).
 * Errors as kvpop_mlstm_fwd. */
typedef struct kvpop_mlstm_grads {
  void* dq;
  void* dk;
  void* dv;
  void* dig;
  void* dfg;
} kvpop_mlstm_grads;
int kvpop_mlstm_bwd(const kvpop_mlstm* a, const kvpop_rows* do_, const void* o, const float* lse,
                    const kvpop_mlstm_grads* grads, void* workspace, size_t workspace_bytes, void* stream);
size_t kvpop_mlstm_bwd_workspace_size(const kvpop_mlstm* a);

/* One token of each sequence: k, v and the gates go into what is held, then q reads it (q is that
 * of the token `delay` before; seq_len is 1, delay 0, and the rows' stride_t means nothing).
 * lens: NULL, or 0 for idle sequences, which keep what they hold and get o = 0.
 * o: bf16 [B, H, D] contiguous. Errors as kvpop_mlstm_fwd, and seq_len != 1 or delay != 0. */
int kvpop_mlstm_step(const kvpop_mlstm* a, const kvpop_mlstm_state* state, void* o, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* KVPOP_MLSTM_H */
