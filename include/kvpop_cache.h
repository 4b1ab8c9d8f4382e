/*
 * kvpop_cache.h -- C ABI of the compact KV cache of a KVpop model (gfx950 / MI355X):
 * what serving needs next to the rankings and the sparse attention of kvpop.h, whose
 * conventions (streams, ownership, status codes, threads) hold here too.
 *
 * A served sequence keeps, for each KV head, a list of the tokens that the running
 * top-k retains (KVpop Sec. 3 eq. kv_budget: sinks, protected window and k long-range
 * tokens per head; App. C.1). Heads keep different tokens, so every list has pages of
 * its own. One decode step is
 *
 *   kvpop_retain_step    which slot of each list the new token takes
 *   kvpop_cache_append   its key and value into that slot, rotated and in 8 bits
 *   kvpop_cache_attn     the new queries over the lists
 *
 * and a prompt ends with kvpop_running_topk (evict), kvpop_retain_prompt and a
 * kvpop_cache_append that gathers the tokens each head keeps. The parts also serve
 * alone: append and attend work on any lists, evicted from or not.
 *
 * The cache
 * ---------
 *  - A page holds P = page_size tokens of one KV head (P 16, 32, 64 or 128) as 8-bit
 *    codes [P, D]; the pool has n_pages of them for keys and as many for values. The
 *    list of (b, h) is the pages page_table[b, h, 0 .. max_pages - 1], of which slot j
 *    (token j of the list) is row j % P of entry j / P. held[b, h] says how many slots
 *    are in use; slots are in use from 0 on without gaps.
 *  - A page's values are code * 2^e, e = k_exp[page] or v_exp[page] in [-32, 32]
 *    (outside of it the nearest bound is meant). Codes are signed bytes in
 *    [-127, 127] (KVPOP_CACHE_INT8) or e4m3 without infinities (KVPOP_CACHE_E4M3,
 *    largest 448). With a power of two as its scale a value's code is one rounding of
 *    the value, and a page whose scale grows moves its codes exactly, except for e4m3
 *    codes that become subnormal and for int8, which round once more.
 *  - Lists may share pages that are only read. A page that a call writes appears once
 *    among the lists' entries that the call writes, or that page's contents are undefined.
 *  - A page_table entry outside [0, n_pages) holds no page: nothing is written there
 *    and its tokens are not attended to.
 */
#ifndef KVPOP_CACHE_H
#define KVPOP_CACHE_H

#include "kvpop.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { KVPOP_CACHE_INT8 = 0, KVPOP_CACHE_E4M3 = 1 };

typedef struct kvpop_cache {
  int32_t batch;             /* B >= 1 */
  int32_t n_kv_heads;        /* Hkv >= 1 */
  int32_t head_dim;          /* D in {64, 128} */
  int32_t format;            /* KVPOP_CACHE_INT8 or KVPOP_CACHE_E4M3 */
  int32_t page_size;         /* P in {16, 32, 64, 128} */
  int32_t n_pages;           /* >= 1 */
  int32_t max_pages;         /* entries per list, >= 1; max_pages * P <= KVPOP_MAX_SEQ_LEN */
  void* k_pages;             /* [n_pages, P, D] bytes */
  void* v_pages;             /* [n_pages, P, D] bytes */
  int8_t* k_exp;             /* [n_pages] */
  int8_t* v_exp;             /* [n_pages] */
  const int32_t* page_table; /* [B, Hkv, max_pages] */
} kvpop_cache;

/* A bf16 array [B, heads, tokens, D] with its strides in elements: each >= 0 and a
 * multiple of 8, the last dimension contiguous, ptr 16-byte aligned. */
typedef struct kvpop_rows {
  const void* ptr;
  int64_t stride_b, stride_h, stride_t;
} kvpop_rows;

/* What kvpop_cache_append adds. */
typedef struct kvpop_append {
  int32_t n_tokens;     /* N >= 1: tokens in k and v (and q) */
  int32_t n_entries;    /* M >= 1: most slots written per list; M = N without src */
  kvpop_rows k;         /* [B, Hkv, N, D] */
  kvpop_rows v;         /* [B, Hkv, N, D] */
  const int32_t* held;  /* [B, Hkv]: tokens in each list after the call */
  const int32_t* count; /* [B, Hkv] or NULL: slots to write (taken into [0, M]); NULL: M */
  const int32_t* start; /* [B, Hkv] or NULL: first slot, negative: nothing is written
                           to that list; NULL: held - count, the list's end */
  const int32_t* src;   /* [B, Hkv, M] or NULL: which token each slot takes; NULL: 0, 1, ... */
  const int32_t* pos0;  /* [B] or NULL (0): position of token 0 */
  const float* cos;     /* fp32 [n_positions, rot_dim / 2], both NULL if rot_dim = 0 */
  const float* sin;
  int32_t n_positions;
  int32_t rot_dim;      /* R: 0 or a multiple of 16 up to D; the first R of a head turn */
  int32_t adjacent;     /* pairs: 0 = (j, j + R / 2), 1 = (2 j, 2 j + 1) */
  int32_t n_q_heads;    /* Hq, 0 without q */
  kvpop_rows q;         /* [B, Hq, N, D], or ptr NULL */
  void* q_out;          /* bf16 [B, Hq, N, D] contiguous: the rotated queries */
} kvpop_append;

/* Appends keys and values to the lists, keys rotated by their positions:
 * for i < count[b, h], with token n = src[b, h, i] (or i) at position p = pos0[b] + n,
 *   slot start[b, h] + i  takes  R(p) k[b, h, n, :]  and  v[b, h, n, :],
 *   R(p): (a, b) -> (a cos[p, j] - b sin[p, j], b cos[p, j] + a sin[p, j]) on pair j < R / 2.
 * Per page that gets tokens, and for keys and values apart: x's needed exponent is the
 * least e in [-32, 32] with |x| <= qmax 2^e (qmax 127 or 448) for every finite x
 * written; if the call leaves other tokens of the list in the page (slots below
 * held[b, h] that it does not write), the page takes the larger of this and its own
 * exponent and their codes move to it; if not, it takes this one. A code is x 2^-e
 * rounded to nearest, ties to even, saturated at qmax; NaN becomes 0 and an infinity
 * the largest code of its sign. Keys are rotated in 64 bits, so that the code is the
 * one rounding of the value. Slots at or past max_pages * P are not written. A token
 * outside [0, N) is stored as zeros, key and value. At a position outside
 * [0, n_positions) (with rot_dim > 0) the key is stored as zeros and the value as it is, so
 * that attention finds the token with a logit of 0. Slots that no token uses keep their bytes.
 * q_out[b, h, n, :] = R(pos0[b] + n) q[b, h, n, :], rotated in 32 bits and rounded to bf16
 * (zeros at a position outside the table), for all N tokens.
 * KVPOP_EINVAL: a missing pointer, dimensions or strides out of range, M != N without
 * src, q without q_out, or q_out or the cache over an input or each other.
 * KVPOP_EUNSUPPORTED: head_dim, page_size, format, rot_dim not a multiple of 16,
 * strides not multiples of 8, alignment (the int32 arrays need 4 bytes, the
 * exponents 1, the others 16), or more than one launch takes (2^32 - 1 threads, of
 * which a page that a list may reach into takes 128 or more). */
int kvpop_cache_append(const kvpop_cache* cache, const kvpop_append* a, void* stream);

/* Attention of the newest N queries of each sequence over its lists. For sequence b
 * with n = q_lens[b] queries (NULL: N; taken into [0, N]), query i < n of query head
 * qh (KV head h = qh / G, G = Hq / Hkv) sees the slots j < held[b, h] - (n - 1 - i): the
 * last n slots are the queries' own tokens, in order. (So several queries at once are for
 * lists that their tokens were added to at the end; a slot that kvpop_retain_step takes from
 * another token serves single queries, which see the whole list.) With values k_j, v_j of the list
 *   lse[b, qh, i]  = log sum_j exp(scale <q_i, k_j>)
 *   o[b, qh, i, :] = sum_j exp(scale <q_i, k_j> - lse) v_j.
 * A query that sees nothing, and rows i >= n, get o = 0 and lse = -inf. held is taken
 * into [0, max_pages * P]. Bytes of slots that a query does not see do not matter,
 * except an e4m3 NaN (which kvpop_cache_append never writes) in a slot that another
 * query of the same call sees. Products are of 16-bit operands with fp32 sums: codes
 * are exact there, and a query's elements are exact down to 2^-28 of its largest. A
 * probability times 2^e of its values' page is rounded to 11 bits where it is above 2^-21
 * of the largest such number of its query, and to 2^-32 of that one below; the
 * normaliser sums the probabilities unrounded. Logits are fp32: they, and scale |q| 2^e of a
 * query's largest element and any page's e of keys, have to lie within +-2^125. What a query
 * with an element that is not finite gets means nothing; the others' results stay the same.
 * q: bf16 [B, Hq, N, D]; o: bf16 [B, Hq, N, D] contiguous; lse: fp32 [B, Hq, N].
 * workspace: kvpop_cache_attn_workspace_size bytes of device memory, 16-byte aligned
 * (may be NULL if that is 0); its contents on entry do not matter. Calls that may run
 * at the same time, and graphs, need workspaces of their own.
 * KVPOP_EINVAL: a missing pointer, Hq % Hkv != 0, N < 1, scale not finite and > 0,
 * strides < 0, too small a workspace, or an output over an input, the cache or the
 * other. KVPOP_EUNSUPPORTED: as above, or Hq / Hkv > 1024. */
int kvpop_cache_attn(const kvpop_cache* cache, int32_t n_q_heads, int32_t n_tokens, float scale, const kvpop_rows* q,
                     const int32_t* held, const int32_t* q_lens, void* o, float* lse, void* workspace,
                     size_t workspace_bytes, void* stream);

/* Bytes of workspace for these sizes (pointers in `cache` are not looked at); 0 also
 * for invalid ones. */
size_t kvpop_cache_attn_workspace_size(const kvpop_cache* cache, int32_t n_q_heads, int32_t n_tokens);

/* One KV head's retained tokens while it decodes: pos (positions) and prio (static
 * priorities fl(r_t - fl(t log_gamma[h])), as in kvpop_running_topk) of slots
 * 0 .. held - 1, in no order. */
typedef struct kvpop_retain {
  int32_t batch;    /* B >= 1 */
  int32_t n_heads;  /* H >= 1 (KV heads) */
  int32_t slots;    /* S >= 1: room per list */
  int32_t* pos;     /* [B, H, S] */
  float* prio;      /* [B, H, S] */
  int32_t* held;    /* [B, H] */
} kvpop_retain;

/* What a prompt leaves behind: for sequence b of n = lens[b] tokens (NULL: T; taken into
 * [0, T]) the tokens t < n with evict[b, h, t] >= n, which are those that its last query
 * keeps, in ascending order. pos[b, h, i] and prio[b, h, i] of the i-th, i < held[b, h];
 * the other slots get -1 and -inf. Tokens beyond the first S do not fit and are dropped:
 * with evict from kvpop_running_topk and S >= sinks + window + topk there are none.
 * scores: fp32 [B, H, T] (of kvpop_running_topk); evict: int32 [B, H, T]; log_gamma: fp32
 * [H] or NULL. All of st's arrays are outputs. evict may be that of a longer sequence:
 * a token's place in the mask does not depend on later tokens.
 * KVPOP_EINVAL: a missing pointer, sizes < 1, or an output over an input or another one.
 * KVPOP_EUNSUPPORTED: T or S > KVPOP_MAX_SEQ_LEN, alignment (4 bytes), or more than one
 * launch takes (2^32 - 1 threads, 1024 per list and 4096 positions). */
int kvpop_retain_prompt(const kvpop_retain* st, int32_t seq_len, const int32_t* evict, const float* scores,
                        const float* log_gamma, const int32_t* lens, void* stream);

/* The running top-k for single tokens: the token at position q = q_pos[b] arrives
 * (q < 0: nothing happens for sequence b, slot = -1). Its predecessor t = q - window leaves the
 * protected window and is eligible from now on, if t >= sinks (Sec. 3.1 eq.
 * eligible_set), with the priority that its score scores[b, h] = r_t gives it (a
 * delayed scorer knows it by now). If the list holds fewer than sinks + window + topk
 * tokens, the new one takes slot[b, h] = held, and held grows by one. Otherwise the
 * eligible token of least priority goes, of equals the latest (kvpop_running_topk's
 * order: NaN by its bits), and its slot is the new token's; slot = -1 if no token of the
 * list is eligible, or if window = 0 and the new token itself is the least. The new token's
 * prio is 0 until it leaves the window (its own if window = 0). A list so held is
 * what kvpop_running_topk's mask keeps at query q. S >= sinks + window + topk.
 * scores: fp32 [B, H]; q_pos: int32 [B]; slot: int32 [B, H] (output).
 * KVPOP_EINVAL: as above, sinks or window < 0, topk < 1, or S too small for them.
 * KVPOP_EUNSUPPORTED: as above (256 threads per list). */
int kvpop_retain_step(const kvpop_retain* st, const float* scores, const float* log_gamma, const int32_t* q_pos,
                      int32_t sinks, int32_t window, int32_t topk, int32_t* slot, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* KVPOP_CACHE_H */
