/*
 * kvpop_mass.h -- C ABI of eviction by accumulated attention weight (gfx950 / MI355X): the
 * policy that keeps the keys which past queries looked at most, for models without a trained
 * scorer and as the baseline of one. It stands beside the retention of kvpop_cache.h, whose
 * lists, pages and conventions (streams, ownership, status codes, threads) hold here too.
 *
 * A key's mass is the attention probability that it got from every query so far, over the
 * query heads of its KV head. For a prompt that is what kvpop_future_attn_target with window 0
 * gives per query head; kvpop_mass_prompt chooses the tokens from it. While tokens come one at
 * a time, a decode step is
 *
 *   kvpop_mass_step      the slot of the token of least mass that is neither a sink nor new
 *   kvpop_cache_append   the new token into that slot (kvpop_cache.h)
 *   kvpop_cache_attn     the new queries over the lists, with their lse
 *   kvpop_cache_mass     their probabilities onto the masses
 */
#ifndef KVPOP_MASS_H
#define KVPOP_MASS_H

#include "kvpop_cache.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Adds to the mass of each slot j < held[b, h] of the lists what the newest queries give it:
 *   mass[b, h, j] = decay mass[b, h, j] + sum_{g, i} exp(scale <q_i, k_j> - lse[b, hG + g, i])
 * over the G = Hq / Hkv query heads of KV head h and the queries i < n = q_lens[b] that see the slot
 * (j < held[b, h] - (n - 1 - i)), as in kvpop_cache_attn, whose lse, q, held and q_lens these
 * are. held is taken into [0, max_pages * P]; slots at or past held[b, h] or n_slots keep their
 * mass. Slots whose entry of the page table holds no page get nothing and are decayed. A query
 * with lse = -inf gives nothing. With decay = 0 the old masses do not matter. Sums are fp32 in an
 * order that only sizes decide; queries are rounded as in kvpop_cache_attn, and their elements
 * have to be finite. The values' side of the cache is not read.
 * q: bf16 [B, Hq, N, D]; lse: fp32 [B, Hq, N]; mass: fp32 [B, Hkv, n_slots], updated.
 * KVPOP_EINVAL: a missing pointer, Hq % Hkv != 0, N < 1, n_slots < 1, scale not finite and > 0,
 * decay not in [0, 1], strides < 0, or mass over an input. KVPOP_EUNSUPPORTED: as
 * kvpop_cache_attn, n_slots > KVPOP_MAX_SEQ_LEN, or alignment (mass, lse: 4 bytes). */
int kvpop_cache_mass(const kvpop_cache* cache, int32_t n_q_heads, int32_t n_tokens, float scale, const kvpop_rows* q,
                     const int32_t* held, const int32_t* q_lens, const float* lse, float decay, int32_t n_slots,
                     float* mass, void* stream);

/* What a prompt leaves behind: for sequence b of n = lens[b] tokens (NULL: T; taken into
 * [0, T]) and KV head h, a token's mass is a_t = sum_g mass[b, hG + g, t], summed in 64 bits and
 * rounded to fp32. Kept are the tokens t < sinks, those with t >= n - window, and of the others the
 * topk of largest mass (of equals the earlier; NaN counts as more than any number), in
 * ascending order: st->pos and st->prio (their masses) of slots 0 .. held - 1; the other
 * slots get -1 and 0. All of st's arrays are outputs.
 * mass: fp32 [B, Hq, T], of kvpop_future_attn_target or kvpop_future_attn_bands with window 0.
 * workspace: kvpop_mass_prompt_workspace_size bytes of device memory, 16-byte aligned (may
 * be NULL if that is 0); its contents on entry do not matter. Calls that may run at the
 * same time, and graphs, need workspaces of their own.
 * KVPOP_EINVAL: a missing pointer, sizes < 1, Hq % H != 0, sinks or window < 0, topk < 1,
 * st->slots < sinks + window + topk, too small a workspace, or an output over an input or another
 * one. KVPOP_EUNSUPPORTED: T or slots > KVPOP_MAX_SEQ_LEN, alignment (4 bytes), or more than a
 * launch takes (2^32 - 1 threads, 1024 per list and per 1024 tokens of one). */
int kvpop_mass_prompt(const kvpop_retain* st, int32_t seq_len, int32_t n_q_heads, const float* mass,
                      const int32_t* lens, int32_t sinks, int32_t window, int32_t topk, void* workspace,
                      size_t workspace_bytes, void* stream);

/* Bytes of workspace for these sizes; 0 also for invalid ones. */
size_t kvpop_mass_prompt_workspace_size(int32_t batch, int32_t n_heads, int32_t n_q_heads, int32_t seq_len);

/* The slot for a new token: the one at position q = q_pos[b] arrives (q < 0: nothing happens
 * for sequence b, slot = -1). If the list holds fewer than sinks + window + topk tokens it takes
 * slot = held, and held grows by one. Otherwise, of the tokens at positions in
 * [sinks, q - window], the one of least mass goes, of equals the latest (NaN as
 * above), and its slot is the new token's; slot = -1 if there is none. The new token's mass is 0,
 * and it does not take part itself. st->prio holds the masses (that kvpop_cache_mass adds to).
 * q_pos: int32 [B]; slot: int32 [B, H] (output).
 * KVPOP_EINVAL: a missing pointer, sizes < 1, sinks or window < 0, topk < 1, st->slots too small
 * for them, or an output over an input or another one. KVPOP_EUNSUPPORTED: as above. */
int kvpop_mass_step(const kvpop_retain* st, const int32_t* q_pos, int32_t sinks, int32_t window, int32_t topk,
                    int32_t* slot, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* KVPOP_MASS_H */
