/*
 * graphattn_cache.h -- holding longer rollouts in the same pool: reading tokens back from a page pool
 * (MXFP4 pools hold 64/17 = 3.76 times the tokens of bf16 ones; ga_dtype in graphattn.h), the attention mass of
 * cached tokens, and the choice of the tokens that stay when a segment gives up the others.
 *
 * Conventions, errors and streams as in graphattn.h.
 */
#ifndef GRAPHATTN_CACHE_H
#define GRAPHATTN_CACHE_H

#include "graphattn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of one page (all kv-heads) of a pool with these parameters, or a negative ga_status. */
int64_t graphattn_kv_page_bytes(const ga_params* params);

/* K and V of cached tokens: slot slot_words[j] (device int32, page * 16 + slot) is written to row j of
 * k_out / v_out [num_tokens][Hkv][D] (device, 16-byte aligned, the type graphattn_kv_append takes: for
 * an MXFP4 pool the bf16 values that its codes stand for).  Rows of words outside [0, num_pages x 16) are
 * left as they were; a word may come twice.  Only params->num_kv_heads, head_dim, dtype and num_pages
 * are used.  Asynchronous on hip_stream; num_tokens 0: nothing is launched. */
ga_status graphattn_kv_read(const void* kv_page_pool, const int32_t* slot_words,
                            int32_t num_tokens, void* k_out, void* v_out,
                            const ga_params* params, void* hip_stream);

/* Eviction of cached tokens by the attention they received.  A rollout whose paths outgrow its pool
 * gives up the tokens that later tokens hardly attend to: every step adds the step's attention weights
 * to a mass per token slot (graphattn_run_mass); when room is needed, each segment's tokens that stay are
 * chosen by it (graphattn_evict_select), moved to fresh pages (graphattn_kv_copy with the chosen slot
 * words as sources) and the segment goes on with its new length and pages.  Keys are stored with their
 * positions applied, so the tokens that stay attend as before.
 * The mass belongs to the slot, and no call here moves or clears it: after the move mass[new word] =
 * mass[kept word] for every token that stayed, and a slot that takes a new token (graphattn_kv_append) is
 * set to 0, or that token goes on from what the slot's last one had gathered.
 *
 * graphattn_run_mass: for every slot w of the tokens of the plan's chains (segments on some path, at
 * their current lengths)
 *   mass_out[w] = decay mass_in[w] + sum over the query rows r that see w, and all q-heads h, of
 *                 exp(scale q[r][h] . k[w] - lse[r][h])
 * with q and kv_page_pool as graphattn_run was given them and the lse [R][Hq] that it wrote.
 *   mass_in   [num_pages x 16] device float32, or NULL (0); may be mass_out itself
 *   mass_out  [num_pages x 16] device float32; other slots are left as they were
 * One array may gather several layers (they share the slots): one call per layer, decay 1 but for the
 * first.  A row whose lse is infinite counts for nothing; a token with a score that is NaN, or +infinite in
 * such a row, has mass NaN.  Sums are float32, and the same bits for the
 * same inputs.  A plan without a current schedule is scheduled first.  GA_EINVAL where two segments on
 * paths own the same page (their slots would be written twice) and for a decay that is not finite,
 * GA_EUNSUPPORTED for a plan of 2^22 chains or with a chain of more than some four million tokens.
 * A plan's first call looks its page table over on the host (110,000 pages: 0.25 ms).
 * Decode and multi-query plans, all pool types; asynchronous on hip_stream, and calls on one plan do not
 * overlap with its other calls (graphattn_run). */
ga_status graphattn_run_mass(ga_plan* plan, const void* q, const void* kv_page_pool,
                             const float* lse, const float* mass_in, float decay, float* mass_out,
                             void* hip_stream);

/* Which tokens of every segment stay.  keep_counts [num_segments] host: segment s keeps
 * keep_counts[s] of its seg_len[s] tokens: its first first_tokens and last recent_tokens tokens, then
 * those with the largest mass, ties to the lower position.  (-0 counts as 0; a NaN mass counts above
 * every number.)  GA_EINVAL unless min(seg_len[s], first_tokens + recent_tokens) <= keep_counts[s] <=
 * seg_len[s]; GA_EUNSUPPORTED for a segment of more than 2^30 tokens.
 *
 * evict_create validates the table, copies it to the device and enqueues the upload on hip_stream (the
 * host arrays may be released on return; the handle serves any number of selections with these lengths
 * and counts); destroy waits for the device.  evict_select writes, for the segments one behind the
 * other and for each in ascending order,
 *   positions   [sum keep_counts] device int32, or NULL: the tokens' positions in their segment
 *   slot_words  [sum keep_counts] device int32, or NULL: their slot words (one of both is given)
 * from mass [num_pages x 16] (device float32).  Asynchronous on hip_stream; deterministic. */
typedef struct ga_evict ga_evict;
ga_status graphattn_evict_create(const ga_segment_table* segment_table,
                                 const int32_t* keep_counts, int32_t first_tokens,
                                 int32_t recent_tokens, int64_t num_pages, void* hip_stream,
                                 ga_evict** evict);
ga_status graphattn_evict_select(ga_evict* evict, const float* mass, int32_t* positions,
                                 int32_t* slot_words, void* hip_stream);
void graphattn_evict_destroy(ga_evict* evict);

#ifdef __cplusplus
}
#endif
#endif /* GRAPHATTN_CACHE_H */
