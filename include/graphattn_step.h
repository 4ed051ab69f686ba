/*
 * graphattn_step.h -- what a rollout step does between two attention calls: pages for the tokens that come
 * (graphattn_page_table), the slot, position and branch of each (graphattn_slot_map), their queries, keys and
 * values from the layer's projection into rows and pages (graphattn_qkv_append), and the rules that the next
 * token's logits follow, among them penalties for the tokens on the branch's path (graphattn_process_logits).
 *
 * Conventions, errors and streams as in graphattn.h, but that the graph is in DEVICE memory here, so that a
 * step needs no copy from the host: its index arrays cannot be validated on the host, and the kernels check
 * every index they read against the sizes in ga_device_graph instead.  Nothing is read or written outside the
 * arrays whatever they hold; what an index outside them means is said at each call.  All calls are
 * asynchronous on hip_stream, allocate nothing, keep nothing, use no atomics on global memory, give the same
 * bits for the same inputs, and may be captured into a graph (the arrays' contents are read at each replay).
 */
#ifndef GRAPHATTN_STEP_H
#define GRAPHATTN_STEP_H

#include "graphattn.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A rollout graph in device memory: ga_segment_table and ga_branch_paths (graphattn.h) with the same meaning
 * and the extents of their arrays.  A length below 0 counts as 0, a segment id outside [0, num_segments) as an
 * empty segment, a path whose offsets decrease or start outside path_segs as empty, and a page-table entry outside
 * its segment's or the table's, or a page id outside [0, num_pages), as no page. */
typedef struct {
  int32_t num_segments;
  int32_t num_branches;
  int64_t num_table_pages;          /* entries of seg_pages */
  int64_t num_path_segs;            /* entries of path_segs */
  int64_t num_pages;                /* extent of the page pool, at most 2^27 */
  const int32_t* seg_len;           /* [num_segments] */
  const int64_t* seg_page_offsets;  /* [num_segments + 1] */
  const int32_t* seg_pages;         /* [num_table_pages] */
  const int64_t* path_offsets;      /* [num_branches + 1] */
  const int32_t* path_segs;         /* [num_path_segs] */
} ga_device_graph;

/* The page table of a step: every segment keeps the pages it has and gets as many more, from the front of a
 * list of free ones, as its tokens and spare_tokens more need.  Segment s owns
 *   need(s) = max(old(s), ceil((seg_len[s] + spare_tokens) / 16)) pages,
 * old(s) = old_offsets[s + 1] - old_offsets[s] for s < num_old_segments (0 where that is negative), else 0:
 *   seg_page_offsets [num_segments + 1] device int64: the exclusive sums of need, the total last
 *   seg_pages        [capacity] device int32: s's old pages, then its new ones.  New pages are taken in the
 *                    order of the segments: (seg_page_offsets[s] - sum of old before s) of them before s's first.
 * Where free_pages ends, -1 is written (a page that no call reads or writes), so the table is usable whole once
 * the total less the old one is at most num_free.  Entries from the total on are left as they were, and those
 * from capacity on are not written.  old_offsets [num_old_segments + 1], old_pages [num_old_pages] and
 * free_pages [num_free]: device; num_old_segments in [0, num_segments], 0 for a table that starts (old_offsets
 * and old_pages may be NULL).  old_offsets holds what an earlier call wrote (or any CSR from 0 on); a value outside
 * [0, num_old_pages] is taken as the nearer end.  GA_EINVAL where an output overlaps
 * another array.
 * Every call, and every replay of a captured one, takes from the front of the list as it then is: before the
 * next one the caller drops the entries that were taken, total less sum of old of them, from free_pages, or the
 * same pages go to two segments.  An old page of -1 stays -1. */
ga_status graphattn_page_table(const int32_t* seg_len, int32_t num_segments, int32_t spare_tokens,
                               const int64_t* old_offsets, const int32_t* old_pages,
                               int32_t num_old_segments, int64_t num_old_pages,
                               const int32_t* free_pages, int64_t num_free,
                               int64_t* seg_page_offsets, int32_t* seg_pages, int64_t capacity,
                               void* hip_stream);

/* Where the new tokens of every branch go.  Branch b's new tokens are the last new_counts[b] ones of its path's
 * last segment, whose length in the graph already counts them (as for graphattn_extend: 1 for a decode step,
 * the segment's length for its prefill or its move to other pages; a branch of one segment names any segment).
 * With n_b = max(0, new_counts[b]) (device int32 [num_branches]; NULL: 1 each), row i = token_offsets[b] + j is
 * token t = len(last) - n_b + j of that segment:
 *   token_offsets [num_branches + 1] device int32: the exclusive sums of n_b, the total last (held at 2^31 - 1)
 *   slot_words    [capacity] device int32: page * 16 + slot, -1 where the table has no page for the token
 *   positions     [capacity] device int32: the token's position in the branch's context (the lengths of the
 *                 path's earlier segments, plus t)
 *   branches      [capacity] device int32: b
 * Rows from the total to capacity are padding, as are the tokens of a branch without a path, whose last segment
 * is outside the graph, with t < 0 or with a position of 2^31 or more: slot word, position and branch are -1.
 * Rows from capacity on are not written.  slot_words, positions and branches may each be NULL; GA_EINVAL where an
 * output overlaps another array.  Branches that
 * end in the same segment name the same slots (graphattn_kv_append wants them once). */
ga_status graphattn_slot_map(const ga_device_graph* graph, const int32_t* new_counts,
                             int32_t* token_offsets, int32_t* slot_words, int32_t* positions,
                             int32_t* branches, int32_t capacity, void* hip_stream);

/* How queries and keys are made from a projection's rows: per head, with x the D values of a head,
 *   y = x / sqrt(mean(x^2) + norm_eps) * weight       where there is a weight, else y = x
 * and then the first rotary_dim channels turn by the token's position p: the pair (a, b) of channels
 * (i, i + rotary_dim / 2), or (2i, 2i + 1) where interleaved, becomes
 *   (a cos - b sin, b cos + a sin) * rotary_scale,    angle p * inv_freq[i]
 * (p * inv_freq[i] and its remainder in float64, sine and cosine float32).  Values are float32 throughout and
 * are rounded once, at the end; a norm holds for all finite x, those too whose squares leave float32's range (a head of
 * zeros with a norm_eps of 0 is NaN). */
typedef struct {
  int32_t rotary_dim;      /* 0 .. D, even; a multiple of 16 unless interleaved (GA_EUNSUPPORTED otherwise) */
  int32_t interleaved;     /* 0 or 1 */
  float norm_eps;          /* finite, not negative */
  float rotary_scale;      /* finite; 0 selects 1 */
  const double* inv_freq;  /* [rotary_dim / 2] device, radians a position; NULL where rotary_dim is 0 */
  const float* q_weight;   /* [D] device, 16-byte aligned, or NULL: no norm */
  const float* k_weight;   /* [D] device, 16-byte aligned, or NULL: no norm */
} ga_qk_transform;

/* One layer's queries, keys and values of a step: q made as above goes to q_out, k made as above and v as it is
 * go to the pool (graphattn_kv_append of these rows: an MXFP4 pool rounds them, K from its bf16 row).
 *   q [n][Hq][D], k, v [n][Hkv][D]  device, the type of q in params (bf16 for an MXFP4 pool), 16-byte aligned;
 *                 token j's heads start q_stride (k_stride, v_stride) x j values in, a multiple of 16 bytes
 *   positions     [n] device int32; a token with a position below 0 is padding: nothing of it is written
 *   slot_words    [n] device int32; K and V of a token whose word is outside [0, num_pages x 16) are not stored
 *                 (its query is written: a token that is in the pool already)
 *   q_out         [n][Hq][D] device, 16-byte aligned; may be q itself where q_stride = Hq D
 * Slot words of tokens that are stored must be distinct.  Only params->num_q_heads, num_kv_heads, head_dim,
 * dtype and num_pages are used.  num_tokens 0: nothing is launched; more than 2^26 - 4: GA_EUNSUPPORTED. */
ga_status graphattn_qkv_append(void* kv_page_pool, const void* q, const void* k, const void* v,
                               int64_t q_stride, int64_t k_stride, int64_t v_stride,
                               const int32_t* positions, const int32_t* slot_words, int32_t num_tokens,
                               void* q_out, const ga_qk_transform* transform, const ga_params* params,
                               void* hip_stream);

/* What the logits of a step's rows are put through.  All arrays: device; NULL leaves a rule out. */
typedef struct {
  const float* repetition;     /* [rows] r: a token of the context has its logit z become z / r where z > 0, else z r */
  const float* frequency;      /* [rows] f: f times its count in the context, the prompt aside, is taken off */
  const float* presence;       /* [rows] taken off once where that count is not 0 */
  const float* temperature;    /* [rows] z / temperature (this and z / r: as z times the float32 reciprocal) */
  int32_t prompt_segments;     /* the first so many segments of every path are the prompt (>= 0) */
  const int64_t* bias_offsets; /* [rows + 1] CSR into bias_tokens and bias_values; entries outside [0, num_bias)
                                  are left out */
  const int32_t* bias_tokens;  /* [num_bias] ascending within a row (otherwise entries may be missed); a token that
                                  comes again has its values added up */
  const float* bias_values;    /* [num_bias] added to the logit */
  int64_t num_bias;
  const uint32_t* masks;       /* [num_masks][mask_words]: bit v % 32 of word v / 32 is set where token v may come */
  int32_t num_masks;
  int64_t mask_words;          /* >= ceil(vocab / 32) */
  const int32_t* row_mask;     /* [rows] which mask; outside [0, num_masks): none */
} ga_logit_rules;

/* Logits of a step's rows put through these rules, in this order for row r and token v, in float32:
 *   z = logits[r][v] + bias;  repetition;  z - f count - presence where count > 0;  z / temperature;
 *   -infinity where the row's mask forbids v (whatever z is, NaN too);  rounded to out's type.
 * The context of row r is the tokens of its branch's path up to and with its position (slot_map's positions and
 * branches; a row that checks a drafted token sees those before it): token t of a segment in slot w is
 * token_ids[w].  An id outside [0, vocab), and a token without a page, count for nothing.
 *   logits        [rows] of vocab values, logits_stride values apart (>= vocab); GA_F32 or GA_BF16 (dtype)
 *   out           the same with out_stride; of dtype, or float32 where out_f32; may be logits itself (same
 *                 type and stride)
 *   row_branches  [rows] device int32, or NULL: row r is branch r; rows outside [0, num_branches) are padding:
 *                 nothing is written
 *   row_positions [rows] device int32, or NULL: every row sees its whole path; a row with a position below 0 is
 *                 padding, one beyond the path sees all of it
 *   token_ids     [num_pages x 16] device int32, one per slot of the pool
 * Where neither repetition, frequency nor presence is given the context is not read, and graph and token_ids may
 * be NULL (row_branches and row_positions mark padding all the same).  A mask that forbids everything leaves a row
 * of -infinity.  GA_EUNSUPPORTED where rows x ceil(vocab / 38912) is 2^22 or more (with biases: vocab / 36864), and
 * for a vocab above 2^28.  Of a context the first 2^31 - 1 tokens
 * are seen; a token's count (below 2^30) is taken as a float32 value, exact up to 2^24. */
ga_status graphattn_process_logits(const void* logits, int64_t logits_stride, int32_t rows,
                                   int32_t vocab, int32_t dtype, const ga_logit_rules* rules,
                                   const ga_device_graph* graph, const int32_t* token_ids,
                                   const int32_t* row_branches, const int32_t* row_positions,
                                   void* out, int64_t out_stride, int32_t out_f32, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* GRAPHATTN_STEP_H */
