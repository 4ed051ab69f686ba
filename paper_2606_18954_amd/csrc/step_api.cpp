// Host side of the calls between two attention calls (include/graphattn_step.h): argument checks and launches.
#include "step_internal.hpp"

#include <cmath>
#include <cstdarg>
#include <cstdio>

namespace ga {
ga_status host_fail(ga_status st, const char* msg);
ga_status host_hip_fail(hipError_t e, const char* what);
void host_clear_error();
ga_status host_check_params(const ga_params* params);
}  // namespace ga

namespace {

ga_status vfail(ga_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
ga_status vfail(ga_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return ga::host_fail(st, buf);
}

bool misaligned(size_t to, std::initializer_list<const void*> ptrs) {
  uintptr_t all = 0;
  for (const void* p : ptrs) all |= reinterpret_cast<uintptr_t>(p);
  return all & (to - 1);
}

// Whether two arrays share bytes.
struct Range {
  const void* p;
  int64_t bytes;
};
bool overlap(Range a, Range b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return a.p && b.p && a.bytes > 0 && b.bytes > 0 && x < y + (uintptr_t)b.bytes && y < x + (uintptr_t)a.bytes;
}
bool overlap(std::initializer_list<Range> outs, std::initializer_list<Range> ins) {
  for (const Range& a : outs)
    for (const Range& b : ins)
      if (overlap(a, b)) return true;
  return false;
}

ga_status check_graph(const ga_device_graph* g) {
  if (!g) return vfail(GA_EINVAL, "graph is NULL");
  if (g->num_segments < 0 || g->num_branches < 0 || g->num_table_pages < 0 || g->num_path_segs < 0 ||
      g->num_pages < 0)
    return vfail(GA_EINVAL, "a size of the graph is negative");
  if (g->num_pages > (1LL << ga::kPageValidShift))
    return vfail(GA_EUNSUPPORTED, "num_pages %lld exceeds 2^%d", (long long)g->num_pages, ga::kPageValidShift);
  if ((g->num_segments > 0 && (!g->seg_len || !g->seg_page_offsets)) || (g->num_table_pages > 0 && !g->seg_pages) ||
      (g->num_branches > 0 && !g->path_offsets) || (g->num_path_segs > 0 && !g->path_segs))
    return vfail(GA_EINVAL, "an array of the graph is NULL");
  if (misaligned(4, {g->seg_len, g->seg_pages, g->path_segs}) || misaligned(8, {g->seg_page_offsets, g->path_offsets}))
    return vfail(GA_EINVAL, "the graph's arrays must be aligned to their elements");
  return GA_OK;
}

}  // namespace

extern "C" {

ga_status graphattn_page_table(const int32_t* seg_len, int32_t num_segments, int32_t spare_tokens,
                               const int64_t* old_offsets, const int32_t* old_pages, int32_t num_old_segments,
                               int64_t num_old_pages, const int32_t* free_pages, int64_t num_free,
                               int64_t* seg_page_offsets, int32_t* seg_pages, int64_t capacity, void* hip_stream) {
  ga::host_clear_error();
  if (num_segments < 0 || spare_tokens < 0 || num_old_pages < 0 || num_free < 0 || capacity < 0)
    return vfail(GA_EINVAL, "a size is negative");
  if (num_old_segments < 0 || num_old_segments > num_segments)
    return vfail(GA_EINVAL, "num_old_segments (%d) outside [0, %d]", num_old_segments, num_segments);
  if (num_old_pages > 0x7fffffff) return vfail(GA_EUNSUPPORTED, "%lld old pages (>= 2^31)", (long long)num_old_pages);
  if (!seg_page_offsets || (num_segments > 0 && !seg_len) || (num_old_segments > 0 && !old_offsets) ||
      (num_old_pages > 0 && !old_pages) || (num_free > 0 && !free_pages) || (capacity > 0 && !seg_pages))
    return vfail(GA_EINVAL, "device pointers must be non-NULL");
  if (misaligned(4, {seg_len, old_pages, free_pages, seg_pages}) || misaligned(8, {old_offsets, seg_page_offsets}))
    return vfail(GA_EINVAL, "arrays must be aligned to their elements");
  const Range offsets{seg_page_offsets, 8 * ((int64_t)num_segments + 1)}, pages{seg_pages, 4 * capacity};
  if (overlap({offsets, pages}, {{seg_len, 4 * (int64_t)num_segments},
                                 {old_offsets, num_old_segments ? 8 * ((int64_t)num_old_segments + 1) : 0},
                                 {old_pages, 4 * num_old_pages},
                                 {free_pages, 4 * num_free}}) ||
      overlap(offsets, pages))
    return vfail(GA_EINVAL, "the new table overlaps another array");
  ga::PageTableArgs a{};
  a.seg_len = seg_len;
  a.old_offsets = old_offsets;
  a.old_pages = old_pages;
  a.free_pages = free_pages;
  a.offsets = seg_page_offsets;
  a.pages = seg_pages;
  a.n_old_pages = num_old_pages;
  a.n_free = num_free;
  a.capacity = capacity;
  a.S = num_segments;
  a.S_old = num_old_segments;
  a.spare = spare_tokens;
  const hipError_t e = ga::launch_page_table(a, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? GA_OK : ga::host_hip_fail(e, "page table launch");
}

ga_status graphattn_slot_map(const ga_device_graph* graph, const int32_t* new_counts, int32_t* token_offsets,
                             int32_t* slot_words, int32_t* positions, int32_t* branches, int32_t capacity,
                             void* hip_stream) {
  ga::host_clear_error();
  const ga_status rc = check_graph(graph);
  if (rc) return rc;
  if (capacity < 0) return vfail(GA_EINVAL, "capacity is negative");
  if (!token_offsets) return vfail(GA_EINVAL, "token_offsets is NULL");
  if (misaligned(4, {new_counts, token_offsets, slot_words, positions, branches}))
    return vfail(GA_EINVAL, "new_counts and the outputs must be 4-byte aligned");
  const int64_t B = graph->num_branches, rows = 4 * (int64_t)capacity;
  const Range offsets{token_offsets, 4 * (B + 1)}, words{slot_words, rows}, pos{positions, rows}, br{branches, rows};
  if (overlap({offsets, words, pos, br}, {{new_counts, 4 * B},
                                          {graph->seg_len, 4 * (int64_t)graph->num_segments},
                                          {graph->seg_page_offsets, 8 * ((int64_t)graph->num_segments + 1)},
                                          {graph->seg_pages, 4 * graph->num_table_pages},
                                          {graph->path_offsets, 8 * (B + 1)},
                                          {graph->path_segs, 4 * graph->num_path_segs}}) ||
      overlap({offsets}, {words, pos, br}) || overlap({words}, {pos, br}) || overlap(pos, br))
    return vfail(GA_EINVAL, "an output overlaps another array");
  ga::SlotMapArgs a{};
  a.g = *graph;
  a.counts = new_counts;
  a.offsets = token_offsets;
  a.words = slot_words;
  a.positions = positions;
  a.branches = branches;
  a.capacity = slot_words || positions || branches ? capacity : 0;
  const hipError_t e = ga::launch_slot_map(a, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? GA_OK : ga::host_hip_fail(e, "slot map launch");
}

ga_status graphattn_qkv_append(void* kv_page_pool, const void* q, const void* k, const void* v, int64_t q_stride,
                               int64_t k_stride, int64_t v_stride, const int32_t* positions,
                               const int32_t* slot_words, int32_t num_tokens, void* q_out,
                               const ga_qk_transform* transform, const ga_params* params, void* hip_stream) {
  ga::host_clear_error();
  const ga_status rc = ga::host_check_params(params);
  if (rc) return rc;
  const int D = params->head_dim;
  if (!transform) return vfail(GA_EINVAL, "transform is NULL");
  const int R = transform->rotary_dim;
  if (R < 0 || R > D || R % 2) return vfail(GA_EINVAL, "rotary_dim %d is odd or outside [0, %d]", R, D);
  if (transform->interleaved != 0 && transform->interleaved != 1)
    return vfail(GA_EINVAL, "interleaved must be 0 or 1");
  if (!transform->interleaved && R % 16)
    return vfail(GA_EUNSUPPORTED, "rotary_dim %d is not a multiple of 16 (pairs half of it apart)", R);
  if (!std::isfinite(transform->norm_eps) || transform->norm_eps < 0.f)
    return vfail(GA_EINVAL, "norm_eps must be finite and >= 0");
  if (!std::isfinite(transform->rotary_scale)) return vfail(GA_EINVAL, "rotary_scale must be finite");
  if (R > 0 && !transform->inv_freq) return vfail(GA_EINVAL, "inv_freq is NULL");
  if (misaligned(8, {transform->inv_freq}) || misaligned(16, {transform->q_weight, transform->k_weight}))
    return vfail(GA_EINVAL, "inv_freq must be 8-byte aligned, the weights 16-byte aligned");
  if (num_tokens < 0) return vfail(GA_EINVAL, "num_tokens is negative");
  // (256 threads for four tokens)
  if ((num_tokens + 3LL) / 4 * 256 >= ga::kLaunchThreads)
    return vfail(GA_EUNSUPPORTED, "%d tokens (> 2^26 - 4)", num_tokens);
  if (params->num_q_heads > (1 << 14)) return vfail(GA_EUNSUPPORTED, "%d heads (> 2^14)", params->num_q_heads);
  if (num_tokens == 0) return GA_OK;
  if (!kv_page_pool || !q || !k || !v || !positions || !slot_words || !q_out)
    return vfail(GA_EINVAL, "device pointers must be non-NULL");
  if (misaligned(16, {kv_page_pool, q, k, v, q_out}))
    return vfail(GA_EINVAL, "kv_page_pool and the q, K and V rows must be 16-byte aligned");
  if (misaligned(4, {positions, slot_words}))
    return vfail(GA_EINVAL, "positions and slot_words must be 4-byte aligned");
  const int elt = params->dtype == GA_F32 ? 4 : 2;
  const int64_t stride[3] = {q_stride, k_stride, v_stride};
  for (const int64_t s : stride)
    if (s < 0 || s * elt % 16) return vfail(GA_EINVAL, "strides must be >= 0 and multiples of 16 bytes");
  const int64_t n = num_tokens, q_row = (int64_t)params->num_q_heads * D, kv_row = (int64_t)params->num_kv_heads * D;
  const Range out{q_out, n * q_row * elt};
  const bool in_place = q_out == q && (q_stride == q_row || n == 1);
  if (overlap({out}, {{q, in_place ? 0 : ((n - 1) * q_stride + q_row) * elt},
                      {k, ((n - 1) * k_stride + kv_row) * elt},
                      {v, ((n - 1) * v_stride + kv_row) * elt}}))
    return vfail(GA_EINVAL,
                 "q_out overlaps the rows that are read; it may be q itself where q's rows lie one behind the other");
  ga::QkvArgs a{};
  a.src[0] = static_cast<const unsigned char*>(q);
  a.src[1] = static_cast<const unsigned char*>(k);
  a.src[2] = static_cast<const unsigned char*>(v);
  for (int i = 0; i < 3; ++i) a.stride[i] = stride[i] * elt;
  a.positions = positions;
  a.words = slot_words;
  a.q_out = static_cast<unsigned char*>(q_out);
  a.pool = static_cast<unsigned char*>(kv_page_pool);
  a.inv_freq = transform->inv_freq;
  a.weight[0] = transform->q_weight;
  a.weight[1] = transform->k_weight;
  a.num_slots = params->num_pages * ga::kPageTokens;
  a.eps = transform->norm_eps;
  a.scale = transform->rotary_scale == 0.f ? 1.f : transform->rotary_scale;
  a.n = num_tokens;
  a.Hq = params->num_q_heads;
  a.Hkv = params->num_kv_heads;
  a.half = R / 2;
  const hipError_t e =
      ga::launch_qkv(a, D, params->dtype, transform->interleaved != 0, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? GA_OK : ga::host_hip_fail(e, "qkv append launch");
}

ga_status graphattn_process_logits(const void* logits, int64_t logits_stride, int32_t rows, int32_t vocab,
                                   int32_t dtype, const ga_logit_rules* rules, const ga_device_graph* graph,
                                   const int32_t* token_ids, const int32_t* row_branches,
                                   const int32_t* row_positions, void* out, int64_t out_stride, int32_t out_f32,
                                   void* hip_stream) {
  ga::host_clear_error();
  if (!rules) return vfail(GA_EINVAL, "rules is NULL");
  if (dtype != GA_F32 && dtype != GA_BF16) return vfail(GA_EUNSUPPORTED, "logits of dtype %d", dtype);
  if (out_f32 != 0 && out_f32 != 1) return vfail(GA_EINVAL, "out_f32 must be 0 or 1");
  if (rows < 0) return vfail(GA_EINVAL, "rows is negative");
  if (vocab < 1) return vfail(GA_EINVAL, "vocab %d (< 1)", vocab);
  if (vocab > (1 << 28)) return vfail(GA_EUNSUPPORTED, "vocab %d (> 2^28)", vocab);
  if (logits_stride < vocab || out_stride < vocab) return vfail(GA_EINVAL, "a row stride is below vocab (%d)", vocab);
  if (rules->prompt_segments < 0 || rules->num_bias < 0 || rules->num_masks < 0)
    return vfail(GA_EINVAL, "a size of the rules is negative");
  const bool counted = rules->repetition || rules->frequency || rules->presence;
  ga_device_graph g{};
  g.num_branches = 0x7fffffff;
  if (graph || counted) {
    const ga_status rc = check_graph(graph);
    if (rc) return rc;
    g = *graph;
  }
  if (rows == 0) return GA_OK;
  if (counted && g.num_pages > 0 && !token_ids) return vfail(GA_EINVAL, "token_ids is NULL");
  if (rules->num_bias > 0 && (!rules->bias_offsets || !rules->bias_tokens || !rules->bias_values))
    return vfail(GA_EINVAL, "biases are offsets, tokens and values together");
  const bool masked = rules->num_masks > 0;
  if (masked && (!rules->masks || !rules->row_mask)) return vfail(GA_EINVAL, "masks or row_mask is NULL");
  if (masked && rules->mask_words < (vocab + 31) / 32)
    return vfail(GA_EINVAL, "mask_words %lld below %d", (long long)rules->mask_words, (vocab + 31) / 32);
  if (misaligned(4, {rules->repetition, rules->frequency, rules->presence, rules->temperature, rules->bias_tokens,
                     rules->bias_values, rules->masks, rules->row_mask, token_ids, row_branches, row_positions}) ||
      misaligned(8, {rules->bias_offsets}))
    return vfail(GA_EINVAL, "the rules' and rows' arrays must be aligned to their elements");
  if (!logits || !out) return vfail(GA_EINVAL, "logits and out must be non-NULL");
  const bool in_f32 = dtype == GA_F32, wide = in_f32 || out_f32;
  if (misaligned(in_f32 ? 4 : 2, {logits}) || misaligned(wide ? 4 : 2, {out}))
    return vfail(GA_EINVAL, "logits and out must be aligned to their elements");
  const int in_elt = in_f32 ? 4 : 2, out_elt = wide ? 4 : 2;
  const bool in_place = out == logits && in_elt == out_elt && (out_stride == logits_stride || rows == 1);
  if (!in_place && overlap({out, ((rows - 1LL) * out_stride + vocab) * out_elt},
                           {logits, ((rows - 1LL) * logits_stride + vocab) * in_elt}))
    return vfail(GA_EINVAL, "out overlaps logits; it may be logits itself with its type and stride");
  ga::LogitArgs a{};
  a.g = g;
  a.rules = *rules;
  if (!masked) a.rules.masks = nullptr;
  if (rules->num_bias == 0) a.rules.bias_offsets = nullptr;
  a.in = static_cast<const unsigned char*>(logits);
  a.out = static_cast<unsigned char*>(out);
  a.in_stride = logits_stride;
  a.out_stride = out_stride;
  a.token_ids = token_ids;
  a.row_branches = row_branches;
  a.row_positions = row_positions;
  a.rows = rows;
  a.vocab = vocab;
  a.counted = counted;
  if (ga::plan_logits(&a) >= ga::kLaunchThreads)
    return vfail(GA_EUNSUPPORTED, "%d rows of %d: %d parts a row are 2^22 or more in all", rows, vocab, a.parts);
  const hipError_t e = ga::launch_logits(a, in_f32, wide, static_cast<hipStream_t>(hip_stream));
  return e == hipSuccess ? GA_OK : ga::host_hip_fail(e, "logits launch");
}

}  // extern "C"
