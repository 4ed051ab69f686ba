// Kernel arguments of the calls between two attention calls (include/graphattn_step.h), and how their
// kernels read a graph that lies in device memory: every index is checked where it is used.
#pragma once

#include "../../include/graphattn_step.h"
#include "ga_internal.hpp"

namespace ga {

struct PageTableArgs {
  const int32_t* seg_len;
  const int64_t* old_offsets;
  const int32_t* old_pages;
  const int32_t* free_pages;
  int64_t* offsets;
  int32_t* pages;
  int64_t n_old_pages, n_free, capacity;
  int32_t S, S_old, spare;
  int32_t tile;                  // segments of a workgroup (blockIdx.x), whose pages gridDim.y of them share
};

struct SlotMapArgs {
  ga_device_graph g;
  const int32_t* counts;
  int32_t* offsets;
  int32_t* words;
  int32_t* positions;
  int32_t* branches;
  int32_t capacity;
  int32_t tile;                  // branches of a workgroup, as above
};

struct QkvArgs {
  const unsigned char* src[3];   // q, k, v
  int64_t stride[3];             // bytes of a token
  const int32_t* positions;
  const int32_t* words;
  unsigned char* q_out;
  unsigned char* pool;
  const double* inv_freq;
  const float* weight[2];        // of q, of k; NULL: no norm
  int64_t num_slots;
  float eps, scale;
  int32_t n, Hq, Hkv, half;      // half: rotary_dim / 2
  int32_t q_units, q_groups;     // waves' shares of a token's queries, and groups of heads in each
  int32_t tokens;                // of a workgroup
};

struct LogitArgs {
  ga_device_graph g;
  ga_logit_rules rules;
  const unsigned char* in;
  unsigned char* out;
  int64_t in_stride, out_stride; // values
  const int32_t* token_ids;
  const int32_t* row_branches;
  const int32_t* row_positions;
  int32_t rows, vocab;
  int32_t slice, parts;          // tokens of a workgroup (a multiple of 32), workgroups of a row
  bool counted;                  // repetition, frequency or presence
};

// A launch has fewer threads along x.
constexpr int64_t kLaunchThreads = 1LL << 32;

hipError_t launch_page_table(const PageTableArgs& a, hipStream_t stream);
hipError_t launch_slot_map(const SlotMapArgs& a, hipStream_t stream);
hipError_t launch_qkv(const QkvArgs& a, int dim, int dtype, bool interleaved, hipStream_t stream);
// Slices of the rows, into a; the threads of the launch.
int64_t plan_logits(LogitArgs* a);
hipError_t launch_logits(const LogitArgs& a, bool in_f32, bool out_f32, hipStream_t stream);

namespace {

// A segment's pages in the table, and its tokens: empty for an id outside the graph.
struct SegRange {
  int64_t first, end;            // entries of seg_pages
  int32_t len;
};
__device__ __forceinline__ SegRange seg_range(const ga_device_graph& g, int32_t s) {
  if (s < 0 || s >= g.num_segments) return {0, 0, 0};
  const int32_t len = g.seg_len[s];
  const int64_t b = g.seg_page_offsets[s], e = g.seg_page_offsets[s + 1];
  const bool in = b >= 0 && b <= g.num_table_pages;
  return {in ? b : 0, in ? (e < g.num_table_pages ? e : g.num_table_pages) : 0, len > 0 ? len : 0};
}

// The page that holds token t of a segment, -1 where the table has none.
__device__ __forceinline__ int32_t page_of(const ga_device_graph& g, int64_t first, int64_t end, int32_t t) {
  const int64_t at = first + (t >> 4);
  if (at >= end) return -1;
  const int32_t page = g.seg_pages[at];
  return page >= 0 && (int64_t)page < g.num_pages ? page : -1;
}

// Branch b's entries of path_segs: both ends within the array.
struct PathRange {
  int64_t first, end;
};
__device__ __forceinline__ PathRange path_range(const ga_device_graph& g, int32_t b) {
  const int64_t first = g.path_offsets[b], e = g.path_offsets[b + 1];
  if (first < 0 || first > g.num_path_segs || e < first) return {0, 0};
  return {first, e < g.num_path_segs ? e : g.num_path_segs};
}

// Sums over a wave by row operations (a scan through lane exchanges waits for LDS twelve times, a microsecond):
// CTRL's lane, or nothing where a row or a mask leaves it out, is added.
template <int CTRL, int ROWS>
__device__ __forceinline__ void add_lane(int64_t* v) {
  const int lo = __builtin_amdgcn_update_dpp(0, (int)*v, CTRL, ROWS, 0xf, false);
  const int hi = __builtin_amdgcn_update_dpp(0, (int)(*v >> 32), CTRL, ROWS, 0xf, false);
  *v += (int64_t)(((uint64_t)(unsigned)hi << 32) | (unsigned)lo);
}
// The sum of the lanes up to and with this one.
__device__ __forceinline__ int64_t wave_scan(int64_t v) {
  add_lane<0x111, 0xf>(&v);                          // one lane up in rows of 16
  add_lane<0x112, 0xf>(&v);
  add_lane<0x114, 0xf>(&v);
  add_lane<0x118, 0xf>(&v);
  add_lane<0x142, 0xa>(&v);                          // the last lane of row 0 to row 1, of 2 to 3
  add_lane<0x143, 0xc>(&v);                          // lane 31 to rows 2 and 3
  return v;
}

}  // namespace

}  // namespace ga
