// Internal declarations of cache eviction: the attention mass of cached tokens (mass.hip), the choice
// of the tokens that stay (evict.hip) and their host side (evict_api.cpp).
#pragma once

#include "../../include/graphattn_cache.h"
#include "ga_internal.hpp"

namespace ga {

// Mass of every slot of a plan's chains: out[w] = decay in[w] + sum over the rows that see slot w and
// their q-heads of exp(scale q.k - lse).
struct MassArgs {
  const void* q;
  const void* pool;
  const float* lse;        // [R][Hq]
  const float* mass_in;    // [num_slots] or nullptr
  float* mass_out;         // [num_slots]
  const int32_t* desc;     // the schedule: work-item descriptors, items, B(s)
  const int64_t* counters;
  const int32_t* grp_br;
  int32_t desc_words, chunk_pages;
  int32_t Hq, Hkv, group, head_dim, dtype;
  bool causal;             // a multi-query plan
  float scale_log2, decay;
  int64_t units;           // upper bound on items
  int32_t pages;           // pages a workgroup takes (at most kMassPages)
};
constexpr int32_t kMassPages = 32;
hipError_t launch_mass(const MassArgs& a, hipStream_t stream);

// The schedule and sizes of a plan as the mass kernel needs them (api.cpp); rows: query rows.
// GA_EINVAL where two of its segments' pages coincide.  schedule: the plan is scheduled first where it
// has no schedule.
ga_status plan_mass_args(ga_plan* plan, bool schedule, hipStream_t stream, MassArgs* a,
                         int64_t* rows);

// One segment of an eviction: its first entry in the page list, its tokens, how many stay and where
// their output starts.
struct EvictSeg {
  int64_t pages, out;
  int32_t len, keep;
};
struct EvictArgs {
  const EvictSeg* segs;    // sorted by kernel: n_wave short ones, n_group medium ones, n_long long ones
  const int32_t* pages;
  const float* mass;
  int32_t* positions;      // may be nullptr
  int32_t* words;          // may be nullptr
  int32_t n_wave, n_group, n_long;
  int32_t first, recent;
};
// Tokens a wave, and a workgroup, holds in registers.
constexpr int32_t kEvictWave = 1024, kEvictGroup = 16384;
hipError_t launch_evict(const EvictArgs& a, hipStream_t stream);

}  // namespace ga
