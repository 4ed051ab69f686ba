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
  const int32_t* seg_len;  // the plan's chains: tokens, page lists, causal origins, and their rows B(s)
  const int64_t* seg_page_off;
  const int32_t* seg_pages;
  const int32_t* seg_causal;
  const int64_t* grp_off;
  const int32_t* grp_br;
  int32_t Hq, Hkv, group, head_dim, dtype;
  bool causal;             // a multi-query plan
  float scale_log2, decay;
  int32_t chains;
  int32_t parts, parts_huge;   // the most parts a chain of up to, of more than kMassHuge rows may have (0: none)
  bool many;                   // some chain has more than kMassRows rows, and up to kMassHuge
  int32_t cost;            // what a workgroup takes: pages x pairs of row tiles
};
// Rows of a chain that are taken two tiles at a time.
constexpr int32_t kMassRows = 128;
// Rows from which on workgroups of more waves share them.
constexpr int32_t kMassHuge = 4096;
constexpr int32_t kMassCost = 128;     // most of it, and so most pages
// Parts a chain is taken in: of about `cost` pages x pairs of row tiles, and of kMassPages pages at least.
constexpr int32_t kMassPages = 4;
__host__ __device__ inline int32_t mass_parts(int64_t pages, int64_t rows, int32_t cost) {
  // (cost: a power of two, at most kMassCost)
  const int64_t pairs = (rows + 31) / 32 < cost ? (rows + 31) / 32 : cost;
  const int32_t parts = (int32_t)((pages * pairs + cost - 1) >> __builtin_ctz(cost));
  const int32_t most = (int32_t)((pages + kMassPages - 1) / kMassPages);
  return parts < most ? parts : most;
}
// Limits of a launch's grid: its first extent counts threads in 32 bits, the second one ends here.
constexpr int32_t kMassChains = (1 << 22) - 1, kMassParts = 65535;
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
