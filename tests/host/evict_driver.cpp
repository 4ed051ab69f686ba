// Host-only driver for the sanitizer build of the eviction's host code: random valid and malformed
// segment tables and keep counts go through graphattn_evict_create.  Without a GPU a valid call stops at
// its first device allocation, after the validation and the sorting of the segments have run.  The kernel
// launchers are stubs.
#include "graphattn_cache.h"

#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "evict_internal.hpp"

namespace ga {
ga_status host_fail(ga_status st, const char*) { return st; }
ga_status host_hip_fail(hipError_t, const char*) { return GA_EHIP; }
void host_clear_error() {}
hipError_t launch_mass(const MassArgs&, hipStream_t) { std::abort(); }
hipError_t launch_evict(const EvictArgs&, hipStream_t) { std::abort(); }
ga_status plan_mass_args(ga_plan*, bool, hipStream_t, MassArgs*, int64_t*) { std::abort(); }
}  // namespace ga

int main(int argc, char** argv) {
  const int trials = argc > 1 ? std::atoi(argv[1]) : 300;
  std::mt19937 rng(20);
  auto U = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); };
  int seen[8] = {0};
  for (int t = 0; t < trials; ++t) {
    const int S = U(0, 30);
    std::vector<int32_t> len(S), keep(S), pages;
    std::vector<int64_t> off(1, 0);
    const int first = U(0, 4), recent = U(0, 4);
    for (int s = 0; s < S; ++s) {
      len[s] = U(0, 9) ? U(1, 2000) : U(1, 40000);
      const int most = len[s], least = std::min(len[s], first + recent);
      keep[s] = U(least, most);
      off.push_back(off.back() + (len[s] + 15) / 16 + U(0, 2));
    }
    for (int64_t i = 0; i < off.back(); ++i) pages.push_back((int32_t)i);
    int64_t num_pages = off.back();
    const int bad = U(0, 9);
    if (S > 0) {
      const int s = U(0, S - 1);
      if (bad == 0) keep[s] = len[s] + 1;
      if (bad == 1) len[s] = 0;
      if (bad == 2) off[s + 1] = off[s] - 1;
      if (bad == 3) --num_pages;
      if (bad == 4) keep[s] = -1;
    }
    const ga_segment_table st{S, len.data(), off.data(), pages.data()};
    ga_evict* h = nullptr;
    const ga_status rc = graphattn_evict_create(&st, keep.data(), first, recent, num_pages, nullptr, &h);
    ++seen[-(int)rc];
    if (h) graphattn_evict_destroy(h);
  }
  std::printf("ok %d %d %d %d %d\n", seen[0], seen[1], seen[2], seen[3], seen[4]);
  return seen[1] > 0 && seen[3] + seen[4] > 0 ? 0 : 1;
}
