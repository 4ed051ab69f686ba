// Host side of cache eviction: validation, the handle, launches and the C entry points of the
// attention mass and the choice of the tokens that stay.
#include "evict_internal.hpp"

#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <new>
#include <vector>

namespace ga {
ga_status host_fail(ga_status st, const char* msg);
ga_status host_hip_fail(hipError_t e, const char* what);
void host_clear_error();
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

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace

// A validated eviction on the device: its segments, sorted by the kernel that takes them, and their
// page lists.
struct ga_evict {
  void* dev = nullptr;
  void* pin = nullptr;
  ga::EvictArgs a{};
};

namespace {

void evict_free(ga_evict* h) {
  if (!h) return;
  if (h->dev) {
    (void)hipDeviceSynchronize();
    (void)hipFree(h->dev);
  }
  if (h->pin) (void)hipHostFree(h->pin);
  delete h;
}

ga_status evict_create(const ga_segment_table* st, const int32_t* keep, int32_t first,
                       int32_t recent, int64_t num_pages, hipStream_t stream, ga_evict** out) {
  if (!st) return vfail(GA_EINVAL, "segment_table is NULL");
  const int32_t S = st->num_segments;
  if (S < 0) return vfail(GA_EINVAL, "num_segments is negative");
  if (!st->seg_page_offsets) return vfail(GA_EINVAL, "seg_page_offsets is NULL");
  if (S > 0 && (!st->seg_len || !keep)) return vfail(GA_EINVAL, "seg_len or keep is NULL");
  if (first < 0 || recent < 0)
    return vfail(GA_EINVAL, "first (%d) and recent (%d) must not be negative", first, recent);
  if (num_pages < 0) return vfail(GA_EINVAL, "num_pages is negative");
  if (num_pages > (1LL << ga::kPageValidShift))
    return vfail(GA_EUNSUPPORTED, "num_pages %lld exceeds 2^%d", (long long)num_pages,
                 ga::kPageValidShift);
  if (st->seg_page_offsets[0] != 0) return vfail(GA_EINVAL, "seg_page_offsets[0] must be 0");
  // Every segment's pages in use, one list behind the other, and the segments by kernel.
  std::vector<int32_t> pages;
  std::vector<ga::EvictSeg> seg[3];
  int64_t total = 0;
  for (int32_t s = 0; s < S; ++s) {
    const int32_t len = st->seg_len[s];
    if (len < 1) return vfail(GA_EINVAL, "segment %d has length %d (< 1)", s, len);
    // (positions run past a segment's end by less than a group of tokens)
    if (len > (1 << 30))
      return vfail(GA_EUNSUPPORTED, "segment %d has %d tokens (> 2^30)", s, len);
    const int64_t b = st->seg_page_offsets[s], e = st->seg_page_offsets[s + 1];
    if (e < b) return vfail(GA_EINVAL, "seg_page_offsets decreases at segment %d", s);
    const int64_t need = ((int64_t)len + ga::kPageTokens - 1) / ga::kPageTokens;
    if (e - b < need)
      return vfail(GA_EINVAL, "segment %d has %d tokens but only %lld pages", s, len,
                   (long long)(e - b));
    if (!st->seg_pages) return vfail(GA_EINVAL, "seg_pages is NULL");
    const int64_t safe = (int64_t)first + recent < len ? (int64_t)first + recent : len;
    if (keep[s] < safe || keep[s] > len)
      return vfail(GA_EINVAL, "segment %d keeps %d tokens, outside [%lld, %d]", s, keep[s],
                   (long long)safe, len);
    const ga::EvictSeg x{(int64_t)pages.size(), total, len, keep[s]};
    seg[len <= ga::kEvictWave ? 0 : len <= ga::kEvictGroup ? 1 : 2].push_back(x);
    total += keep[s];
    for (int64_t i = 0; i < need; ++i) {
      const int32_t pg = st->seg_pages[b + i];
      if (pg < 0 || pg >= num_pages)
        return vfail(GA_ERANGE, "seg_pages[%lld] = %d outside [0, %lld)", (long long)(b + i), pg,
                     (long long)num_pages);
      pages.push_back(pg);
    }
  }
  ga_evict* h = new ga_evict();
  const size_t seg_bytes = align256(sizeof(ga::EvictSeg) * (size_t)S);
  const size_t bytes = seg_bytes + align256(sizeof(int32_t) * pages.size());
  if (bytes > 0) {
    if (hipMalloc(&h->dev, bytes) != hipSuccess) {
      (void)hipGetLastError();
      h->dev = nullptr;
      evict_free(h);
      return vfail(GA_ENOMEM, "device copy of %zu bytes", bytes);
    }
    if (hipHostMalloc(&h->pin, bytes) != hipSuccess) {
      (void)hipGetLastError();
      h->pin = nullptr;
      evict_free(h);
      return vfail(GA_ENOMEM, "pinned staging of %zu bytes", bytes);
    }
    char* p = static_cast<char*>(h->pin);
    for (const auto& v : seg) {
      if (!v.empty()) std::memcpy(p, v.data(), sizeof(ga::EvictSeg) * v.size());
      p += sizeof(ga::EvictSeg) * v.size();
    }
    if (!pages.empty())
      std::memcpy(static_cast<char*>(h->pin) + seg_bytes, pages.data(),
                  sizeof(int32_t) * pages.size());
    const hipError_t e = hipMemcpyAsync(h->dev, h->pin, bytes, hipMemcpyHostToDevice, stream);
    if (e != hipSuccess) {
      evict_free(h);
      return ga::host_hip_fail(e, "eviction upload");
    }
  }
  h->a.segs = static_cast<const ga::EvictSeg*>(h->dev);
  h->a.pages = reinterpret_cast<const int32_t*>(static_cast<char*>(h->dev) + seg_bytes);
  h->a.n_wave = (int32_t)seg[0].size();
  h->a.n_group = (int32_t)seg[1].size();
  h->a.n_long = (int32_t)seg[2].size();
  h->a.first = first;
  h->a.recent = recent;
  *out = h;
  return GA_OK;
}

}  // namespace

extern "C" {

ga_status graphattn_run_mass(ga_plan* plan, const void* q, const void* kv_page_pool,
                             const float* lse, const float* mass_in, float decay, float* mass_out,
                             void* hip_stream) {
  ga::host_clear_error();
  if (!plan) return vfail(GA_EINVAL, "plan is NULL");
  if (!std::isfinite(decay)) return vfail(GA_EINVAL, "decay must be finite");
  const hipStream_t stream = static_cast<hipStream_t>(hip_stream);
  try {
    ga::MassArgs a{};
    int64_t rows = 0;
    // (the arguments first: a refused call leaves the plan as it was)
    ga_status rc = ga::plan_mass_args(plan, false, stream, &a, &rows);
    if (rc) return rc;
    if (rows == 0) return GA_OK;
    if (!q || !kv_page_pool || !lse || !mass_out)
      return vfail(GA_EINVAL, "q, kv_page_pool, lse and mass_out must be non-NULL");
    if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(kv_page_pool)) & 15)
      return vfail(GA_EINVAL, "q and kv_page_pool must be 16-byte aligned");
    if ((reinterpret_cast<uintptr_t>(lse) | reinterpret_cast<uintptr_t>(mass_in) |
         reinterpret_cast<uintptr_t>(mass_out)) & 3)
      return vfail(GA_EINVAL, "lse and the mass arrays must be 4-byte aligned");
    rc = ga::plan_mass_args(plan, true, stream, &a, &rows);
    if (rc) return rc;
    a.q = q;
    a.pool = kv_page_pool;
    a.lse = lse;
    a.mass_in = mass_in;
    a.mass_out = mass_out;
    a.decay = decay;
    const hipError_t e = ga::launch_mass(a, stream);
    if (e != hipSuccess) return ga::host_hip_fail(e, "mass launch");
    return GA_OK;
  } catch (const std::bad_alloc&) {
    return vfail(GA_ENOMEM, "host memory");
  }
}

ga_status graphattn_evict_create(const ga_segment_table* segment_table,
                                 const int32_t* keep_counts, int32_t first_tokens,
                                 int32_t recent_tokens, int64_t num_pages, void* hip_stream,
                                 ga_evict** evict) {
  ga::host_clear_error();
  if (!evict) return vfail(GA_EINVAL, "evict out-pointer is NULL");
  *evict = nullptr;
  try {
    return evict_create(segment_table, keep_counts, first_tokens, recent_tokens, num_pages,
                        static_cast<hipStream_t>(hip_stream), evict);
  } catch (const std::bad_alloc&) {
    return vfail(GA_ENOMEM, "host memory");
  }
}

ga_status graphattn_evict_select(ga_evict* evict, const float* mass, int32_t* positions,
                                 int32_t* slot_words, void* hip_stream) {
  ga::host_clear_error();
  if (!evict) return vfail(GA_EINVAL, "evict is NULL");
  ga::EvictArgs a = evict->a;
  if (a.n_wave + a.n_group + a.n_long == 0) return GA_OK;
  if (!mass || (!positions && !slot_words))
    return vfail(GA_EINVAL, "mass and one of positions and slot_words must be non-NULL");
  if ((reinterpret_cast<uintptr_t>(mass) | reinterpret_cast<uintptr_t>(positions) |
       reinterpret_cast<uintptr_t>(slot_words)) & 3)
    return vfail(GA_EINVAL, "mass, positions and slot_words must be 4-byte aligned");
  a.mass = mass;
  a.positions = positions;
  a.words = slot_words;
  const hipError_t e = ga::launch_evict(a, static_cast<hipStream_t>(hip_stream));
  if (e != hipSuccess) return ga::host_hip_fail(e, "eviction launch");
  return GA_OK;
}

void graphattn_evict_destroy(ga_evict* evict) { evict_free(evict); }

}  // extern "C"
