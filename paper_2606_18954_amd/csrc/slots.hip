// Pages and slots of a step's tokens, from lengths that are on the device: the page table of all segments, and
// the slot word, position and branch of every new token.
//
// Both spread the items of a list (pages of a segment, new tokens of a branch) behind one another: an exclusive
// sum of counts, and for every output the item it belongs to.  A rollout's lists are short (some hundred to some
// ten thousand items), so what costs is the number of launches and of dependent loads, and one launch does it all:
// every workgroup adds up the counts before its items by itself (they come from the L2 of its XCD), scans its own
// in LDS and writes its items' outputs.  No workgroup waits for another, and no memory is needed between them.
// Items per workgroup: as many as leave some 512 workgroups; with fewer items several workgroups share one item's
// outputs.
#include "step_internal.hpp"

namespace ga {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxTile = 1024;
constexpr int kAhead = 4;          // outputs of a thread whose loads are in flight together

struct Two {
  int64_t n, x;
};

// Exclusive sums over the workgroup's threads (in thread order), and the total.
__device__ __forceinline__ Two block_scan(Two v, Two* total) {
  __shared__ Two wave_sum[kThreads / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  Two s = v;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t n = __shfl_up(s.n, d), x = __shfl_up(s.x, d);
    if (lane >= d) {
      s.n += n;
      s.x += x;
    }
  }
  if (lane == 63) wave_sum[wave] = s;
  __syncthreads();
  Two before{0, 0}, all{0, 0};
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w == wave) before = all;
    all.n += wave_sum[w].n;
    all.x += wave_sum[w].x;
  }
  __syncthreads();
  *total = all;
  return {before.n + s.n - v.n, before.x + s.x - v.x};
}

// The last i with begin[i] <= j, of n items in ascending order (begin[0] = 0 <= j).
__device__ __forceinline__ int find(const int64_t* begin, int n, int64_t j) {
  int lo = 0;
  for (int step = n > 1 ? 1 << (31 - __builtin_clz(n - 1)) : 0; step > 0; step >>= 1)
    if (lo + step < n && begin[lo + step] <= j) lo += step;
  return lo;
}

__device__ __forceinline__ int64_t old_offset(const PageTableArgs& a, int64_t s) {
  const int64_t o = a.old_offsets[s];
  return o < 0 ? 0 : o < a.n_old_pages ? o : a.n_old_pages;
}

struct Need {
  int64_t pages, had;
};
__device__ __forceinline__ Need need_of(const PageTableArgs& a, int32_t s) {
  const int32_t len = a.seg_len[s];
  const int64_t want = ((int64_t)(len > 0 ? len : 0) + a.spare + kPageTokens - 1) / kPageTokens;
  int64_t had = 0;
  if (s < a.S_old) {
    had = old_offset(a, s + 1) - old_offset(a, s);
    had = had < 0 ? 0 : had;
  }
  return {want > had ? want : had, had};
}

__global__ __launch_bounds__(kThreads) void k_page_table(PageTableArgs a) {
  __shared__ int64_t begin[kMaxTile], old[kMaxTile], fresh[kMaxTile];
  __shared__ int32_t had[kMaxTile];
  const int tid = threadIdx.x;
  const int64_t t0 = (int64_t)blockIdx.x * a.tile;
  const int n = (int)(a.S - t0 < a.tile ? a.S - t0 : a.tile);
  // Pages, and new ones, of the segments before this workgroup's.
  Two sum{0, 0};
#pragma unroll 4
  for (int64_t s = tid; s < t0; s += kThreads) {
    const Need d = need_of(a, (int32_t)s);
    sum.n += d.pages;
    sum.x += d.pages - d.had;
  }
  Two before;
  block_scan(sum, &before);
  const int per = (a.tile + kThreads - 1) / kThreads;
  Two mine{0, 0}, total;
  for (int k = 0; k < per; ++k) {
    const int i = tid * per + k;
    if (i < n) {
      const Need d = need_of(a, (int32_t)(t0 + i));
      begin[i] = d.pages;
      had[i] = (int32_t)d.had;
      mine.n += d.pages;
      mine.x += d.pages - d.had;
    }
  }
  Two at = block_scan(mine, &total);
  for (int k = 0; k < per; ++k) {
    const int i = tid * per + k;
    if (i < n) {
      const int64_t pages = begin[i];
      begin[i] = at.n;
      old[i] = t0 + i < a.S_old ? old_offset(a, t0 + i) : 0;
      fresh[i] = before.x + at.x - had[i];           // ... of page had[i], its first new one
      if (blockIdx.y == 0) a.offsets[t0 + i] = before.n + at.n;
      at.n += pages;
      at.x += pages - had[i];
    }
  }
  if (blockIdx.y == 0 && blockIdx.x == gridDim.x - 1 && tid == 0) a.offsets[a.S] = before.n + total.n;
  __syncthreads();
  const int64_t room = a.capacity - before.n;        // (may be negative)
  const int64_t end = total.n < room ? total.n : room;
  const int64_t stride = (int64_t)gridDim.y * kThreads;
  for (int64_t j0 = (int64_t)blockIdx.y * kThreads + tid; j0 < end; j0 += kAhead * stride) {
    int32_t page[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int64_t j = j0 + k * stride;
      page[k] = -1;
      if (j < end) {
        const int i = find(begin, n, j);
        const int64_t p = j - begin[i];
        const bool is_old = p < had[i];
        const int64_t from = is_old ? old[i] + p : fresh[i] + p;
        if (from < (is_old ? a.n_old_pages : a.n_free)) page[k] = (is_old ? a.old_pages : a.free_pages)[from];
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (j0 + k * stride < end) a.pages[before.n + j0 + k * stride] = page[k];
  }
}

__device__ __forceinline__ int64_t count_of(const SlotMapArgs& a, int64_t b) {
  if (!a.counts) return 1;
  const int32_t c = a.counts[b];
  return c > 0 ? c : 0;
}

__global__ __launch_bounds__(kThreads) void k_slot_map(SlotMapArgs a) {
  __shared__ int64_t begin[kMaxTile], first[kMaxTile], last[kMaxTile], base[kMaxTile];
  __shared__ int32_t token[kMaxTile];                // of the item's first row; may be below 0
  const int tid = threadIdx.x;
  const int32_t B = a.g.num_branches;
  const int64_t t0 = (int64_t)blockIdx.x * a.tile;
  const int n = (int)(B - t0 < a.tile ? B - t0 : a.tile);
  const int per = (a.tile + kThreads - 1) / kThreads;
  // The items' own loads first: three that depend on each other, beside the sum of the counts before them.
  Two mine{0, 0}, total;
  for (int k = 0; k < per; ++k) {
    const int i = tid * per + k;
    if (i < n) {
      const int64_t c = count_of(a, t0 + i);
      begin[i] = c;
      mine.n += c;
      const PathRange p = path_range(a.g, (int32_t)(t0 + i));
      int64_t before = 0;
      int32_t s = -1;
      for (int64_t e = p.first; e < p.end; ++e) {
        if (s >= 0 && s < a.g.num_segments) before += max(a.g.seg_len[s], 0);
        s = a.g.path_segs[e];
      }
      const SegRange r = seg_range(a.g, s);
      const bool known = s >= 0 && s < a.g.num_segments;
      // (no segment: a token below 0 in every row)
      const int64_t t = known ? (int64_t)r.len - c : -(int64_t)0x7fffffff;
      token[i] = (int32_t)(t < -0x7fffffff ? -0x7fffffff : t);
      first[i] = r.first;
      last[i] = known ? r.end : r.first;
      base[i] = before;
    }
  }
  Two sum{0, 0}, before;
  if (a.counts) {
#pragma unroll 4
    for (int64_t b = tid; b < t0; b += kThreads) sum.n += count_of(a, b);
    block_scan(sum, &before);
  } else {
    before = {t0, 0};
  }
  Two at = block_scan(mine, &total);
  auto held = [](int64_t x) { return (int32_t)(x < 0x7fffffff ? x : 0x7fffffff); };
  for (int k = 0; k < per; ++k) {
    const int i = tid * per + k;
    if (i < n) {
      const int64_t c = begin[i];
      begin[i] = at.n;
      if (blockIdx.y == 0) a.offsets[t0 + i] = held(before.n + at.n);
      at.n += c;
    }
  }
  const bool closes = blockIdx.x == gridDim.x - 1;
  if (blockIdx.y == 0 && closes && tid == 0) a.offsets[B] = held(before.n + total.n);
  __syncthreads();
  const int64_t room = (int64_t)a.capacity - before.n;
  const int64_t rows = total.n < room ? total.n : room;
  // The last items' workgroups write the padding behind the rows too.
  const int64_t end = closes ? room : rows;
  const int64_t stride = (int64_t)gridDim.y * kThreads;
  for (int64_t j0 = (int64_t)blockIdx.y * kThreads + tid; j0 < end; j0 += kAhead * stride) {
    int32_t word[kAhead], pos[kAhead], branch[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int64_t j = j0 + k * stride;
      word[k] = pos[k] = branch[k] = -1;
      if (j < rows) {
        const int i = find(begin, n, j);
        const int64_t t = token[i] + (j - begin[i]), p = base[i] + t;
        if (t >= 0 && p < 0x80000000LL) {
          pos[k] = (int32_t)p;
          branch[k] = (int32_t)t0 + i;
          const int32_t page = a.words ? page_of(a.g, first[i], last[i], (int32_t)t) : -1;
          word[k] = page < 0 ? -1 : page * kPageTokens + (int32_t)(t & (kPageTokens - 1));
        }
      }
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int64_t j = j0 + k * stride;
      if (j >= end) continue;
      if (a.words) a.words[before.n + j] = word[k];
      if (a.positions) a.positions[before.n + j] = pos[k];
      if (a.branches) a.branches[before.n + j] = branch[k];
    }
  }
}

// Items of a workgroup, and workgroups of the same items.
dim3 tiles_of(int64_t items, int32_t* tile) {
  const int64_t t = (items + 511) / 512;
  *tile = (int32_t)(t < 1 ? 1 : t > kMaxTile ? kMaxTile : t);
  const int64_t tiles = items > 0 ? (items + *tile - 1) / *tile : 1;
  return dim3((unsigned)tiles, (unsigned)(tiles < 512 ? 512 / tiles : 1));
}

}  // namespace

hipError_t launch_page_table(const PageTableArgs& args, hipStream_t stream) {
  PageTableArgs a = args;
  const dim3 grid = tiles_of(a.S, &a.tile);
  hipLaunchKernelGGL(k_page_table, grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_slot_map(const SlotMapArgs& args, hipStream_t stream) {
  SlotMapArgs a = args;
  const dim3 grid = tiles_of(a.g.num_branches, &a.tile);
  hipLaunchKernelGGL(k_slot_map, grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ga
