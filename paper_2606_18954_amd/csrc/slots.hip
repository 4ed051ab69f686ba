// Pages and slots of a step's tokens, from lengths that are on the device: the page table of all segments, and
// the slot word, position and branch of every new token.
//
// Both spread the items of a list (pages of a segment, new tokens of a branch) behind one another: an exclusive
// sum of counts, and for every output the item it belongs to.  A rollout's lists are short (some hundred to some
// ten thousand items), so what costs is the number of launches and of dependent loads, and one launch does it all:
// every workgroup adds up the counts before its items by itself (they come from the L2 of its XCD), scans its own
// in LDS and writes its items' outputs.  No workgroup waits for another, and no memory is needed between them.
// (The price is quadratic: 24,000 segments take 13 us, 1,000,000 take 230, their 1.5 million new tokens 440.)
// Items per workgroup: as many as leave some 512 workgroups; with fewer items several workgroups share one item's
// outputs.
//
// Measured: the table of 240 segments 5.0 us and the slots of 1024 branches' next tokens 6.2, both a chain of four
// or five dependent loads behind the launch; the table of 24,064 segments with 1.4 million pages 13.2 us (21 with
// sums exchanged through LDS; a workgroup of 1024 threads and 90 registers has its CU alone, so 512 of them take
// 20), half of it the counts before a workgroup's items; the slots of 2.6 million prompt tokens 11.7 us = 2.7 TB/s
// of what is written (14.6 with every token found by itself).
#include "step_internal.hpp"

namespace ga {
namespace {

constexpr int kMaxTile = 1024;
constexpr int kGroup = 16;         // lanes that walk a branch's path together

typedef int i32x4 __attribute__((ext_vector_type(4), aligned(4)));
typedef long i64x2 __attribute__((ext_vector_type(2), aligned(8)));

struct Two {
  int64_t n, x;
};

// Exclusive sums of v over the workgroup's threads (in thread order), its total, and the total of w.
template <int NT>
__device__ __forceinline__ Two block_scan(Two v, Two* total, Two w, Two* other) {
  __shared__ Two sums[NT / 64][2];
  const int wave = threadIdx.x >> 6;
  const Two s{wave_scan(v.n), wave_scan(v.x)}, t{wave_scan(w.n), wave_scan(w.x)};
  if ((threadIdx.x & 63) == 63) {
    sums[wave][0] = s;
    sums[wave][1] = t;
  }
  __syncthreads();
  Two before{0, 0}, all{0, 0}, rest{0, 0};
#pragma unroll
  for (int i = 0; i < NT / 64; ++i) {
    if (i == wave) before = all;
    all.n += sums[i][0].n;
    all.x += sums[i][0].x;
    rest.n += sums[i][1].n;
    rest.x += sums[i][1].x;
  }
  *total = all;
  *other = rest;
  return {before.n + s.n - v.n, before.x + s.x - v.x};
}

// The last i with begin[i] <= j, of n items in ascending order (begin[0] = 0 <= j).
__device__ __forceinline__ int find(const int64_t* begin, int n, int64_t j) {
  int lo = 0;
  for (int step = n > 1 ? 1 << (31 - __builtin_clz(n - 1)) : 0; step > 0; step >>= 1)
    if (lo + step < n && begin[lo + step] <= j) lo += step;
  return lo;
}

// (fewer than 2^31 old pages: what is left of an offset fits 32 bits)
__device__ __forceinline__ int32_t held(const PageTableArgs& a, int64_t offset) {
  return offset < 0 ? 0 : (int32_t)(offset < a.n_old_pages ? offset : a.n_old_pages);
}
struct Need {
  int32_t pages, had;
};
__device__ __forceinline__ Need need_of(const PageTableArgs& a, int32_t len, int32_t had) {
  len = max(len, 0);
  had = max(had, 0);
  // ceil((len + spare) / 16) without their sum, which may pass 32 bits.
  const int32_t want = (len >> 4) + (a.spare >> 4) + (((len & 15) + (a.spare & 15) + kPageTokens - 1) >> 4);
  return {max(want, had), had};
}
__device__ __forceinline__ Need need_of(const PageTableArgs& a, int32_t s) {
  return need_of(a, a.seg_len[s], s < a.S_old ? held(a, a.old_offsets[s + 1]) - held(a, a.old_offsets[s]) : 0);
}

template <int NT>
__global__ __launch_bounds__(NT) void k_page_table(PageTableArgs a) {
  extern __shared__ int64_t lds[];
  int64_t* const begin = lds;                        // of a segment's pages, among the tile's
  int64_t* const old = begin + a.tile;               // its first old page
  int64_t* const fresh = old + a.tile;               // the free page that its page 0 would be
  int32_t* const had = reinterpret_cast<int32_t*>(fresh + a.tile);
  const int tid = threadIdx.x;
  const int64_t t0 = (int64_t)blockIdx.x * a.tile;
  const int n = (int)(a.S - t0 < a.tile ? a.S - t0 : a.tile);
  const int per = (a.tile + NT - 1) / NT;
  Two mine{0, 0}, total;
  for (int k = 0; k < per; ++k) {
    const int i = tid * per + k;
    if (i < n) {
      const Need d = need_of(a, (int32_t)(t0 + i));
      begin[i] = d.pages;
      had[i] = d.had;
      old[i] = t0 + i < a.S_old ? held(a, a.old_offsets[t0 + i]) : 0;
      mine.n += d.pages;
      mine.x += d.pages - d.had;
    }
  }
  // Pages, and new ones, of the segments before this workgroup's: four segments a thread at a time, those that had
  // pages (up to `both`) and those that had none.
  Two sum{0, 0}, before;
  const int64_t both = (a.S_old < t0 ? a.S_old : t0) & ~3LL;
  const auto add = [&](const Need& d) {
    sum.n += d.pages;
    sum.x += d.pages - d.had;
  };
#pragma unroll 2
  for (int64_t s = 4 * tid; s < both; s += 4 * NT) {
    const i32x4 len = *reinterpret_cast<const i32x4*>(a.seg_len + s);
    const i64x2 lo = *reinterpret_cast<const i64x2*>(a.old_offsets + s);
    const i64x2 hi = *reinterpret_cast<const i64x2*>(a.old_offsets + s + 2);
    const int32_t o[5] = {held(a, lo[0]), held(a, lo[1]), held(a, hi[0]), held(a, hi[1]),
                          held(a, a.old_offsets[s + 4])};
#pragma unroll
    for (int k = 0; k < 4; ++k) add(need_of(a, len[k], o[k + 1] - o[k]));
  }
  const int64_t one = a.S_old < t0 ? a.S_old : t0, rest = one + ((t0 - one) & ~3LL);
  if (both + tid < one) add(need_of(a, (int32_t)(both + tid)));
#pragma unroll 2
  for (int64_t s = one + 4 * tid; s < rest; s += 4 * NT) {
    const i32x4 len = *reinterpret_cast<const i32x4*>(a.seg_len + s);
#pragma unroll
    for (int k = 0; k < 4; ++k) add(need_of(a, len[k], 0));
  }
  if (rest + tid < t0) add(need_of(a, (int32_t)(rest + tid)));
  Two at = block_scan<NT>(mine, &total, sum, &before);
  for (int k = 0; k < per; ++k) {
    const int i = tid * per + k;
    if (i < n) {
      const int64_t pages = begin[i];
      begin[i] = at.n;
      fresh[i] = before.x + at.x - had[i];
      if (blockIdx.y == 0) a.offsets[t0 + i] = before.n + at.n;
      at.n += pages;
      at.x += pages - had[i];
    }
  }
  if (blockIdx.y == 0 && blockIdx.x == gridDim.x - 1 && tid == 0) a.offsets[a.S] = before.n + total.n;
  __syncthreads();
  const int64_t room = a.capacity - before.n;        // (may be negative)
  const int64_t end = total.n < room ? total.n : room;
  for (int64_t j = 4 * ((int64_t)blockIdx.y * NT + tid); j < end; j += 4 * NT * (int64_t)gridDim.y) {
    int i = find(begin, n, j);
    i32x4 page;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      while (i + 1 < n && begin[i + 1] <= j + k) ++i;
      const int64_t p = j + k - begin[i];
      const bool is_old = p < had[i];
      const int64_t from = p + (is_old ? old[i] : fresh[i]);
      page[k] = -1;
      if (j + k < end && from < (is_old ? a.n_old_pages : a.n_free))
        page[k] = (is_old ? a.old_pages : a.free_pages)[from];
    }
    int32_t* const out = a.pages + before.n + j;
    if (j + 4 <= end) *reinterpret_cast<i32x4*>(out) = page;
    else
      for (int k = 0; k < (int)(end - j); ++k) out[k] = page[k];
  }
}

__device__ __forceinline__ int64_t count_of(int32_t c) { return c > 0 ? c : 0; }

template <int NT>
__global__ __launch_bounds__(NT) void k_slot_map(SlotMapArgs a) {
  extern __shared__ int64_t lds[];
  int64_t* const begin = lds;                        // of a branch's rows, among the tile's
  int64_t* const first = begin + a.tile;             // its last segment's pages
  int64_t* const last = first + a.tile;
  int64_t* const base = last + a.tile;               // tokens of its other segments
  int32_t* const token = reinterpret_cast<int32_t*>(base + a.tile);   // of its first row; may be below 0
  const int tid = threadIdx.x;
  const int32_t B = a.g.num_branches;
  const int64_t tile0 = (int64_t)blockIdx.x * a.tile;
  const int n = (int)(B - tile0 < a.tile ? B - tile0 : a.tile);
  // Its branches' paths, by some lanes each.
  const int lane = tid % kGroup;
  for (int i0 = 0; i0 < n; i0 += NT / kGroup) {      // (whole waves go round, for the row operations)
    const int i = i0 + tid / kGroup;
    const bool there = i < n;
    const int64_t c = there && a.counts ? count_of(a.counts[tile0 + i]) : 1;
    const PathRange p = there ? path_range(a.g, (int32_t)(tile0 + i)) : PathRange{0, 0};
    int64_t before = 0;
    if (there && p.first >= p.end && lane == 0) {             // no segment: a token below 0 in every row
      token[i] = -0x7fffffff;
      first[i] = last[i] = 0;
    }
    for (int64_t e = p.first + lane; e < p.end; e += kGroup) {
      const int32_t s = a.g.path_segs[e];
      const SegRange r = seg_range(a.g, s);
      if (e + 1 < p.end) {
        before += r.len;
      } else {
        const int64_t t = s >= 0 && s < a.g.num_segments ? r.len - c : -0x7fffffff;
        token[i] = (int32_t)(t < -0x7fffffff ? -0x7fffffff : t);
        first[i] = r.first;
        last[i] = r.end;
      }
    }
    if (there && lane == 0) begin[i] = c;
    // (the sum of a group's lanes, in its last one)
    add_lane<0x111, 0xf>(&before);
    add_lane<0x112, 0xf>(&before);
    add_lane<0x114, 0xf>(&before);
    add_lane<0x118, 0xf>(&before);
    if (there && lane == kGroup - 1) base[i] = before;
  }
  Two sum{0, 0}, before;
  if (a.counts) {
    const int64_t whole = tile0 & ~3LL;
#pragma unroll 2
    for (int64_t b = 4 * tid; b < whole; b += 4 * NT) {
      const i32x4 c = *reinterpret_cast<const i32x4*>(a.counts + b);
#pragma unroll
      for (int k = 0; k < 4; ++k) sum.n += count_of(c[k]);
    }
    if (whole + tid < tile0) sum.n += count_of(a.counts[whole + tid]);
  }
  __syncthreads();
  const int per = (a.tile + NT - 1) / NT;
  Two mine{0, 0}, total;
  for (int k = 0; k < per; ++k)
    if (tid * per + k < n) mine.n += begin[tid * per + k];
  Two at = block_scan<NT>(mine, &total, sum, &before);
  if (!a.counts) before = {tile0, 0};
  auto held = [](int64_t x) { return (int32_t)(x < 0x7fffffff ? x : 0x7fffffff); };
  for (int k = 0; k < per; ++k) {
    const int i = tid * per + k;
    if (i < n) {
      const int64_t c = begin[i];
      begin[i] = at.n;
      if (blockIdx.y == 0) a.offsets[tile0 + i] = held(before.n + at.n);
      at.n += c;
    }
  }
  const bool closes = blockIdx.x == gridDim.x - 1;
  if (blockIdx.y == 0 && closes && tid == 0) a.offsets[B] = held(before.n + total.n);
  __syncthreads();
  const int64_t room = (int64_t)a.capacity - before.n;
  const int64_t rows = total.n < room ? total.n : room;
  // The last branches' workgroups write the padding behind the rows too.
  const int64_t end = closes ? room : rows;
  for (int64_t j = 4 * ((int64_t)blockIdx.y * NT + tid); j < end; j += 4 * NT * (int64_t)gridDim.y) {
    i32x4 word, pos, branch;
    int i = n > 0 && j < rows ? find(begin, n, j) : 0;
    const int64_t next = i + 1 < n ? begin[i + 1] : total.n;
    const int64_t t0 = n > 0 ? token[i] + (j - begin[i]) : -1;
    if (j + 4 <= rows && j + 4 <= next && t0 >= 0 && (t0 & 15) <= 12 && base[i] + t0 < 0x7ffffff0LL) {
      // Four tokens of one segment and page.
      const int32_t page = a.words ? page_of(a.g, first[i], last[i], (int32_t)t0) : -1;
      const int32_t w = page * kPageTokens + (int32_t)(t0 & (kPageTokens - 1)), p = (int32_t)(base[i] + t0);
      const int32_t one = page < 0 ? 0 : 1, from = page < 0 ? -1 : w;
      word = i32x4{from, from + one, from + 2 * one, from + 3 * one};
      pos = i32x4{p, p + 1, p + 2, p + 3};
      const int32_t b = (int32_t)tile0 + i;
      branch = i32x4{b, b, b, b};
    } else {
      int64_t entry = -1;                            // of the table, whose page `page` is
      int32_t page = -1;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        word[k] = pos[k] = branch[k] = -1;
        if (j + k < rows) {
          while (i + 1 < n && begin[i + 1] <= j + k) ++i;
          const int64_t t = token[i] + (j + k - begin[i]), p = base[i] + t;
          if (t >= 0 && p < 0x80000000LL) {
            pos[k] = (int32_t)p;
            branch[k] = (int32_t)tile0 + i;
            if (a.words) {
              const int64_t at = first[i] + (t >> 4);
              if (at != entry && at < last[i]) {
                page = page_of(a.g, first[i], last[i], (int32_t)t);
                entry = at;
              }
              word[k] = at < last[i] && page >= 0 ? page * kPageTokens + (int32_t)(t & (kPageTokens - 1)) : -1;
            }
          }
        }
      }
    }
    const int64_t out = before.n + j;
    const auto put = [&](int32_t* to, const i32x4& v) {
      if (!to) return;
      if (j + 4 <= end) *reinterpret_cast<i32x4*>(to + out) = v;
      else
        for (int k = 0; k < (int)(end - j); ++k) to[out + k] = v[k];
    };
    put(a.words, word);
    put(a.positions, pos);
    put(a.branches, branch);
  }
}

// Items of a workgroup, and workgroups of the same items: one for every four outputs a thread that the caller's
// capacity lets expect, up to 1024 of 256 threads.  (64 to 512 workgroups of items are as fast as each other for
// 1024 branches, 6.2 to 6.5 us; of 2.6 million rows 1024 workgroups take 11.7 us, 2048 12.3.)
dim3 tiles_of(int64_t items, int64_t capacity, int threads, int32_t* tile) {
  const int64_t most = threads == 256 ? 512 : 256, t = (items + most - 1) / most;
  *tile = (int32_t)(t < 1 ? 1 : t > kMaxTile ? kMaxTile : t);
  const int64_t tiles = items > 0 ? (items + *tile - 1) / *tile : 1;
  const int64_t want = capacity / (tiles * 4 * threads), room = 1024 * 256 / threads / tiles;
  const int64_t splits = want < room ? want : room;
  return dim3((unsigned)tiles, (unsigned)(splits < 1 ? 1 : splits));
}
// From some thousand items on, the counts before a workgroup's are worth more threads.  256 and 1024 threads, us:
// tables of 1504 segments 5.1 and 7.0, 4089 6.1 and 7.4, 7050 7.0 and 8.0, 8930 8.9 and 8.5, 12032 10.8 and 8.8,
// 24064 16.4 and 12.4; slots of 1024 branches 5.7 and 7.5, 6400 7.1 and 8.3, 11200 8.4 and 8.2, 24000 10.5 and 9.6,
// 96000 36 and 22.
int threads_of(int64_t items) { return items > 4096 ? 1024 : 256; }

}  // namespace

hipError_t launch_page_table(const PageTableArgs& args, hipStream_t stream) {
  PageTableArgs a = args;
  const int threads = threads_of(a.S);
  const dim3 grid = tiles_of(a.S, a.capacity, threads, &a.tile);
  const size_t lds = (size_t)a.tile * 28;
  if (threads == 256) hipLaunchKernelGGL(k_page_table<256>, grid, dim3(256), lds, stream, a);
  else hipLaunchKernelGGL(k_page_table<1024>, grid, dim3(1024), lds, stream, a);
  return hipGetLastError();
}

hipError_t launch_slot_map(const SlotMapArgs& args, hipStream_t stream) {
  SlotMapArgs a = args;
  const int threads = threads_of(a.g.num_branches);
  const dim3 grid = tiles_of(a.g.num_branches, a.capacity, threads, &a.tile);
  const size_t lds = (size_t)a.tile * 36;
  if (threads == 256) hipLaunchKernelGGL(k_slot_map<256>, grid, dim3(256), lds, stream, a);
  else hipLaunchKernelGGL(k_slot_map<1024>, grid, dim3(1024), lds, stream, a);
  return hipGetLastError();
}

}  // namespace ga
