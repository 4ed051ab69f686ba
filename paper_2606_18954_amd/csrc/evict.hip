// Which tokens of a segment stay: its first tokens, its most recent ones and, of the others, those with
// the largest mass, ties to the lower position; in ascending order, as positions and as slot words.
//
// Keys order like the masses: the float's bits, negative ones inverted and positive ones with the sign
// bit set; -0 counts as 0, a NaN above every number (its weight is unknown: the token stays), and a
// protected token above that.  The keep-th largest key T is built bit by bit from the top (the largest
// T that at least keep keys reach); a step is one comparison and one ballot for 64 keys, and the
// search ends early once exactly keep keys reach the candidate.  Then every key above T stays and, in
// order of position, as many of those equal to T as are missing.
//
// Segments of up to kEvictWave tokens: one wave each, keys and words in registers, no barrier.  Up to
// kEvictGroup: one workgroup of 1024 threads, a barrier a bit.  Longer ones: the same, but the keys are
// read again for every bit.
#include "evict_internal.hpp"

namespace ga {
namespace {

__device__ __forceinline__ unsigned key_of(float x) {
  const unsigned b = __builtin_bit_cast(unsigned, x + 0.f);
  if ((b & 0x7fffffffu) > 0x7f800000u) return 0xfffffffeu;
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Word and key of token t (key 0, below every token's, past the segment's end).
__device__ __forceinline__ void token(const EvictArgs& a, const EvictSeg& s, int t, int& word,
                                      unsigned& key) {
  word = 0;
  key = 0;
  if (t < s.len) {
    word = a.pages[s.pages + (t >> 4)] * kPageTokens + (t & 15);
    key = t < a.first || t >= s.len - a.recent ? 0xffffffffu : key_of(a.mass[word]);
  }
}

__device__ __forceinline__ int below(uint64_t m, int lane) {
  return __builtin_popcountll(m & ((1ull << lane) - 1));
}

__global__ __launch_bounds__(256) void k_evict_wave(EvictArgs a) {
  constexpr int NK = kEvictWave / 64;
  const int lane = threadIdx.x & 63;
  const int id = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  if (id >= a.n_wave) return;
  const EvictSeg s = a.segs[id];
  int word[NK];
  unsigned key[NK];
#pragma unroll
  for (int i = 0; i < NK; ++i) token(a, s, 64 * i + lane, word[i], key[i]);
  unsigned T = 0;
  int reach = 0;
  if (s.keep > 0)
    for (int bit = 31; bit >= 0; --bit) {
      const unsigned cand = T | (1u << bit);
      int c = 0;
#pragma unroll
      for (int i = 0; i < NK; ++i) c += __builtin_popcountll(__ballot(key[i] >= cand));
      if (c >= s.keep) {
        T = cand;
        reach = c;
        if (c == s.keep) break;
      }
    }
  else
    T = 0xffffffffu;
  // Keys that reach T all stay where they are as many as wanted; else those equal to it only as far
  // as wanted.
  int above = 0;
  if (s.keep > 0 && reach != s.keep) {
#pragma unroll
    for (int i = 0; i < NK; ++i) above += __builtin_popcountll(__ballot(key[i] > T));
  }
  int ties = s.keep > 0 ? (reach == s.keep ? 0x7fffffff : s.keep - above) : 0;
  int64_t out = s.out;
#pragma unroll
  for (int i = 0; i < NK; ++i) {
    const bool eq = key[i] == T && key[i] != 0;
    const uint64_t me = __ballot(eq);
    const bool stay = key[i] > T || (eq && below(me, lane) < ties);
    ties -= min(ties, (int)__builtin_popcountll(me));
    const uint64_t ms = __ballot(stay);
    if (stay) {
      const int64_t o = out + below(ms, lane);
      if (a.positions) a.positions[o] = 64 * i + lane;
      if (a.words) a.words[o] = word[i];
    }
    out += __builtin_popcountll(ms);
  }
}

// One workgroup of 16 waves per segment.
template <bool LONG>
__global__ __launch_bounds__(1024) void k_evict_group(EvictArgs a) {
  constexpr int NK = 16;
  __shared__ int s_cnt[33];
  __shared__ int s_gt[NK * 16], s_eq[NK * 16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const EvictSeg s = a.segs[a.n_wave + (LONG ? a.n_group : 0) + (int)blockIdx.x];
  const int nblk = LONG ? (s.len + kEvictGroup - 1) / kEvictGroup : 1;
  if (tid < 33) s_cnt[tid] = 0;
  int word[NK];
  unsigned key[NK];
  auto load = [&](int blk) {
#pragma unroll
    for (int i = 0; i < NK; ++i)
      token(a, s, blk * kEvictGroup + 1024 * i + tid, word[i], key[i]);
  };
  load(0);
  __syncthreads();
  unsigned T = 0;
  int reach = 0;
  // Keys of the whole segment that reach x, through counter slot k.
  auto count = [&](unsigned x, int k) {
    int c = 0;
    for (int blk = 0; blk < nblk; ++blk) {
      if (LONG) load(blk);
#pragma unroll
      for (int i = 0; i < NK; ++i) c += __builtin_popcountll(__ballot(key[i] >= x));
    }
    if (lane == 0) atomicAdd(&s_cnt[k], c);
    __syncthreads();
    return s_cnt[k];
  };
  if (s.keep > 0)
    for (int bit = 31; bit >= 0; --bit) {
      const unsigned cand = T | (1u << bit);
      const int c = count(cand, bit);
      if (c >= s.keep) {
        T = cand;
        reach = c;
        if (c == s.keep) break;
      }
    }
  else
    T = 0xffffffffu;
  int ties = 0;
  if (s.keep > 0) ties = reach == s.keep ? 0x7fffffff : s.keep - (T == 0xffffffffu ? 0 : count(T + 1, 32));
  int64_t out = s.out;
  for (int blk = 0; blk < nblk; ++blk) {
    if (LONG) load(blk);
    // Per run of 64 tokens: keys above T and equal to it; then the running sums of both.
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const int g = __builtin_popcountll(__ballot(key[i] > T));
      const int e = __builtin_popcountll(__ballot(key[i] == T && key[i] != 0));
      if (lane == 0) {
        s_gt[16 * i + wave] = g;
        s_eq[16 * i + wave] = e;
      }
    }
    __syncthreads();
    if (wave == 0) {
      // 256 runs, four a lane
      int g[4], e[4], sg = 0, se = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        g[k] = s_gt[4 * lane + k];
        e[k] = s_eq[4 * lane + k];
        sg += g[k];
        se += e[k];
      }
      int pg = sg, pe = se;
#pragma unroll
      for (int d = 1; d < 64; d *= 2) {
        const int x = __shfl_up(pg, d), y = __shfl_up(pe, d);
        if (lane >= d) { pg += x; pe += y; }
      }
      pg -= sg;
      pe -= se;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        s_gt[4 * lane + k] = pg;
        s_eq[4 * lane + k] = pe;
        pg += g[k];
        pe += e[k];
      }
      if (lane == 63) {
        s_cnt[0] = pg;            // (the bits' counters are no longer needed)
        s_cnt[1] = pe;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NK; ++i) {
      const int pg = s_gt[16 * i + wave], pe = s_eq[16 * i + wave];
      const bool eq = key[i] == T && key[i] != 0;
      const uint64_t me = __ballot(eq);
      const bool stay = key[i] > T || (eq && pe + below(me, lane) < ties);
      const uint64_t ms = __ballot(stay);
      if (stay) {
        const int64_t o = out + pg + min(pe, ties) + below(ms, lane);
        if (a.positions) a.positions[o] = blk * kEvictGroup + 1024 * i + tid;
        if (a.words) a.words[o] = word[i];
      }
    }
    const int tg = s_cnt[0], te = min(s_cnt[1], ties);
    out += tg + te;
    ties -= te;
    __syncthreads();
  }
}

}  // namespace

hipError_t launch_evict(const EvictArgs& a, hipStream_t stream) {
  if (a.n_wave)
    hipLaunchKernelGGL(k_evict_wave, dim3((unsigned)((a.n_wave + 3) / 4)), dim3(256), 0, stream, a);
  if (a.n_group)
    hipLaunchKernelGGL(k_evict_group<false>, dim3((unsigned)a.n_group), dim3(1024), 0, stream, a);
  if (a.n_long)
    hipLaunchKernelGGL(k_evict_group<true>, dim3((unsigned)a.n_long), dim3(1024), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ga
