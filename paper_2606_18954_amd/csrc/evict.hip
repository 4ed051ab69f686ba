// Which tokens of a segment stay: its first tokens, its most recent ones and, of the others, those with
// the largest mass, ties to the lower position; in ascending order, as positions and as slot words.
//
// Keys order like the masses: the float's bits, negative ones inverted and positive ones with the sign
// bit set; -0 counts as 0, a NaN above every number (its weight is unknown: the token stays), and a
// protected token above that.  With need = keep - (protected tokens), the search keeps a lower key that at
// least need of the other keys reach and an upper one that fewer reach, and counts how many reach a key
// between them, where the line through the two counts meets need.  A step is one comparison and one ballot
// for 64 keys.  Where at most 64 keys are left between the bounds they are gathered in LDS, one a lane, and
// ranked against each other.  Zeros (tokens that no row saw) lie far below all other masses: the search
// begins above them where enough keys do.  Masses of a softmax take three steps at 500 tokens and six at
// 8,000 (bit by bit it took 14 and 18); every other step after the twelfth halves the range, so that 76 end
// it whatever the masses are.  Then every key above T stays and, in order of position, as many of those
// equal to T as are missing.
//
// Segments of up to kEvictWave tokens: one wave each, keys and words in registers, no barrier.  Up to
// kEvictGroup: one workgroup of 1024 threads, a barrier a step.  Longer ones: the same, but the keys are
// read again for every step.
//
// What bounds it: latency.  3266 segments of 64 to 1024 tokens (1.8 M tokens, 14 MB), half of them kept: 11 to
// 14 us, half of it the three dependent loads (segment, page word, mass) of each wave; 256 segments of 8192:
// 14 to 15 us, one workgroup per CU with a barrier a step.  The bytes would take 2.8 and 2.4 us.  Bit by bit,
// and one token's loads after another's, they took 15.4 and 20.2.
//
// A segment that is read again must find the masses it found before; where another stream writes them
// meanwhile, the choice is any, but nothing outside the segment's outputs is written and every search ends.
#include "evict_internal.hpp"

namespace ga {
namespace {

__device__ __forceinline__ unsigned key_of(float x) {
  const unsigned b = __builtin_bit_cast(unsigned, x + 0.f);
  return x != x ? 0xfffffffeu : b ^ ((unsigned)((int)b >> 31) | 0x80000000u);
}

// Words and keys of N tokens from t on, STEP apart (key 0, below every token's, past the segment's end: those
// lanes load the last token's, so that every load is issued before the first is waited for).
template <int N, int STEP>
__device__ __forceinline__ void tokens(const EvictArgs& a, const EvictSeg& s, int t, int* word,
                                       unsigned* key) {
  float m[N];
  const int32_t* pages = a.pages + s.pages;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const unsigned u = (unsigned)min(t + STEP * i, s.len - 1);
    word[i] = pages[u >> 4] * kPageTokens + (int)(u & 15);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) m[i] = a.mass[(unsigned)word[i]];
#pragma unroll
  for (int i = 0; i < N; ++i) key[i] = key_of(m[i]);
  // (t - lane: uniform, the first of the wave's tokens)
  const int t0 = __builtin_amdgcn_readfirstlane(t);
  if (t0 >= a.first && t0 + STEP * (N - 1) + 63 < s.len - a.recent) return;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int u = t + STEP * i;
    if (u < a.first || u >= s.len - a.recent) key[i] = 0xffffffffu;
    if (u >= s.len) key[i] = 0;
  }
}

// Lanes below this one in m.
__device__ __forceinline__ int below(uint64_t m) {
  return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0));
}

constexpr unsigned kZeroKey = 0x80000000u;           // of no mass, and of -0

// The search's bounds: of the unprotected keys clo >= need reach lo, chi < need reach hi.  A bound that stays
// twice weighs half as much in the next line (an uneven spread of the keys would keep one for many steps).
struct Bounds {
  unsigned lo, hi;
  int clo, chi;
  float wlo = 1.f, whi = 1.f;
  int last = 0;
  __device__ __forceinline__ bool closed(int need) const { return clo == need || hi - lo == 1; }
  __device__ __forceinline__ bool far(int need) const { return !closed(need) && clo - chi > 64; }
  __device__ __forceinline__ bool holds(unsigned k) const { return k - lo < hi - lo; }
  // The step's key, in (lo, hi).
  __device__ __forceinline__ unsigned next(int need, int step) const {
    const unsigned span = hi - lo;
    if (step == 0 && hi == kZeroKey + 1) return kZeroKey;   // (often they are all zero)
    if (step >= 12 && (step & 1)) return lo + span / 2;
    const float b = ((float)(clo - need) + 0.5f) * wlo, t = ((float)(need - chi) - 0.5f) * whi;
    const float at = (float)span * (b * __builtin_amdgcn_rcpf(b + t));
    // (a product that rounds up to the span is kept below it)
    return lo + min(max((unsigned)fminf(at, 4.2e9f), 1u), span - 1);
  }
  __device__ __forceinline__ void set(unsigned x, int c, int need) {
    if (c >= need) {
      lo = x;
      clo = c;
      wlo = 1.f;
      whi = last > 0 ? 0.5f * whi : 1.f;
      last = 1;
    } else {
      hi = x;
      chi = c;
      whi = 1.f;
      wlo = last < 0 ? 0.5f * wlo : 1.f;
      last = -1;
    }
  }
};

// Among the m = clo - chi <= 64 keys between the bounds, one a lane (0: none), the one at which need is reached
// becomes the lower bound, with its neighbour above.
__device__ __forceinline__ void rank_rest(Bounds& x, unsigned mine, int need) {
  const int m = min(x.clo - x.chi, 64), want = need - x.chi;
  int above = 0, reach = 0;
  for (int j = 0; j < m; ++j) {
    const unsigned k = __builtin_amdgcn_readlane(mine, j);
    above += k > mine;
    reach += k >= mine;
  }
  const uint64_t at = __ballot(mine != 0 && above < want && want <= reach);
  const int l = at ? __builtin_ctzll(at) : 0;
  x.lo = __builtin_amdgcn_readlane(mine, l);
  x.hi = x.lo + 1;
  x.clo = x.chi + __builtin_amdgcn_readlane(reach, l);
  x.chi += __builtin_amdgcn_readlane(above, l);
}

// The bounds the search begins with: of n open keys pos lie above zero's, kmin .. kmax.  (Below them no key is
// under 0x7fffff, minus infinity's.)
__device__ __forceinline__ Bounds first_bounds(int n, int pos, unsigned kmin, unsigned kmax, int need) {
  if (pos >= need) return Bounds{kmin, kmax + 1, pos, 0};
  return Bounds{1, kZeroKey + 1, n, pos};
}

__device__ __forceinline__ bool positive_key(unsigned k) { return k > kZeroKey && k != 0xffffffffu; }

// Least and largest of a wave's values, in every lane: exchanges within rows of 16 lanes, then between them.
__device__ __forceinline__ void wave_min_max(unsigned& lo, unsigned& hi) {
  auto step = [&](auto f) {
    lo = min(lo, (unsigned)f((int)lo));
    hi = max(hi, (unsigned)f((int)hi));
  };
  step([](int x) { return __builtin_amdgcn_mov_dpp(x, 0xB1, 0xf, 0xf, true); });    // lane ^ 1
  step([](int x) { return __builtin_amdgcn_mov_dpp(x, 0x4E, 0xf, 0xf, true); });    // lane ^ 2
  step([](int x) { return __builtin_amdgcn_mov_dpp(x, 0x141, 0xf, 0xf, true); });   // 7 - lane, of 8
  step([](int x) { return __builtin_amdgcn_mov_dpp(x, 0x140, 0xf, 0xf, true); });   // 15 - lane, of 16
  unsigned l = 0xffffffffu, h = 0;
#pragma unroll
  for (int row = 0; row < 64; row += 16) {
    l = min(l, (unsigned)__builtin_amdgcn_readlane((int)lo, row));
    h = max(h, (unsigned)__builtin_amdgcn_readlane((int)hi, row));
  }
  lo = l;
  hi = h;
}

// LDS written by a wave's lanes, read by its others.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

__global__ __launch_bounds__(256) void k_evict_wave(EvictArgs a) {
  constexpr int NK = kEvictWave / 64, NB = 4;        // keys a lane, in runs of NB that a segment has or not
  __shared__ unsigned s_rest[4][64];                 // (each wave has its own: no barrier)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  const int id = (int)blockIdx.x * 4 + wave;
  if (id >= a.n_wave) return;
  s_rest[wave][lane] = 0;
  wave_sync();
  const EvictSeg s = a.segs[id];
  int word[NK];
  unsigned key[NK];
  unsigned kmin = 0xffffffffu, kmax = 0;
  int pos = 0;
  auto runs = [&](auto f) {
#pragma unroll
    for (int b = 0; b < NK; b += NB)
      if (64 * b < s.len) f(b);
  };
  runs([&](int b) {
    tokens<NB, 64>(a, s, 64 * b + lane, word + b, key + b);
  });
  runs([&](int b) {
#pragma unroll
    for (int i = b; i < b + NB; ++i) {
      const bool p = positive_key(key[i]);
      pos += __builtin_popcountll(__ballot(p));
      kmin = min(kmin, p ? key[i] : 0xffffffffu);
      kmax = max(kmax, p ? key[i] : 0);
    }
  });
  const int safe = (int)min((int64_t)s.len, (int64_t)a.first + a.recent);
  const int need = s.keep - safe;
  unsigned T = 0xfffffffeu;                          // keys above T stay, and `ties` of those equal to it
  int ties = 0;
  if (need > 0) {
    wave_min_max(kmin, kmax);
    Bounds x = first_bounds(s.len - safe, pos, kmin, kmax, need);
    for (int step = 0; x.far(need); ++step) {
      const unsigned k = __builtin_amdgcn_readfirstlane(x.next(need, step));
      int c = -safe;                                 // (protected keys reach every k)
      runs([&](int b) {
#pragma unroll
        for (int i = b; i < b + NB; ++i) c += __builtin_popcountll(__ballot(key[i] >= k));
      });
      x.set(k, c, need);
    }
    if (!x.closed(need)) {
      int at = 0;
      runs([&](int b) {
#pragma unroll
        for (int i = b; i < b + NB; ++i) {
          const uint64_t in = __ballot(x.holds(key[i]));
          if (x.holds(key[i])) s_rest[wave][at + below(in)] = key[i];
          at += __builtin_popcountll(in);
        }
      });
      wave_sync();
      rank_rest(x, s_rest[wave][lane], need);
    }
    T = x.clo == need ? x.lo - 1 : x.lo;
    ties = x.clo == need ? 0 : need - x.chi;
  }
  int32_t* positions = a.positions ? a.positions + s.out : nullptr;
  int32_t* words = a.words ? a.words + s.out : nullptr;
  unsigned out = 0;
  runs([&](int b) {
#pragma unroll
    for (int i = b; i < b + NB; ++i) {
      bool stay = key[i] > T;
      if (ties > 0) {                                // (the same in every lane)
        const bool eq = key[i] == T;
        const uint64_t me = __ballot(eq);
        stay = stay || (eq && below(me) < ties);
        ties -= min(ties, (int)__builtin_popcountll(me));
      }
      const uint64_t ms = __ballot(stay);
      if (stay) {
        const unsigned o = out + (unsigned)below(ms);
        if (positions) positions[o] = 64 * i + lane;
        if (words) words[o] = word[i];
      }
      out += (unsigned)__builtin_popcountll(ms);
    }
  });
}

// One workgroup of 16 waves per segment.
template <bool LONG>
__global__ __launch_bounds__(1024) void k_evict_group(EvictArgs a) {
  constexpr int NK = 16, NB = 4;
  __shared__ int s_cnt[3];                           // counts of three steps in turn
  __shared__ int s_sum[2], s_pos, s_num;
  __shared__ unsigned s_rest[64];
  __shared__ unsigned s_min, s_max;
  __shared__ int s_gt[NK * 16], s_eq[NK * 16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const EvictSeg s = a.segs[a.n_wave + (LONG ? a.n_group : 0) + (int)blockIdx.x];
  const int nblk = LONG ? (s.len + kEvictGroup - 1) / kEvictGroup : 1;
  if (tid < 3) s_cnt[tid] = 0;
  if (tid < 64) s_rest[tid] = 0;
  if (tid == 0) {
    s_pos = s_num = 0;
    s_min = 0xffffffffu;
    s_max = 0;
  }
  int word[NK];
  unsigned key[NK];
  auto runs = [&](int blk, auto f) {
#pragma unroll
    for (int b = 0; b < NK; b += NB)
      if (blk * kEvictGroup + 1024 * b < s.len) f(b);
  };
  auto load = [&](int blk) {
    runs(blk, [&](int b) {
      tokens<NB, 1024>(a, s, blk * kEvictGroup + 1024 * b + tid, word + b, key + b);
    });
  };
  load(0);
  const int safe = (int)min((int64_t)s.len, (int64_t)a.first + a.recent);
  const int need = s.keep - safe;
  unsigned T = 0xfffffffeu;
  int ties = 0;
  __syncthreads();
  if (need > 0) {
    unsigned kmin = 0xffffffffu, kmax = 0;
    int pos = 0;
    for (int blk = 0; blk < nblk; ++blk) {
      if (LONG && blk) load(blk);
      runs(blk, [&](int b) {
#pragma unroll
        for (int i = b; i < b + NB; ++i) {
          const bool p = positive_key(key[i]);
          pos += __builtin_popcountll(__ballot(p));
          kmin = min(kmin, p ? key[i] : 0xffffffffu);
          kmax = max(kmax, p ? key[i] : 0);
        }
      });
    }
    wave_min_max(kmin, kmax);
    if (lane == 0) {
      atomicAdd(&s_pos, pos);
      atomicMin(&s_min, kmin);
      atomicMax(&s_max, kmax);
    }
    __syncthreads();
    Bounds x = first_bounds(s.len - safe, __builtin_amdgcn_readfirstlane(s_pos),
                            __builtin_amdgcn_readfirstlane(s_min),
                            __builtin_amdgcn_readfirstlane(s_max), need);
    for (int step = 0, k3 = 0; x.far(need); ++step, k3 = k3 == 2 ? 0 : k3 + 1) {
      const unsigned k = __builtin_amdgcn_readfirstlane(x.next(need, step));
      int c = 0;
      for (int blk = 0; blk < nblk; ++blk) {
        if (LONG) load(blk);
        runs(blk, [&](int b) {
#pragma unroll
          for (int i = b; i < b + NB; ++i) c += __builtin_popcountll(__ballot(key[i] >= k));
        });
      }
      if (lane == 0) atomicAdd(&s_cnt[k3], c);
      __syncthreads();
      // The last step's counter is cleared: its readers are past this barrier, its next writers behind the
      // next one.
      if (tid == 0) s_cnt[k3 == 0 ? 2 : k3 - 1] = 0;
      x.set(k, __builtin_amdgcn_readfirstlane(s_cnt[k3]) - safe, need);
    }
    if (!x.closed(need)) {
      for (int blk = 0; blk < nblk; ++blk) {
        if (LONG) load(blk);
        int c = 0;
        runs(blk, [&](int b) {
#pragma unroll
          for (int i = b; i < b + NB; ++i) c += __builtin_popcountll(__ballot(x.holds(key[i])));
        });
        if (c == 0) continue;
        int at = 0;
        if (lane == 0) at = atomicAdd(&s_num, c);
        at = __builtin_amdgcn_readfirstlane(at);
        runs(blk, [&](int b) {
#pragma unroll
          for (int i = b; i < b + NB; ++i) {
            const uint64_t in = __ballot(x.holds(key[i]));
            if (x.holds(key[i]) && (!LONG || at + below(in) < 64)) s_rest[at + below(in)] = key[i];
            at += __builtin_popcountll(in);
          }
        });
      }
      __syncthreads();
      // (one wave: all sixteen would take four times as long)
      if (wave == 0) {
        rank_rest(x, s_rest[lane], need);
        if (lane == 0) {
          s_min = x.lo;
          s_sum[0] = x.clo;
          s_sum[1] = x.chi;
        }
      }
      __syncthreads();
      x.lo = __builtin_amdgcn_readfirstlane(s_min);
      x.clo = __builtin_amdgcn_readfirstlane(s_sum[0]);
      x.chi = __builtin_amdgcn_readfirstlane(s_sum[1]);
    }
    T = x.clo == need ? x.lo - 1 : x.lo;
    ties = x.clo == need ? 0 : need - x.chi;
  }
  unsigned base = 0;                                 // tokens that stayed in the blocks before
  for (int blk = 0; blk < nblk; ++blk) {
    if (LONG) load(blk);
    // Per run of 64 tokens: keys above T and equal to it; then the running sums of both.
#pragma unroll
    for (int b = 0; b < NK; b += NB) {
      const bool any = blk * kEvictGroup + 1024 * b < s.len;
#pragma unroll
      for (int i = b; i < b + NB; ++i) {
        int g = 0, e = 0;
        if (any) {
          g = __builtin_popcountll(__ballot(key[i] > T));
          if (ties > 0) e = __builtin_popcountll(__ballot(key[i] == T));
        }
        if (lane == 0) {
          s_gt[16 * i + wave] = g;
          s_eq[16 * i + wave] = e;
        }
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
        s_sum[0] = pg;
        s_sum[1] = pe;
      }
    }
    __syncthreads();
    int32_t* positions = a.positions ? a.positions + s.out + base : nullptr;
    int32_t* words = a.words ? a.words + s.out + base : nullptr;
    runs(blk, [&](int b) {
#pragma unroll
      for (int i = b; i < b + NB; ++i) {
        unsigned o = (unsigned)s_gt[16 * i + wave];
        bool stay = key[i] > T;
        if (ties > 0) {
          const int pe = s_eq[16 * i + wave];
          const bool eq = key[i] == T;
          stay = stay || (eq && pe + below(__ballot(eq)) < ties);
          o += (unsigned)min(pe, ties);
        }
        const uint64_t ms = __ballot(stay);
        o += (unsigned)below(ms);
        if (stay && (!LONG || base + o < (unsigned)s.keep)) {
          if (positions) positions[o] = blk * kEvictGroup + 1024 * i + tid;
          if (words) words[o] = word[i];
        }
      }
    });
    const int tg = s_sum[0], te = min(s_sum[1], ties);
    base += (unsigned)(tg + te);
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
