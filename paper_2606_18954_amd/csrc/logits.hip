// Logits of a step's rows through penalties, biases, temperature and masks, in one pass over them.
//
// The penalties of a row go by the tokens of its branch's path.  Most of a vocabulary's tokens are not among
// them, so what a row needs is a sparse count, which a dense array per row in memory would turn into as many
// bytes again as the logits.  Here a workgroup takes a slice of a row's vocabulary, counts the path's tokens that
// fall into it in LDS, and streams the slice past the counts; memory carries the logits, once each way.
//
// Counts are 16 bits a token of the slice: 14 bits of count, one for a token with a bias, one for a token of the
// prompt (which counts for the repetition penalty alone).  Rows that could count further than 14 bits take the
// slice in two halves with 32 bits a token.  Every workgroup of a row reads the whole path (4 bytes a token, four
// tokens a load, from L2).
// Biases: the flag says that there is one.  A list of up to 512 a row lies in LDS with the place of the first bias of
// every 32 tokens; a longer one is searched in memory.
//
// Memory bounds it: 1024 rows of 152064 float32 values with penalties and biases, 1.25 GB in 238-254 us (a plain
// copy: 234; without rules 238).  Eight waves per SIMD hide the counting (55 vector registers, one of them with the
// 52 scalar ones that do not fit; at five 376 us): what is uniform and rare, counts of 32 bits, has a loop of its
// own.  1024 rows of four drafted tokens a branch, 65024 bf16 values to float32, contexts of 12200 tokens on average:
// 96-109 us by the card, where the same without penalties takes 63 and a copy 69: the vector unit is busy two thirds
// of the time.  128 rows of 50001 with 300 biases and a mask each: 14 us, half of it the chain from the branch to its
// tokens' counts; one row 6.2.
// (Rows of a branch in one workgroup that goes on with their counts: the drafts 115 us where they took 122, but the
// 1024 rows 303 where they took 256.  Loads of 8 bytes where the output is twice as wide: 84 -> 63 us without rules.)
#include <type_traits>

#include "pool_load.hpp"
#include "step_internal.hpp"

namespace ga {
namespace {

constexpr int kThreads = 1024;
constexpr int kPath = 64;          // segments of a path taken at once
constexpr int kAhead = 2;          // fours of tokens of a thread whose loads are in flight together
constexpr int kBias = 512;         // biases of a row that LDS holds; a longer list is looked up in memory
// Tokens of a slice, so that two workgroups share a CU's LDS: 76 KB of counts, or 72 and the biases.  (With half the
// threads and slices, and four workgroups, every row's path is read twice as often: logits of 1024 rows of four drafted
// tokens a branch over 65024 tokens, contexts of 12200, take 117 us, not 99; 128 rows of 50001 15.6, not 14.6.)
constexpr int kMaxSlice = 38912, kMaxSliceBiased = 36864;

typedef unsigned u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
typedef int i32x4_any __attribute__((ext_vector_type(4), aligned(4)));

struct Path {
  int64_t first[kPath], last[kPath];     // pages of the segments
  int32_t end[kPath];                    // fours of tokens up to and with each (of these kPath)
  int32_t tokens[kPath];                 // that the row sees
  bool prompt[kPath];
};

// What a wave found in them: tokens, fours of tokens that the row sees, and such tokens that are not the prompt's.
struct Found {
  int64_t tokens, said;
  int32_t fours;
};

struct Row {
  const unsigned char* in;
  unsigned char* out;
  float rep, inv_rep, freq, pres, inv_t;
  const uint32_t* mask;                  // or NULL
};

// The last lane's value, in every lane.
__device__ __forceinline__ int64_t last_lane(int64_t v) {
  const unsigned lo = (unsigned)__builtin_amdgcn_readlane((int)v, 63);
  const int hi = __builtin_amdgcn_readlane((int)(v >> 32), 63);
  return (int64_t)(((uint64_t)(unsigned)hi << 32) | lo);
}

// Entries [at, at + kPath) of a path, by one wave; `start` is the position of their first token, and positions from
// `limit` on are not seen.  Entries behind the path's last are empty.
__device__ __forceinline__ Found take_path(const LogitArgs& a, const PathRange& range, int64_t at, int64_t start,
                                           int64_t limit, Path* p) {
  const int lane = threadIdx.x & 63;
  const int64_t e = range.first + at + lane;
  const SegRange s = e < range.end ? seg_range(a.g, a.g.path_segs[e]) : SegRange{0, 0, 0};
  const int64_t end = wave_scan(s.len);
  const int64_t room = limit - (start + end - s.len);
  const int32_t seen = room <= 0 ? 0 : s.len < room ? s.len : (int32_t)room;
  const int64_t fours = wave_scan((seen + 3LL) / 4);
  const bool prompt = at + lane < a.rules.prompt_segments;
  p->first[lane] = s.first;
  p->last[lane] = s.end;
  p->end[lane] = (int32_t)fours;
  p->tokens[lane] = seen;
  p->prompt[lane] = prompt;
  return {last_lane(end), last_lane(wave_scan(prompt ? 0 : seen)), __builtin_amdgcn_readlane((int)fours, 63)};
}

// The sum of a token's values in a list that is ascending by token.
__device__ __forceinline__ float sum_of(const int32_t* tokens, const float* values, int n, int v) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int mid = lo + (hi - lo) / 2;
    if (tokens[mid] < v) lo = mid + 1;
    else hi = mid;
  }
  float s = 0.f;
  for (; lo < n && tokens[lo] == v; ++lo) s += values[lo];
  return s;
}

// The same from an entry at or before its first.
struct alignas(8) Bias {
  int32_t token;
  float value;
};
__device__ __forceinline__ float sum_from(const Bias* list, int at, int n, int v) {
  float s = 0.f;
  for (; at < n; ++at) {
    const Bias b = list[at];
    if (b.token > v) break;
    s += b.token == v ? b.value : 0.f;
  }
  return s;
}

// Values as they are loaded: as many as are 16 bytes of the wider type.
template <class T, int E>
struct Values {
  static constexpr int W = E * sizeof(T) / 4;
  unsigned w[W];
  __device__ __forceinline__ void load(const unsigned char* row, int v) {
    typedef unsigned words __attribute__((ext_vector_type(W), aligned(2)));
    const words x = __builtin_nontemporal_load(reinterpret_cast<const words*>(row + (unsigned)v * (unsigned)sizeof(T)));
#pragma unroll
    for (int k = 0; k < W; ++k) w[k] = x[k];
  }
  __device__ __forceinline__ void load_some(const unsigned char* row, int v, int n) {
#pragma unroll
    for (int k = 0; k < W; ++k) w[k] = 0;
#pragma unroll
    for (int k = 0; k < E; ++k)
      if (k < n) {
        const T x = reinterpret_cast<const T*>(row)[v + k];
        if constexpr (sizeof(T) == 4) w[k] = __builtin_bit_cast(unsigned, x);
        else w[k / 2] |= (unsigned)__builtin_bit_cast(unsigned short, x) << (16 * (k & 1));
      }
  }
  __device__ __forceinline__ float at(int k) const {
    const unsigned u = sizeof(T) == 4 ? w[k] : k & 1 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16;
    return __builtin_bit_cast(float, u);
  }
};

template <class TO, int E>
__device__ __forceinline__ void store(unsigned char* row, int v, const float (&z)[E]) {
  unsigned char* const to = row + (unsigned)v * (unsigned)sizeof(TO);
#pragma unroll
  for (int i = 0; i < E * (int)sizeof(TO) / 16; ++i) {
    u32x4 w;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if constexpr (sizeof(TO) == 4) {
        w[k] = __builtin_bit_cast(unsigned, z[4 * i + k]);
      } else {
        typedef __bf16 two __attribute__((ext_vector_type(2)));
        w[k] = __builtin_bit_cast(unsigned, two{(__bf16)z[2 * k], (__bf16)z[2 * k + 1]});
      }
    }
    reinterpret_cast<u32x4_any*>(to)[i] = w;
  }
}

template <class TI, class TO>
__global__ __launch_bounds__(kThreads, 8) void k_logits(LogitArgs a) {
  // Values of a load; loads of a thread in flight together.
  constexpr int E = 16 / sizeof(TO), LOADS = sizeof(TI) == 4 ? 3 : 16 / E;
  extern __shared__ unsigned counts[];
  __shared__ Path path;
  __shared__ int64_t said_of, tokens_of;
  __shared__ int32_t fours_of;
  const int tid = threadIdx.x;
  // (A row's workgroups go round the XCDs.  Kept on one, with their neighbours', the path's tokens would come from one
  // L2, but a row of 152064 alone would have an eighth of the device: 10.4 us, not 6.1; 1024 rows 253, not 248.)
  const int64_t q = blockIdx.x, r = q / a.parts;
  const int lo0 = (int)(q % a.parts) * a.slice, hi0 = min(lo0 + a.slice, a.vocab);
  const int32_t b = a.row_branches ? a.row_branches[r] : (int32_t)r;
  if (b < 0 || b >= a.g.num_branches) return;
  int64_t limit = 0x7fffffff;
  if (a.row_positions) {
    const int32_t p = a.row_positions[r];
    if (p < 0) return;
    limit = (int64_t)p + 1;
  }
  Row row;
  row.in = a.in + r * a.in_stride * (int64_t)sizeof(TI);
  row.out = a.out + r * a.out_stride * (int64_t)sizeof(TO);
  Values<TI, E> x[LOADS];
  const auto fetch_one = [&](Values<TI, E>* to, int v, int hi) {
    if (v + E <= hi) to->load(row.in, v);
    else to->load_some(row.in, v, hi - v);
  };
  const auto fetch = [&](int v0, int hi) {
#pragma unroll
    for (int i = 0; i < LOADS; ++i) fetch_one(&x[i], v0 + E * (tid + i * kThreads), hi);
  };
  row.rep = a.rules.repetition ? a.rules.repetition[r] : 1.f;
  row.inv_rep = 1.f / row.rep;
  row.freq = a.rules.frequency ? a.rules.frequency[r] : 0.f;
  row.pres = a.rules.presence ? a.rules.presence[r] : 0.f;
  row.inv_t = a.rules.temperature ? 1.f / a.rules.temperature[r] : 1.f;
  row.mask = nullptr;
  if (a.rules.masks) {
    const int32_t m = a.rules.row_mask[r];
    if (m >= 0 && m < a.rules.num_masks) row.mask = a.rules.masks + m * a.rules.mask_words;
  }
  int64_t bias_first = 0, bias_end = 0;
  if (a.rules.bias_offsets) {
    const int64_t f = a.rules.bias_offsets[r], e = a.rules.bias_offsets[r + 1];
    bias_first = f < 0 ? 0 : f;
    bias_end = e < a.rules.num_bias ? e : a.rules.num_bias;
  }
  const bool biased = bias_first < bias_end;

  // Values of the first loads, counts of 0, and, by one wave, the path: before they are waited for.
  fetch(lo0, hi0);
  const bool flags = a.counted || biased;
  const auto clear = [&]() {
    typedef unsigned u32x4_lds __attribute__((ext_vector_type(4), aligned(16)));
    for (int i = tid; i < a.slice / 8 + 4; i += kThreads)
      reinterpret_cast<u32x4_lds*>(counts)[i] = u32x4_lds{0, 0, 0, 0};
  };
  if (flags) clear();
  PathRange range{0, 0};
  int64_t said = 0, chunks = 0;
  if (a.counted) {
    range = path_range(a.g, b);
    chunks = (range.end - range.first + kPath - 1) / kPath;
    if (tid < 64) {
      int64_t start = 0;
      Found f{0, 0, 0};
      for (int64_t c = 0; c < chunks; ++c) {
        f = take_path(a, range, c * kPath, start, limit, &path);
        said += f.said;
        start += f.tokens;
      }
      if (tid == 0) {
        said_of = said;
        tokens_of = f.tokens;
        fours_of = f.fours;
      }
    }
  }
  if (flags) __syncthreads();
  if (a.counted) said = said_of;
  const bool wide = said > 0x3fff;
  const int n_bias = (int)min(bias_end - bias_first, (int64_t)0x7fffffff);
  const bool near = biased && n_bias <= kBias;
  Bias* const near_list = reinterpret_cast<Bias*>(counts + a.slice / 2 + 16);
  unsigned short* const near_first = reinterpret_cast<unsigned short*>(near_list + kBias);

  // The slice [lo, hi), with counts of 16 or 32 bits.
  const auto pass = [&](auto wide_counts, int lo, int hi) {
    constexpr bool WIDE = decltype(wide_counts)::value;
    if (lo != lo0) {
      __syncthreads();
      clear();
      __syncthreads();
    }
    const auto note = [&](int v) {                   // (v: from lo on)
      if constexpr (WIDE) atomicAdd(&counts[v], 1u);
      else atomicAdd(&counts[v >> 1], 1u << ((v & 1) * 16));
    };
    const auto flag = [&](int v, unsigned n) {       // (n: as 16 bits hold it)
      if constexpr (WIDE) atomicOr(&counts[v], n << 16);
      else atomicOr(&counts[v >> 1], n << ((v & 1) * 16));
    };
    int64_t start = 0;
    for (int64_t c = 0; c < chunks; ++c) {
      if (chunks > 1) {
        __syncthreads();
        if (tid < 64) {
          const Found f = take_path(a, range, c * kPath, start, limit, &path);
          if (tid == 0) {
            tokens_of = f.tokens;
            fours_of = f.fours;
          }
        }
        __syncthreads();
      }
      // Four tokens a thread: a segment starts a page, so they lie in one.
      const int n = fours_of;
      for (int i0 = tid; i0 < n; i0 += kAhead * kThreads) {
        int32_t slot[kAhead], left[kAhead];          // of the first token; tokens that are seen
        bool prompt[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int i = i0 + k * kThreads;
          slot[k] = -1;
          left[k] = 0;
          prompt[k] = false;
          if (i < n) {
            int s = 0;                               // the first segment that ends behind i
            for (int d = kPath / 2; d > 0; d >>= 1)
              if (path.end[s + d - 1] <= i) s += d;
            const int32_t t = 4 * (i - (s ? path.end[s - 1] : 0));
            const int32_t page = page_of(a.g, path.first[s], path.last[s], t);
            slot[k] = page < 0 ? -1 : page * kPageTokens + (t & (kPageTokens - 1));
            left[k] = page < 0 ? 0 : path.tokens[s] - t;
            prompt[k] = path.prompt[s];
          }
        }
        i32x4_any id[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          if (slot[k] >= 0) id[k] = *reinterpret_cast<const i32x4_any*>(a.token_ids + slot[k]);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int32_t v = id[k][e];
            if (e < left[k] && v >= lo && v < hi) {
              if (prompt[k]) flag(v - lo, 0x8000u);
              else note(v - lo);
            }
          }
      }
      start += tokens_of;
    }
    if (biased)
      for (unsigned e = tid; e < (unsigned)n_bias; e += kThreads) {
        const int v = a.rules.bias_tokens[bias_first + e];
        if (near) near_list[e] = {v, a.rules.bias_values[bias_first + e]};
        if (v >= lo && v < hi) {
          flag(v - lo, 0x4000u);
          // The first of 32 tokens says where in the list theirs are.
          const int before = e ? a.rules.bias_tokens[bias_first + e - 1] : -1;
          if (near && (before < lo || before >> 5 != v >> 5)) near_first[(v - lo) >> 5] = (unsigned short)e;
        }
      }
    if (flags) __syncthreads();

    const auto work = [&](const Values<TI, E>& in, int v, int m) {
      unsigned allowed = 0;                        // (loaded ahead of the counts)
      if (row.mask) allowed = row.mask[v >> 5] >> (v & 31);
      float z[E];
#pragma unroll
      for (int k = 0; k < E; ++k) z[k] = in.at(k);
      if (flags) {
        constexpr int W = WIDE ? E : E / 2;
        const unsigned* const word = counts + (WIDE ? v - lo : (v - lo) >> 1);
        unsigned w[W], any = 0;
#pragma unroll
        for (int k = 0; k < W; ++k) any |= w[k] = word[k];
        // The tokens that have a bias, one after the other: few have.
        if (any & (WIDE ? 0x40000000u : 0x40004000u)) {
          unsigned some = 0;
#pragma unroll
          for (int k = 0; k < E; ++k)
            some |= w[WIDE ? k : k / 2] & (WIDE ? 0x40000000u : k & 1 ? 0x40000000u : 0x4000u) ? 1u << k : 0u;
          for (some &= (1u << m) - 1; some; some &= some - 1) {
            const int j = __builtin_ctz(some);
            const float bias =
                near ? sum_from(near_list, near_first[(v + j - lo) >> 5], n_bias, v + j)
                     : sum_of(a.rules.bias_tokens + bias_first, a.rules.bias_values + bias_first, n_bias, v + j);
#pragma unroll
            for (int k = 0; k < E; ++k) z[k] = j == k ? z[k] + bias : z[k];
          }
        }
        if (any && a.counted)
#pragma unroll
          for (int k = 0; k < E; ++k) {
            const unsigned u = w[WIDE ? k : k / 2];
            const float count = (float)(WIDE ? u & 0x3fffffffu : (u >> (16 * (k & 1))) & 0x3fffu);
            const float size = z[k] > 0.f ? row.inv_rep : row.rep;
            if (u & (WIDE ? 0xbfffffffu : 0xbfffu << (16 * (k & 1)))) z[k] *= size;
            // (not as products with 0: an infinite penalty bans what came and nothing else)
            if (count > 0.f) z[k] = __builtin_fmaf(-row.freq, count, z[k]) - row.pres;
          }
      }
#pragma unroll
      for (int k = 0; k < E; ++k) z[k] *= row.inv_t;
      if (row.mask) {
#pragma unroll
        for (int k = 0; k < E; ++k) {
          const unsigned keep = (unsigned)((int)(allowed << (31 - k)) >> 31);
          z[k] = __builtin_bit_cast(float, (__builtin_bit_cast(unsigned, z[k]) & keep) | (0xff800000u & ~keep));
        }
      }
      if (m == E) {
        store<TO, E>(row.out, v, z);
      } else {
#pragma unroll
        for (int k = 0; k < E; ++k)
          if (k < m) reinterpret_cast<TO*>(row.out)[v + k] = (TO)z[k];
      }
    };
    if constexpr (WIDE) {
      // (rare: one load at a time)
      for (int v = lo + E * tid; v < hi; v += E * kThreads) {
        fetch_one(&x[0], v, hi);
        work(x[0], v, min(E, hi - v));
      }
    } else {
      for (int v0 = lo; v0 < hi; v0 += E * LOADS * kThreads) {
        if (v0 != lo) fetch(v0, hi);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
          const int v = v0 + E * (tid + i * kThreads), m = min(E, hi - v);
          if (m > 0) work(x[i], v, m);
        }
      }
    }
  };
  if (!wide) {
    pass(std::false_type{}, lo0, hi0);
  } else {
    const int step = (a.slice / 2 + 31) / 32 * 32;
    for (int lo = lo0; lo < hi0; lo += step) pass(std::true_type{}, lo, min(lo + step, hi0));
  }
}

}  // namespace

int64_t plan_logits(LogitArgs* a) {
  // Slices of a row: as many as its counts need, and so many that a few rows fill the device.  (128 rows of 50001: 512
  // workgroups 14.6 us, 1024 20.0; one row is as fast in 8, 16 or 32.)
  const int64_t largest = a->rules.bias_offsets ? kMaxSliceBiased : kMaxSlice;
  const int64_t least = (a->vocab + largest - 1) / largest, most = (a->vocab + 2047) / 2048;
  int64_t parts = (512 + a->rows - 1) / a->rows;
  parts = parts < least ? least : parts > most ? most : parts;
  a->slice = (int32_t)(((a->vocab + parts - 1) / parts + 31) / 32 * 32);
  a->parts = (a->vocab + a->slice - 1) / a->slice;
  return (int64_t)a->rows * a->parts * kThreads;
}

hipError_t launch_logits(const LogitArgs& a, bool in_f32, bool out_f32, hipStream_t stream) {
  const size_t lds = (size_t)a.slice * 2 + 64 + (a.rules.bias_offsets ? kBias * 8 + a.slice / 16 : 0);
  const dim3 g((unsigned)(a.rows * a.parts)), t(kThreads);
  if (in_f32) hipLaunchKernelGGL((k_logits<float, float>), g, t, lds, stream, a);
  else if (out_f32) hipLaunchKernelGGL((k_logits<__bf16, float>), g, t, lds, stream, a);
  else hipLaunchKernelGGL((k_logits<__bf16, __bf16>), g, t, lds, stream, a);
  return hipGetLastError();
}

}  // namespace ga
