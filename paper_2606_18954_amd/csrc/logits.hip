// Logits of a step's rows through penalties, biases, temperature and masks, in one pass over them.
//
// The penalties of a row go by the tokens of its branch's path.  Most of a vocabulary's tokens are not among
// them, so what a row needs is a sparse count, which a dense array per row in memory would turn into as many
// bytes again as the logits.  Here a workgroup takes a slice of a row's vocabulary, counts the path's tokens that
// fall into it in LDS, and streams the slice past the counts; memory carries the logits, once each way.
//
// Counts are 16 bits a token of the slice: 14 bits of count, one for a token with a bias, one for a token of the
// prompt (which counts for the repetition penalty alone).  Rows that could count further than 14 bits take the
// slice in two halves with 32 bits a token.  Every workgroup of a row reads the whole path (4 bytes a token,
// from L2: rows of one XCD are neighbours, whose paths share segments).
// Biases: the flag says that there is one, and its value is looked up (the row's list is ascending).
// Memory bounds it: a row of V values of four bytes moves 8 V.
#include "pool_load.hpp"
#include "step_internal.hpp"

namespace ga {
namespace {

constexpr int kThreads = 512;
constexpr int kPath = 64;          // segments of a path taken at once
constexpr int kAhead = 4;          // tokens of a thread whose loads are in flight together
constexpr int kMaxSlice = 19456;   // 2 bytes a token: 38 KB, four workgroups a CU

typedef unsigned u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

struct Path {
  int64_t first[kPath], last[kPath];     // pages of the segments
  int64_t end[kPath];                    // tokens of the path up to and with each (of these kPath)
  bool prompt[kPath];
};

// What a wave found in them: tokens, and how many of them before a position are not the prompt's.
struct Found {
  int64_t tokens, said;
};

template <class TI, class TO>
struct Row {
  const unsigned char* in;
  unsigned char* out;
  float rep, freq, pres, inv_t;
  const uint32_t* mask;                  // or NULL
  int64_t bias_first, bias_end;
};

__device__ __forceinline__ int64_t wave_sum(int64_t v) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) v += __shfl_xor(v, d);
  return v;
}

// Entries [at, at + kPath) of a path, by one wave; `start` is the position of their first token.  Entries behind the
// path's last are empty.
__device__ __forceinline__ Found take_path(const LogitArgs& a, const PathRange& range, int64_t at, int64_t start,
                                           int64_t limit, Path* p) {
  const int lane = threadIdx.x & 63;
  const int64_t e = range.first + at + lane;
  const int n = (int)(range.end - range.first - at < kPath ? range.end - range.first - at : kPath);
  const SegRange s = lane < n ? seg_range(a.g, a.g.path_segs[e]) : SegRange{0, 0, 0};
  int64_t end = s.len;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int64_t x = __shfl_up(end, d);
    if (lane >= d) end += x;
  }
  const bool prompt = at + lane < a.rules.prompt_segments;
  p->first[lane] = s.first;
  p->last[lane] = s.end;
  p->end[lane] = end;
  p->prompt[lane] = prompt;
  const int64_t room = limit - (start + end - s.len);
  return {__shfl(end, 63), wave_sum(prompt || room <= 0 ? 0 : s.len < room ? s.len : room)};
}

template <class TI, class TO>
__device__ __forceinline__ float bias_of(const LogitArgs& a, const Row<TI, TO>& row, int v) {
  int64_t lo = row.bias_first, hi = row.bias_end;
  while (lo < hi) {
    const int64_t mid = lo + (hi - lo) / 2;
    if (a.rules.bias_tokens[mid] < v) lo = mid + 1;
    else hi = mid;
  }
  float s = 0.f;
  for (; lo < row.bias_end && a.rules.bias_tokens[lo] == v; ++lo) s += a.rules.bias_values[lo];
  return s;
}

template <class TO>
__device__ __forceinline__ void put(unsigned char* out, int64_t v, float z) {
  reinterpret_cast<TO*>(out)[v] = (TO)z;
}

template <class TI, class TO>
__global__ __launch_bounds__(kThreads) void k_logits(LogitArgs a) {
  constexpr int E = 16 / sizeof(TI);                 // values of a load
  extern __shared__ unsigned counts[];
  __shared__ Path path;
  __shared__ int64_t said_of, tokens_of;
  const int tid = threadIdx.x;
  // Workgroups go round the 8 XCDs: a row's stay on one, with its neighbours'.
  const int64_t q = blockIdx.x / 8;
  const int64_t r = (int64_t)(blockIdx.x % 8) * a.rows_per_xcd + q / a.parts;
  if (q / a.parts >= a.rows_per_xcd || r >= a.rows) return;
  const int lo0 = (int)(q % a.parts) * a.slice, hi0 = min(lo0 + a.slice, a.vocab);
  const int32_t b = a.row_branches ? a.row_branches[r] : (int32_t)r;
  if (b < 0 || b >= a.g.num_branches) return;
  int64_t limit = 1LL << 62;
  if (a.row_positions) {
    const int32_t p = a.row_positions[r];
    if (p < 0) return;
    limit = (int64_t)p + 1;
  }
  Row<TI, TO> row;
  row.in = a.in + r * a.in_stride * (int64_t)sizeof(TI);
  row.out = a.out + r * a.out_stride * (int64_t)sizeof(TO);
  row.rep = a.rules.repetition ? a.rules.repetition[r] : 1.f;
  row.freq = a.rules.frequency ? a.rules.frequency[r] : 0.f;
  row.pres = a.rules.presence ? a.rules.presence[r] : 0.f;
  row.inv_t = a.rules.temperature ? 1.f / a.rules.temperature[r] : 1.f;
  row.mask = nullptr;
  if (a.rules.masks) {
    const int32_t m = a.rules.row_mask[r];
    if (m >= 0 && m < a.rules.num_masks) row.mask = a.rules.masks + m * a.rules.mask_words;
  }
  row.bias_first = row.bias_end = 0;
  if (a.rules.bias_offsets) {
    const int64_t f = a.rules.bias_offsets[r], e = a.rules.bias_offsets[r + 1];
    row.bias_first = f < 0 ? 0 : f;
    row.bias_end = e < a.rules.num_bias ? e : a.rules.num_bias;
  }
  const bool biased = row.bias_first < row.bias_end;

  PathRange range{0, 0};
  int64_t said = 0, chunks = 0;
  if (a.counted) {
    range = path_range(a.g, b);
    chunks = range.end > range.first ? (range.end - range.first + kPath - 1) / kPath : 0;
    if (tid < 64) {
      int64_t start = 0;
      Found f{0, 0};
      for (int64_t c = 0; c < chunks; ++c) {
        f = take_path(a, range, c * kPath, start, limit, &path);
        said += f.said;
        start += f.tokens;
      }
      if (tid == 0) {
        said_of = said;
        tokens_of = f.tokens;
      }
    }
    __syncthreads();
    said = said_of;
  }
  const bool wide = said > 0x3fff;
  const bool flags = a.counted || biased;

  for (int half = 0; half < (wide ? 2 : 1); ++half) {
    const int step = wide ? (a.slice / 2 + 31) / 32 * 32 : a.slice;
    const int lo = lo0 + half * step, hi = half == 0 ? min(lo0 + step, hi0) : hi0;
    if (lo >= hi) break;
    if (flags) {
      if (half) __syncthreads();
      const int words = wide ? hi - lo : (hi - lo + 1) / 2;
      for (int i = tid; i < words; i += kThreads) counts[i] = 0;
      __syncthreads();
    }
    const auto note = [&](int v) {
      if (wide) atomicAdd(&counts[v - lo], 1u);
      else atomicAdd(&counts[(v - lo) >> 1], 1u << (((v - lo) & 1) * 16));
    };
    const auto flag = [&](int v, unsigned n) {       // (as 16 bits hold it)
      if (wide) atomicOr(&counts[v - lo], n << 16);
      else atomicOr(&counts[(v - lo) >> 1], n << (((v - lo) & 1) * 16));
    };
    int64_t start = 0;
    for (int64_t c = 0; c < chunks; ++c) {
      if (chunks > 1) {
        __syncthreads();
        if (tid < 64) {
          const Found f = take_path(a, range, c * kPath, start, limit, &path);
          if (tid == 0) tokens_of = f.tokens;
        }
        __syncthreads();
      }
      const int64_t tokens = tokens_of, left = limit - start;
      const int64_t n = tokens < left ? tokens : left;
      for (int64_t i0 = tid; i0 < n; i0 += kAhead * kThreads) {
        int32_t slot[kAhead];
        bool prompt[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          const int64_t i = i0 + k * kThreads;
          slot[k] = -1;
          prompt[k] = false;
          if (i < n) {
            int s = 0;                               // the first segment that ends behind i
            for (int d = kPath / 2; d > 0; d >>= 1)
              if (path.end[s + d - 1] <= i) s += d;
            const int32_t t = (int32_t)(i - (s ? path.end[s - 1] : 0));
            const int32_t page = page_of(a.g, path.first[s], path.last[s], t);
            slot[k] = page < 0 ? -1 : page * kPageTokens + (t & (kPageTokens - 1));
            prompt[k] = path.prompt[s];
          }
        }
        int32_t id[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) id[k] = slot[k] >= 0 ? a.token_ids[slot[k]] : -1;
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          if (id[k] >= lo && id[k] < hi) {
            if (prompt[k]) flag(id[k], 0x8000u);
            else note(id[k]);
          }
      }
      start += tokens;
    }
    if (biased)
      for (int64_t e = row.bias_first + tid; e < row.bias_end; e += kThreads) {
        const int v = a.rules.bias_tokens[e];
        if (v >= lo && v < hi) flag(v, 0x4000u);
      }
    if (flags) __syncthreads();

    const auto rule = [&](float z, unsigned word, int v) {   // word: as 32 bits hold it
      const unsigned count = word & 0x3fffffffu;
      if (word & 0x40000000u) z += bias_of(a, row, v);
      if (word & 0xbfffffffu) z = z > 0.f ? z / row.rep : z * row.rep;
      if (count) z -= row.freq * (float)count + row.pres;
      return z;
    };
    const auto wide_word = [](unsigned w16) { return ((w16 & 0xc000u) << 16) | (w16 & 0x3fffu); };
    for (int v0 = lo + E * tid; v0 < hi; v0 += E * kThreads) {
      const int m = min(E, hi - v0);
      float z[E];
      if (m == E) {
        const u32x4 w = *reinterpret_cast<const u32x4_any*>(row.in + (int64_t)v0 * sizeof(TI));
#pragma unroll
        for (int k = 0; k < E; ++k) {
          // (a vector's element is no object that bit_cast could take)
          const unsigned u = sizeof(TI) == 4 ? w[k] : k & 1 ? w[k / 2] & 0xffff0000u : w[k / 2] << 16;
          z[k] = __builtin_bit_cast(float, u);
        }
      } else {
#pragma unroll
        for (int k = 0; k < E; ++k) z[k] = k < m ? (float)reinterpret_cast<const TI*>(row.in)[v0 + k] : 0.f;
      }
      unsigned allowed = ~0u;
      if (row.mask) allowed = row.mask[v0 >> 5] >> (v0 & 31);
      if (flags) {
        const int at = v0 - lo;
        unsigned w[E], any = 0;
#pragma unroll
        for (int k = 0; k < E; ++k) {
          if (wide) w[k] = k < m ? counts[at + k] : 0;
          else w[k] = k < m ? (counts[(at + k) >> 1] >> ((k & 1) * 16)) & 0xffffu : 0;
          any |= w[k];
        }
        if (any)
#pragma unroll
          for (int k = 0; k < E; ++k)
            if (w[k]) z[k] = rule(z[k], wide ? w[k] : wide_word(w[k]), v0 + k);
      }
#pragma unroll
      for (int k = 0; k < E; ++k) {
        z[k] *= row.inv_t;
        if (!((allowed >> k) & 1)) z[k] = -__builtin_inff();
      }
      if (m == E) {
        if constexpr (sizeof(TO) == 4) {
#pragma unroll
          for (int i = 0; i < E / 4; ++i) {
            u32x4 w;
#pragma unroll
            for (int k = 0; k < 4; ++k) w[k] = __builtin_bit_cast(unsigned, z[4 * i + k]);
            reinterpret_cast<u32x4_any*>(row.out + (int64_t)v0 * 4)[i] = w;
          }
        } else {
          u32x4 w;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            typedef __bf16 two __attribute__((ext_vector_type(2)));
            w[k] = __builtin_bit_cast(unsigned, two{(__bf16)z[2 * k], (__bf16)z[2 * k + 1]});
          }
          *reinterpret_cast<u32x4_any*>(row.out + (int64_t)v0 * 2) = w;
        }
      } else {
#pragma unroll
        for (int k = 0; k < E; ++k)
          if (k < m) put<TO>(row.out, v0 + k, z[k]);
      }
    }
  }
}

}  // namespace

hipError_t launch_logits(const LogitArgs& args, bool in_f32, bool out_f32, hipStream_t stream) {
  LogitArgs a = args;
  // Slices of a row: as many as its counts need, and so many that a few rows fill the device.
  const int64_t least = (a.vocab + kMaxSlice - 1) / kMaxSlice, most = (a.vocab + 2047) / 2048;
  int64_t parts = (1024 + a.rows - 1) / a.rows;
  parts = parts < least ? least : parts > most ? most : parts;
  a.slice = (int32_t)(((a.vocab + parts - 1) / parts + 31) / 32 * 32);
  a.parts = (a.vocab + a.slice - 1) / a.slice;
  a.rows_per_xcd = (a.rows + 7) / 8;
  const int64_t grid = (int64_t)a.rows_per_xcd * 8 * a.parts;
  if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
  const size_t lds = (size_t)a.slice * 2 + 64;
  const dim3 g((unsigned)grid), t(kThreads);
  if (in_f32) hipLaunchKernelGGL((k_logits<float, float>), g, t, lds, stream, a);
  else if (out_f32) hipLaunchKernelGGL((k_logits<__bf16, float>), g, t, lds, stream, a);
  else hipLaunchKernelGGL((k_logits<__bf16, __bf16>), g, t, lds, stream, a);
  return hipGetLastError();
}

}  // namespace ga
