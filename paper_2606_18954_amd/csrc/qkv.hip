// Queries, keys and values of a step's tokens: norm of each head, rotation by the token's position, and the
// write into rows (q) and the pool's pages (k, v), in one pass over the projection's rows.
//
// A head of D values x: y = x rs w with rs = 1 / sqrt(mean x^2 + eps); a pair (a, b) of its channels turns to
// (a cos - b sin, b cos + a sin).  With C = cos (1 for a channel that does not turn) and S = -sin, sin (0) the
// channel c with partner c' is rs (x[c] w[c] C[c] + x[c'] w[c'] S[c]): the weights are folded into C and S once
// for all heads of a token, and a head costs two products a channel and the sum of its squares.
//
// 8 channels a lane, 16 bytes of bf16, so D / 8 lanes hold a head and a wave's load is a group of 512 / D heads.  A
// workgroup takes one token, or four where there are many.  A token's rotary_dim / 2 angles are a wave's lanes', one
// each (float64 product and remainder in turns, then sine and cosine of half turns in float32); they and the weights
// go through LDS.  No table of angles is read, and positions go up to 2^31 - 1 (those below 0 are padding).  The
// groups are dealt to the waves in units, three of q or one of k with the same heads of v, so that all loads of a
// unit go out before its first store: a wave that waits for a load behind a store waits for the store too.
//
// Memory bounds it: 32768 tokens of 40 + 2 x 8 heads of 128, bf16, 940 MB in 170-187 us = 5.0-5.5 TB/s by the card (a
// plain copy of as many bytes runs at 5.3), without norms or rotation the same; of 28 + 2 x 4 heads 105-119 us =
// 5.1-5.8 TB/s; a step's 1024 tokens 5.5-6.3 us, one token 3.1 (replayed from a graph).  Counters: reads and writes
// are what the rows hold, the vector unit is busy 37% of the time.  Before: one group after the other with a load
// ahead, angles exchanged between lanes and made by every wave, 226 us and 20; five groups of q a unit 192 and 6.9
// (more registers, five waves per SIMD).
#include "mxfp4.hpp"
#include "pool_load.hpp"
#include "step_internal.hpp"

namespace ga {
namespace {

constexpr int kWaves = 4;          // of a workgroup

// Groups of heads that a wave takes at once, all of their loads ahead of the first store: of q, or of k and of v.
// (Two to five of q, one or two of k and v: 185 to 192 us for the 32768 tokens above; float32 two or three: the same.)
template <class T>
struct Units {
  static constexpr int Q = sizeof(T) == 4 ? 2 : 3, KV = 1;
};

__device__ __forceinline__ float bf16_lo(unsigned w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float bf16_hi(unsigned w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
__device__ __forceinline__ unsigned bf16_pair(float lo, float hi) {
  const bf16x2_t p = {(__bf16)lo, (__bf16)hi};
  return __builtin_bit_cast(unsigned, p);
}

// Eight channels as they lie in memory.
template <class T>
struct Raw {
  static constexpr int W = sizeof(T) * 2;            // words
  unsigned w[W];
  __device__ __forceinline__ void load(const unsigned char* p) {
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
      const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p) + i);
#pragma unroll
      for (int k = 0; k < 4; ++k) w[4 * i + k] = v[k];
    }
  }
  __device__ __forceinline__ void store(unsigned char* p) const {
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
      const u32x4 v = {w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
      reinterpret_cast<u32x4*>(p)[i] = v;
    }
  }
  __device__ __forceinline__ void to(float (&x)[8]) const {
#pragma unroll
    for (int k = 0; k < 8; ++k)
      x[k] = sizeof(T) == 4 ? __builtin_bit_cast(float, w[k]) : k & 1 ? bf16_hi(w[k / 2]) : bf16_lo(w[k / 2]);
  }
  __device__ __forceinline__ void from(const float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < W; ++i)
      w[i] = sizeof(T) == 4 ? __builtin_bit_cast(unsigned, x[i]) : bf16_pair(x[2 * i], x[2 * i + 1]);
  }
};

template <int CTRL>
__device__ __forceinline__ float from_lane(float x) {
  return __builtin_bit_cast(
      float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, x), CTRL, 0xf, 0xf, true));
}
// The sum over the D / 8 lanes of a head, in each of them: two quad permutations, then (sums of quads being the
// same in a quad) the mirror image in 8 and in 16 lanes.
template <int D>
__device__ __forceinline__ float head_sum(float s) {
  s += from_lane<0xB1>(s);
  s += from_lane<0x4E>(s);
  s += from_lane<0x141>(s);
  if constexpr (D == 128) s += from_lane<0x140>(s);
  return s;
}

// What the heads of a kind are made with: cosine and sine of this lane's channels (the sine with its sign), weights
// folded in.
struct Turn {
  float c[8], s[8];
  bool normed;
};

template <int D, class T, bool FP4, bool PAIRS>
__global__ __launch_bounds__(64 * kWaves) void k_qkv(QkvArgs a) {
  constexpr int LPH = D / 8, HPG = 64 / LPH, SZ = (int)sizeof(T), ROW = D * SZ;
  using U = Units<T>;
  __shared__ __align__(16) float cosines[kWaves][64], sines[kWaves][64], weights[2 * D + 8];   // (and eight zeros)
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int64_t first = (int64_t)blockIdx.x * a.tokens;
  const int half = a.half;
  const int g = lane / LPH, c = 8 * (lane % LPH);
  const bool turns = c < 2 * half;
  const int shift = c < half ? half : -half;
  const int partner = PAIRS || !turns ? lane : lane + shift / 8;
  const int pc = PAIRS || !turns ? c : c + shift;
  // Groups of heads, and units of a token: uq of queries, then those of keys and values.
  const int nq = (a.Hq + HPG - 1) / HPG, nk = (a.Hkv + HPG - 1) / HPG;
  const int units = a.q_units + (nk + U::KV - 1) / U::KV;

  // Positions and words first, while nothing is written yet: they come through the scalar cache.
  int32_t positions[kWaves], words[kWaves];
#pragma unroll
  for (int i = 0; i < kWaves; ++i) {
    const bool there = i < a.tokens && first + i < a.n;
    positions[i] = there ? a.positions[first + i] : -1;
    words[i] = there ? a.words[first + i] : -1;
  }
  for (int i = threadIdx.x; i < 2 * D; i += 64 * kWaves)
    if (const float* const w = i < D ? a.weight[0] : a.weight[1]) weights[i] = w[i & (D - 1)];
  if (threadIdx.x < 8) weights[2 * D + threadIdx.x] = 0.f;
  if (wave < a.tokens && lane < half) {
    const int32_t pos = first + wave < a.n ? a.positions[first + wave] : 0;
    const double t = (double)pos * (a.inv_freq[lane] * 0.15915494309189533577);
    float sn, cs;
    sincospif((float)(2.0 * (t - rint(t))), &sn, &cs);
    cosines[wave][lane] = cs * a.scale;
    sines[wave][lane] = sn * a.scale;
  }
  __syncthreads();

  // Eight channels of head h of a token's rows (lanes behind the last head read that one's again).
  const auto fetch = [&](int kind, int64_t token, int h, int heads, Raw<T>* r) {
    const unsigned char* const row = a.src[kind] + token * a.stride[kind];
    r->load(row + (unsigned)(min(h, heads - 1) * ROW + c * SZ));
  };
  const auto turn_of = [&](int at, int kind, bool normed, Turn* t) {
    // (what is read for channels that do not turn is not used)
    const int angle = (PAIRS ? c >> 1 : c < half ? c : c - half) & (PAIRS ? 60 : 56);
#pragma unroll
    for (int k = 0; k < 8; k += PAIRS ? 2 : 1) {
      const bool on = PAIRS ? c + k < 2 * half : turns;
      const float o = cosines[at][angle + (PAIRS ? k / 2 : k)], s = sines[at][angle + (PAIRS ? k / 2 : k)];
      t->c[k] = on ? o : 1.f;
      t->s[k] = !on ? 0.f : PAIRS || c < half ? -s : s;
      if constexpr (PAIRS) {
        t->c[k + 1] = t->c[k];
        t->s[k + 1] = -t->s[k];
      }
    }
    t->normed = normed;
    if (normed) {
      const float* const w = weights + kind * D;
      const float* const partners = turns ? w + pc : weights + 2 * D;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        t->c[k] *= w[c + k];
        if constexpr (PAIRS) t->s[k] *= c + k < 2 * half ? w[c + (k ^ 1)] : 0.f;
        else t->s[k] *= partners[k];
      }
    }
  };
  const auto made = [&](const Raw<T>& r, const Turn& t) {
    // Partners; a channel that does not turn takes nothing from another, not its infinity either.
    float x[8], p[8], z[8];
    r.to(x);
    if constexpr (PAIRS) {
#pragma unroll
      for (int k = 0; k < 8; ++k) p[k] = c + k < 2 * half ? x[k ^ 1] : 0.f;
    } else {
      Raw<T> o;
#pragma unroll
      for (int k = 0; k < Raw<T>::W; ++k) {
        const unsigned w = (unsigned)__shfl((int)r.w[k], partner);
        o.w[k] = turns ? w : 0;
      }
      o.to(p);
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) z[k] = x[k] * t.c[k] + p[k] * t.s[k];
    if (t.normed) {
      float s = 0.f;
#pragma unroll
      for (int k = 0; k < 8; ++k) s += x[k] * x[k];
      float mean = head_sum<D>(s) * (1.f / D) + a.eps;
      // Squares that leave float32's range (or are subnormal, which the root takes as 0): the heads that have them
      // once more, their values times a power of two.
      const bool low = mean < 0x1p-100f, leaves = low || !(mean < __builtin_inff());
      if (__any(leaves)) {
        const float by = !leaves ? 1.f : low ? 0x1p96f : 0x1p-96f;
        s = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          x[k] *= by;
          z[k] = x[k] * t.c[k] + p[k] * by * t.s[k];
          s += x[k] * x[k];
        }
        mean = head_sum<D>(s) * (1.f / D) + a.eps * by * by;
      }
      const float rs = __builtin_amdgcn_rsqf(mean);
#pragma unroll
      for (int k = 0; k < 8; ++k) z[k] *= rs;
    }
    Raw<T> y;
    y.from(z);
    return y;
  };
  // Head h of a token's K or V to its slot.
  const auto store_kv = [&](const Raw<T>& y, int32_t word, int h, bool value) {
    if constexpr (!FP4) {
      unsigned char* const page =
          a.pool + ((int64_t)(word >> 4) * a.Hkv * (2 * kPageTokens) + ((value ? kPageTokens : 0) + (word & 15))) * ROW;
      if (h < a.Hkv) y.store(page + (unsigned)(h * (2 * kPageTokens * ROW) + c * SZ));
    } else {
      unsigned code, byte;
      const unsigned w[4] = {y.w[0], y.w[1], y.w[2], y.w[3]};
      fp4_round(w, &code, &byte);
      if (h < a.Hkv) {
        unsigned char* const dst = a.pool + ((int64_t)(word >> 4) * a.Hkv + h) * Fp4<D>::PAGE;
        store_codes<D>(dst, word & 15, c, value, code);
        if ((c & 31) == 0) dst[fp4_scale<D>(word & 15, c, value)] = (unsigned char)byte;
      }
    }
  };

  // The units of the workgroup's tokens in turn; every wave takes each kind of unit in its turns.
  for (int u = (int)(blockIdx.y * kWaves) + wave; u < units * a.tokens; u += kWaves * (int)gridDim.y) {
    const int at = u / units;
    const int64_t token = first + at;
    if (token >= a.n) break;
    const int unit = (u - at * units + at) % units;
    const int32_t pos = at == 0 ? positions[0] : at == 1 ? positions[1] : at == 2 ? positions[2] : positions[3];
    const int32_t word = at == 0 ? words[0] : at == 1 ? words[1] : at == 2 ? words[2] : words[3];
    if (pos < 0) continue;
    Raw<T> r[U::Q > 2 * U::KV ? U::Q : 2 * U::KV];
    Turn t;
    if (unit < a.q_units) {
      const int i0 = unit * a.q_groups, n = min(a.q_groups, nq - i0);
#pragma unroll
      for (int i = 0; i < U::Q; ++i)
        if (i < n) fetch(0, token, (i0 + i) * HPG + g, a.Hq, &r[i]);
      turn_of(at, 0, a.weight[0] != nullptr, &t);
#pragma unroll
      for (int i = 0; i < U::Q; ++i)
        if (i < n) {
          const int h = (i0 + i) * HPG + g;
          const Raw<T> y = made(r[i], t);
          if (h < a.Hq) y.store(a.q_out + token * (a.Hq * ROW) + (unsigned)(h * ROW + c * SZ));
        }
    } else if (word >= 0 && (int64_t)word < a.num_slots) {
      const int i0 = (unit - a.q_units) * U::KV, n = min(U::KV, nk - i0);
#pragma unroll
      for (int i = 0; i < U::KV; ++i)
        if (i < n) {
          fetch(1, token, (i0 + i) * HPG + g, a.Hkv, &r[i]);
          fetch(2, token, (i0 + i) * HPG + g, a.Hkv, &r[U::KV + i]);
        }
      turn_of(at, 1, a.weight[1] != nullptr, &t);
#pragma unroll
      for (int i = 0; i < U::KV; ++i)
        if (i < n) {
          const int h = (i0 + i) * HPG + g;
          store_kv(made(r[i], t), word, h, false);
          store_kv(r[U::KV + i], word, h, true);
        }
    }
  }
}

template <int D, class T, bool FP4>
void launch(const QkvArgs& a, dim3 grid, bool pairs, hipStream_t stream) {
  if (pairs) hipLaunchKernelGGL((k_qkv<D, T, FP4, true>), grid, dim3(64 * kWaves), 0, stream, a);
  else hipLaunchKernelGGL((k_qkv<D, T, FP4, false>), grid, dim3(64 * kWaves), 0, stream, a);
}
template <int D>
void launch(const QkvArgs& a, dim3 grid, int dtype, bool pairs, hipStream_t stream) {
  if (dtype == GA_F32) launch<D, float, false>(a, grid, pairs, stream);
  else if (dtype == GA_BF16) launch<D, __bf16, false>(a, grid, pairs, stream);
  else launch<D, __bf16, true>(a, grid, pairs, stream);
}

}  // namespace

hipError_t launch_qkv(const QkvArgs& args, int dim, int dtype, bool interleaved, hipStream_t stream) {
  QkvArgs a = args;
  const int group = 512 / dim, nq = (a.Hq + group - 1) / group, nk = (a.Hkv + group - 1) / group;
  const int q = dtype == GA_F32 ? Units<float>::Q : Units<__bf16>::Q;
  const int kv = dtype == GA_F32 ? Units<float>::KV : Units<__bf16>::KV;
  a.q_units = (nq + q - 1) / q;
  a.q_groups = (nq + a.q_units - 1) / a.q_units;
  // Four tokens a workgroup where there are enough of them to fill the device, else one, its units on as many
  // workgroups as they need.  One and four, us: 28 + 2 x 4 heads of 128, bf16, 1024 tokens 6.5 and 9.4, 2048 11.1 and
  // 12.2, 3000 14.0 and 13.8, 4096 18.3 and 16.3, 8192 29.9 and 28.4, but 16384 58.5 and 61.5, 32768 110.5 and 118.2
  // (40 + 2 x 8: 181 and 186); 12 + 2 x 12 of 64 2048 8.2 and 8.3, 4096 13.2 and 11.1, 16384 40.4 and 30.5; 16 + 2 x
  // 2 of 64, float32, 2048 8.4 and 7.5, 16384 43.5 and 35.3.
  a.tokens = a.n >= 4096 ? kWaves : 1;
  const int units = a.q_units + (nk + kv - 1) / kv;
  const dim3 grid((unsigned)((a.n + a.tokens - 1) / a.tokens),
                  (unsigned)(a.tokens > 1 ? 1 : (units + kWaves - 1) / kWaves));
  if (dim == 64) launch<64>(a, grid, dtype, interleaved, stream);
  else launch<128>(a, grid, dtype, interleaved, stream);
  return hipGetLastError();
}

}  // namespace ga
