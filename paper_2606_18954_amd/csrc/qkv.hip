// Queries, keys and values of a step's tokens: norm of each head, rotation by the token's position, and the
// write into rows (q) and the pool's pages (k, v), in one pass over the projection's rows.
//
// A head of D values x: y = x rs w with rs = 1 / sqrt(mean x^2 + eps); a pair (a, b) of its channels turns to
// (a cos - b sin, b cos + a sin).  With C = cos (1 for a channel that does not turn) and S = -sin, sin (0) the
// channel c with partner c' is rs (x[c] w[c] C[c] + x[c'] w[c'] S[c]): the weights are folded into C and S once
// for all heads of a token, and a head costs two products a channel and the sum of its squares.
//
// A wave takes a token and some groups of its heads; 8 channels a lane, 16 bytes of bf16, so D / 8 lanes hold a
// head and 512 / D heads are a group.  The token's rotary_dim / 2 angles are the lanes', one each (float64 product
// and remainder in turns, then sine and cosine of half turns in float32); the lanes fetch those of their channels
// from each other.  No table of angles is read, and positions may be any int32.  The next group's loads go out
// before the present one is worked on.
#include "mxfp4.hpp"
#include "pool_load.hpp"
#include "step_internal.hpp"

namespace ga {
namespace {

constexpr int kWaves = 4;          // of a workgroup

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
    for (int i = 0; i < W / 4; ++i)
      reinterpret_cast<u32x4*>(p)[i] = u32x4{w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
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

template <int D, class T, bool FP4, bool PAIRS>
__global__ __launch_bounds__(64 * kWaves) void k_qkv(QkvArgs a) {
  constexpr int LPH = D / 8, HPG = 64 / LPH, ROW = D * (int)sizeof(T);
  const int lane = threadIdx.x & 63;
  const unsigned task = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * kWaves + (threadIdx.x >> 6)));
  const unsigned token = task / (unsigned)a.parts;
  if (token >= (unsigned)a.n) return;
  const int32_t pos = a.positions[token];
  if (pos < 0) return;
  const int32_t word = a.words[token];
  const bool stored = word >= 0 && (int64_t)word < a.num_slots;
  const int g = lane / LPH, c = 8 * (lane % LPH);
  const int nq = (a.Hq + HPG - 1) / HPG, nk = (a.Hkv + HPG - 1) / HPG;
  int it = (int)(task - token * a.parts) * a.per;
  const int end = min(it + a.per, stored ? nq + 2 * nk : nq);
  if (it >= end) return;

  auto kind_of = [&](int i) { return i < nq ? 0 : i < nq + nk ? 1 : 2; };
  auto head_of = [&](int i, int kind) { return (i - (kind == 0 ? 0 : kind == 1 ? nq : nq + nk)) * HPG + g; };
  auto fetch = [&](int i, Raw<T>* r) {
    const int kind = kind_of(i), h = head_of(i, kind);
    if (h < (kind == 0 ? a.Hq : a.Hkv))
      r->load(a.src[kind] + (int64_t)token * a.stride[kind] + h * ROW + c * (int)sizeof(T));
    else
#pragma unroll
      for (int k = 0; k < Raw<T>::W; ++k) r->w[k] = 0;
  };
  Raw<T> next;
  fetch(it, &next);

  // Sine and cosine of this lane's channels, the sine with its sign.
  const int half = a.half;
  const bool turns = PAIRS ? c < 2 * half : c < 2 * half && half > 0;
  float C0[8], S0[8];
  {
    float sn = 0.f, cs = 1.f;
    if (lane < half) {
      const double t = (double)pos * (a.inv_freq[lane] * 0.15915494309189533577);
      sincospif((float)(2.0 * (t - rint(t))), &sn, &cs);
      sn *= a.scale;
      cs *= a.scale;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const int ch = c + k;
      const int at = PAIRS ? ch >> 1 : ch < half ? ch : ch - half;
      const float s = __shfl(sn, at & 63), o = __shfl(cs, at & 63);
      const bool on = ch < 2 * half;
      C0[k] = on ? o : 1.f;
      S0[k] = !on ? 0.f : (PAIRS ? !(k & 1) : ch < half) ? -s : s;
    }
  }
  // The lane and the first channel of the partners.
  const int shift = c < half ? half : -half;
  const int partner = PAIRS || !turns ? lane : lane + shift / 8;
  const int pc = PAIRS || !turns ? c : c + shift;

  int kind = -1;
  bool normed = false;
  float C[8], S[8];
  for (; it < end; ++it) {
    const Raw<T> r = next;
    if (it + 1 < end) fetch(it + 1, &next);
    const int now = kind_of(it), h = head_of(it, now);
    const bool there = h < (now == 0 ? a.Hq : a.Hkv);
    if (now != kind && now < 2) {
      const float* w = a.weight[now];
      normed = w != nullptr;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        C[k] = C0[k] * (normed ? w[c + k] : 1.f);
        S[k] = S0[k] * (normed ? w[PAIRS ? c + (k ^ 1) : pc + k] : 1.f);
      }
    }
    kind = now;
    Raw<T> y = r;
    if (kind < 2) {
      float x[8], p[8], z[8];
      r.to(x);
      if constexpr (PAIRS) {
#pragma unroll
        for (int k = 0; k < 8; ++k) p[k] = x[k ^ 1];
      } else {
        Raw<T> o;
#pragma unroll
        for (int k = 0; k < Raw<T>::W; ++k) o.w[k] = (unsigned)__shfl((int)r.w[k], partner);
        o.to(p);
      }
      float rs = 1.f;
      if (normed) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < 8; ++k) s += x[k] * x[k];
        rs = __builtin_amdgcn_rsqf(head_sum<D>(s) * (1.f / D) + a.eps);
      }
      // (a channel that does not turn takes nothing from another, not its infinity either)
#pragma unroll
      for (int k = 0; k < 8; ++k) z[k] = x[k] * C[k] + (c + k < 2 * half ? p[k] * S[k] : 0.f);
      if (normed)
#pragma unroll
        for (int k = 0; k < 8; ++k) z[k] *= rs;
      y.from(z);
    }
    if (kind == 0) {
      if (there) y.store(a.q_out + ((int64_t)token * a.Hq + h) * ROW + c * (int)sizeof(T));
    } else if constexpr (!FP4) {
      if (there)
        y.store(a.pool + ((((int64_t)(word >> 4) * a.Hkv + h) * 2 + (kind - 1)) * kPageTokens + (word & 15)) * ROW +
                c * (int)sizeof(T));
    } else {
      unsigned code, byte;
      const unsigned w[4] = {y.w[0], y.w[1], y.w[2], y.w[3]};
      fp4_round(w, &code, &byte);
      if (there) {
        unsigned char* dst = a.pool + ((int64_t)(word >> 4) * a.Hkv + h) * Fp4<D>::PAGE;
        store_codes<D>(dst, word & 15, c, kind == 2, code);
        if ((c & 31) == 0) dst[fp4_scale<D>(word & 15, c, kind == 2)] = (unsigned char)byte;
      }
    }
  }
}

template <int D, class T, bool FP4>
void launch(const QkvArgs& a, unsigned grid, bool pairs, hipStream_t stream) {
  if (pairs) hipLaunchKernelGGL((k_qkv<D, T, FP4, true>), dim3(grid), dim3(64 * kWaves), 0, stream, a);
  else hipLaunchKernelGGL((k_qkv<D, T, FP4, false>), dim3(grid), dim3(64 * kWaves), 0, stream, a);
}
template <int D>
void launch(const QkvArgs& a, unsigned grid, int dtype, bool pairs, hipStream_t stream) {
  if (dtype == GA_F32) launch<D, float, false>(a, grid, pairs, stream);
  else if (dtype == GA_BF16) launch<D, __bf16, false>(a, grid, pairs, stream);
  else launch<D, __bf16, true>(a, grid, pairs, stream);
}

}  // namespace

hipError_t launch_qkv(const QkvArgs& args, int dim, int dtype, bool interleaved, hipStream_t stream) {
  QkvArgs a = args;
  const int group = 512 / dim;
  const int groups = (a.Hq + group - 1) / group + 2 * ((a.Hkv + group - 1) / group);
  // Groups of heads a wave.
  const int64_t most = (int64_t)groups * a.n / 8192;
  a.per = (int32_t)(most < 1 ? 1 : most > groups ? groups : most);
  a.parts = (groups + a.per - 1) / a.per;
  const int64_t tasks = (int64_t)a.n * a.parts;
  const int64_t grid = (tasks + kWaves - 1) / kWaves;
  if (grid > 0x3fffffffLL / kWaves) return hipErrorInvalidValue;
  if (dim == 64) launch<64>(a, (unsigned)grid, dtype, interleaved, stream);
  else launch<128>(a, (unsigned)grid, dtype, interleaved, stream);
  return hipGetLastError();
}

}  // namespace ga
