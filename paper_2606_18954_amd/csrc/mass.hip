// Attention mass of cached tokens: for every slot w of the plan's segments
//   out[w] = decay in[w] + sum over the query rows r that see w, and their q-heads h, of
//            exp(scale q[r,h] . k[w] - lse[r,h]),
// the softmax weights of a step that has been attended (lse is its result), summed per token.
//
// A slot belongs to one chain, so one workgroup that takes some pages of a chain with all of its rows
// and all kv-heads owns those slots: no atomics, one order of the sums, the same bits every time.  Its
// waves take different kv-heads first, and different pages where heads are few.
//   S = Q K^T (16 rows x 16 tokens per matrix tile), p = 2^(S scale log2 e - lse log2 e)
// A lane holds four rows' scores of one token, so a token's sum is three additions in the lane; the
// four lanes of a token meet in LDS, with the kv-heads, once per unit.
//
// Few rows (up to kFewTiles tiles: every page of a decode step): two tiles' queries stay in registers and
// the pages stream past, several of them on their way, once per two tiles (from the caches after the first
// time).  More rows (prefill): a few pages stay, as matrix operands, and the rows stream past, one tile's
// queries and the next one's row numbers on their way.
#include "attn_dev.hpp"
#include "evict_internal.hpp"
#include "mxfp4.hpp"
#include "pool_load.hpp"

#include <type_traits>

namespace ga {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Waves per SIMD the registers are kept to.
constexpr int mass_waves(int D, int type) { return type == GA_F32 ? 2 : D == 64 ? 4 : 3; }

template <int D, int TYPE>
struct MCfg {
  static constexpr bool F32 = TYPE == GA_F32;
  static constexpr int ELT = F32 ? 4 : 2;
  static constexpr int OPS = F32 ? D / 4 : D / 32;  // contraction steps
  static constexpr int NW = TYPE == GA_MXFP4 ? D / 32 : D * ELT / 16;   // words a lane holds of a page's K
  static constexpr int HEAD = TYPE == GA_MXFP4 ? 17 * D : 32 * D * ELT; // bytes of a page's head
  static constexpr int PG = F32 ? 2 : 4;            // pages that stay (many rows)
  // Pages on their way or in use (few rows).
  static constexpr int PF = TYPE == GA_MXFP4 ? 4 : NW <= 8 ? 3 : NW <= 16 ? 2 : 1;
};

// Most row tiles that are taken two at a time: a row block, whose branches the descriptor lists.
constexpr int kFewTiles = kRowsPerBlock / 16;

template <bool F32> struct Op;
template <> struct Op<true> { float v; };
template <> struct Op<false> { bf16x8 v; };

// One page's K as loaded: token r16, channels kg D / 4 ..+ D / 4 - 1.
template <int D, int TYPE>
struct RawK {
  u32x4 w[(MCfg<D, TYPE>::NW + 3) / 4];
  unsigned scale;                                   // the word with its scale
};
// Place of the scale of the lane's channels among a page's K scales.
template <int D>
__device__ __forceinline__ unsigned scale_byte(int r16, int kg) {
  return r16 * Fp4<D>::NS + (kg * (D / 4)) / 32;
}
template <int D, int TYPE>
__device__ __forceinline__ void load_k(RawK<D, TYPE>& k, page_t page, int r16, int kg) {
  using C = MCfg<D, TYPE>;
  if constexpr (TYPE == GA_MXFP4) {
    const unsigned off = r16 * (D / 2) + kg * (D / 8);
    if constexpr (D == 128) {
      k.w[0] = load16(page, off);
    } else {
      const u32x2 x = load8(page, off);
      k.w[0] = u32x4{x[0], x[1], 0, 0};
    }
    k.scale = load4(page, Fp4<D>::KS + (scale_byte<D>(r16, kg) & ~3u));
  } else {
    const unsigned off = (r16 * D + kg * (D / 4)) * C::ELT;
#pragma unroll
    for (int i = 0; i < C::NW / 4; ++i) k.w[i] = load16(page, off + 16 * i);
  }
}
template <int D, int TYPE, int S>
__device__ __forceinline__ Op<MCfg<D, TYPE>::F32> operand(const RawK<D, TYPE>& k, unsigned shift) {
  Op<MCfg<D, TYPE>::F32> o;
  if constexpr (TYPE == GA_F32) {
    const unsigned w = k.w[S / 4][S % 4];           // (a bit cast takes no vector element)
    o.v = __builtin_bit_cast(float, w);
  } else if constexpr (TYPE == GA_BF16) {
    o.v = __builtin_bit_cast(bf16x8, k.w[S]);
  } else {
    const float s = fp4_exp_at(k.scale, shift);
    const unsigned w = k.w[S / 4][S % 4];
    const u32x4 x = {fp4_pair<0>(w, s), fp4_pair<1>(w, s), fp4_pair<2>(w, s), fp4_pair<3>(w, s)};
    o.v = __builtin_bit_cast(bf16x8, x);
  }
  return o;
}
// The lane's operands of one row of Q: the same channels.
template <int D, bool F32>
__device__ __forceinline__ void load_row(Op<F32> (&op)[F32 ? D / 4 : D / 32], const unsigned char* p,
                                         int kg) {
  if constexpr (F32) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(p + kg * D + 16 * s);
#pragma unroll
      for (int i = 0; i < 4; ++i) op[4 * s + i].v = x[i];
    }
  } else {
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
      op[s].v = *reinterpret_cast<const bf16x8*>(p + kg * (D / 2) + 16 * s);
  }
}
template <bool F32>
__device__ __forceinline__ f32x4 product(Op<F32> a, Op<F32> b, f32x4 c) {
  if constexpr (F32) return __builtin_amdgcn_mfma_f32_16x16x4f32(a.v, b.v, c, 0, 0, 0);
  else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, b.v, c, 0, 0, 0);
}
template <int N, int I = 0, typename F>
__device__ __forceinline__ void steps(F f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    steps<N, I + 1>(f);
  }
}

// A row's offset of the exponent: -lse in the log2 domain; a row without any weight counts for
// nothing.
__device__ __forceinline__ float offset_of(float lse, bool live) {
  return live && fabsf(lse) != __builtin_huge_valf() ? -1.4426950408889634f * lse
                                                     : -__builtin_huge_valf();
}

template <int D, int TYPE, bool CAUSAL>
__global__ __launch_bounds__(256, mass_waves(D, TYPE)) void k_mass(MassArgs a) {
  using C = MCfg<D, TYPE>;
  using OpT = Op<C::F32>;
  __shared__ float s_mass[4][kMassPages * 64];      // [kv-head slot][page][kg][token]
  const int gpc = (a.chunk_pages + a.pages - 1) / a.pages;
  const int item = (int)blockIdx.x / gpc;
  const int pg0 = ((int)blockIdx.x - item * gpc) * a.pages;
  if (item >= a.counters[0]) return;
  const int32_t* d = a.desc + (int64_t)item * a.desc_words;
  const int np = d[0], cw = d[1], cnt = d[3], goff = d[5];
  if (d[4] != 0 || pg0 >= np) return;               // (the first row block's item takes all rows)
  const int npg = min(a.pages, np - pg0);
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kg = lane >> 4;
  const int hs = a.Hkv >= 4 ? 4 : a.Hkv >= 2 ? 2 : 1;     // waves that take different kv-heads
  const int rs = 4 / hs;                                  // waves that share a head's pages
  const int hslot = wave % hs, split = wave / hs;
  const unsigned char* q = static_cast<const unsigned char*>(a.q);
  const int pw = d[kDescHead + pg0 + min(lane, npg - 1)]; // lane p: word of page pg0 + p
  const bool cm = CAUSAL && cw != kNoCausal;
  const int rows = cnt * a.group;
  const int ntile = (rows + 15) >> 4;
  const unsigned magic = 0xffffffffu / (unsigned)a.group;
  // r / group and its remainder: the truncated reciprocal is at most one short.
  auto split_row = [&](int r, int& j, int& gi) {
    j = (int)__umulhi((unsigned)r, magic);
    gi = r - j * a.group;
    if (gi >= a.group) { gi -= a.group; ++j; }
  };
  float* region = s_mass[hslot];
  // The first tile with a row that sees page pg0 (causal units; the newest row sees every page).
  auto first_tile = [&](int page) {
    return cm ? (int)(((int64_t)max(0, kPageTokens * page - cw) * a.group) >> 4) : 0;
  };
  const int tile0 = first_tile(pg0);
  const unsigned shift = 8 * (scale_byte<D>(r16, kg) & 3);    // (MXFP4)

  for (int h = hslot; h < a.Hkv; h += hs) {
    const unsigned char* pool_h = static_cast<const unsigned char*>(a.pool) + (int64_t)h * C::HEAD;
    auto page_of = [&](int p) {
      const int word = __builtin_amdgcn_readlane(pw, min(p, npg - 1));
      return page_at(pool_h + (int64_t)(word & kPageIdMask) * a.Hkv * C::HEAD, C::HEAD);
    };
    auto put = [&](int p, float x, bool fresh) {
      float* at = region + p * 64 + lane;
      *at = fresh ? x : *at + x;
    };
    // (A slot past the segment's end may hold anything: only its own sums see it, and they are not
    // stored.)
    auto few = [&](auto nt_tag, int t0) {
      constexpr int NT = decltype(nt_tag)::value;
      OpT qo[NT][C::OPS];
      float nl[NT][4];
      int lim[NT][4];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        int j, gi;
        split_row(min(16 * (t0 + t) + r16, rows - 1), j, gi);
        const int64_t row = (int64_t)d[kDescHead + a.chunk_pages + j] * a.Hq + h * a.group + gi;
        load_row<D, C::F32>(qo[t], q + row * D * C::ELT, kg);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = 16 * (t0 + t) + 4 * kg + i;
          split_row(min(r, rows - 1), j, gi);
          const int64_t lr = (int64_t)d[kDescHead + a.chunk_pages + j] * a.Hq + h * a.group + gi;
          nl[t][i] = offset_of(a.lse[lr], r < rows);
          if constexpr (CAUSAL)
            lim[t][i] = cw + j - kPageTokens * pg0 - r16;   // sees page p's token r16 for 16 p <= lim
        }
      }
      // (Behind the queries, whose wait then leaves the pages in flight.  The pages are loaded whether
      // or not they exist, the last one again, so that every path has the same loads outstanding, and
      // nothing of a page is touched before its turn: either would be waited for with vmcnt(0).)
      RawK<D, TYPE> buf[C::PF];
#pragma unroll
      for (int i = 0; i < C::PF; ++i) load_k<D, TYPE>(buf[i], page_of(split + rs * i), r16, kg);
      for (int p0 = split; p0 < npg; p0 += rs * C::PF) {
#pragma unroll
        for (int i = 0; i < C::PF; ++i) {
          const int p = p0 + rs * i;
          __builtin_amdgcn_sched_barrier(0);
          if (p < npg) {
            f32x4 S[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) S[t] = f32x4{0.f, 0.f, 0.f, 0.f};
            steps<C::OPS>([&](auto st) {
              constexpr int s = decltype(st)::value;
              const OpT kb = operand<D, TYPE, s>(buf[i], shift);
#pragma unroll
              for (int t = 0; t < NT; ++t) S[t] = product<C::F32>(qo[t][s], kb, S[t]);
            });
            float x = 0.f;
#pragma unroll
            for (int t = 0; t < NT; ++t) {
              float e[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                e[k] = exp2_(fmaf(S[t][k], a.scale_log2, nl[t][k]));
                if constexpr (CAUSAL)
                  if (cm && kPageTokens * p > lim[t][k]) e[k] = 0.f;
              }
              x += (e[0] + e[1]) + (e[2] + e[3]);
            }
            put(p, x, h == hslot && t0 == tile0);
          }
          load_k<D, TYPE>(buf[i], page_of(p + rs * C::PF), r16, kg);
        }
      }
    };
    auto many = [&] {
      for (int p0 = C::PG * split; p0 < npg; p0 += C::PG * rs) {
        OpT kb[C::PG][C::OPS];
        {
          RawK<D, TYPE> raw[C::PG];
#pragma unroll
          for (int g = 0; g < C::PG; ++g) load_k<D, TYPE>(raw[g], page_of(p0 + g), r16, kg);
#pragma unroll
          for (int g = 0; g < C::PG; ++g)
            steps<C::OPS>([&](auto st) {
              constexpr int s = decltype(st)::value;
              kb[g][s] = operand<D, TYPE, s>(raw[g], shift);
            });
        }
        float acc[C::PG];
#pragma unroll
        for (int g = 0; g < C::PG; ++g) acc[g] = 0.f;
        int t = first_tile(pg0 + p0);
        // Row of the lane in tile x: its number in q (clamped to the last row), and its rank.
        auto row_of = [&](int x, int& j) {
          int gi;
          split_row(min(16 * x + r16, rows - 1), j, gi);
          return (int64_t)a.grp_br[goff + j] * a.Hq + h * a.group + gi;
        };
        OpT qo[C::OPS], qn[C::OPS];
        int j0 = 0, j1 = 0;
        int64_t row1 = row_of(t, j0);
        float l0 = a.lse[row1], l1 = 0.f;
        load_row<D, C::F32>(qo, q + row1 * D * C::ELT, kg);
        row1 = row_of(t + 1, j1);
        for (; t < ntile; ++t) {
          load_row<D, C::F32>(qn, q + row1 * D * C::ELT, kg);
          l1 = a.lse[row1];
          int j2;
          row1 = row_of(t + 2, j2);
          f32x4 S[C::PG];
#pragma unroll
          for (int g = 0; g < C::PG; ++g) S[g] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int s = 0; s < C::OPS; ++s)
#pragma unroll
            for (int g = 0; g < C::PG; ++g) S[g] = product<C::F32>(qo[s], kb[g][s], S[g]);
          // The lane's scores are of rows 4 kg + i of the tile.
          const float nr = offset_of(l0, 16 * t + r16 < rows);
          float nl[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) nl[i] = __shfl(nr, 4 * kg + i);
          if (cm) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int lim = cw + __shfl(j0, 4 * kg + i) - kPageTokens * (pg0 + p0) - r16;
#pragma unroll
              for (int g = 0; g < C::PG; ++g)
                S[g][i] = kPageTokens * g > lim ? -__builtin_huge_valf() : S[g][i];
            }
          }
#pragma unroll
          for (int g = 0; g < C::PG; ++g) {
            float e[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) e[i] = exp2_(fmaf(S[g][i], a.scale_log2, nl[i]));
            acc[g] += (e[0] + e[1]) + (e[2] + e[3]);
          }
#pragma unroll
          for (int s = 0; s < C::OPS; ++s) qo[s] = qn[s];
          l0 = l1;
          j0 = j1;
          j1 = j2;
        }
#pragma unroll
        for (int g = 0; g < C::PG; ++g)
          if (p0 + g < npg) put(p0 + g, acc[g], h == hslot);
      }
    };
    if (ntile > kFewTiles) {
      many();
    } else {
      int t = tile0;
      for (; t + 1 < ntile; t += 2) few(std::integral_constant<int, 2>{}, t);
      if (t < ntile) few(std::integral_constant<int, 1>{}, t);
    }
  }
  __syncthreads();
  for (int x = tid; x < 16 * npg; x += 256) {
    const int p = x >> 4, tok = x & 15;
    const int word = d[kDescHead + pg0 + p];
    if (tok > (int)((unsigned)word >> kPageValidShift)) continue;
    float sum = 0.f;
    for (int k = 0; k < hs; ++k) {
      const float* r = s_mass[k] + p * 64 + tok;
      sum += (r[0] + r[16]) + (r[32] + r[48]);
    }
    const int64_t slot = (int64_t)(word & kPageIdMask) * kPageTokens + tok;
    a.mass_out[slot] = a.mass_in ? fmaf(a.decay, a.mass_in[slot], sum) : sum;
  }
}

template <int D>
hipError_t launch_t(const MassArgs& a, hipStream_t stream) {
  const int64_t grid = a.units * ((a.chunk_pages + a.pages - 1) / a.pages);
  if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
  auto go = [&](auto kernel) {
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(256), 0, stream, a);
  };
  auto type = [&](auto causal) {
    constexpr bool CAUSAL = decltype(causal)::value;
    if (a.dtype == GA_F32) go(k_mass<D, GA_F32, CAUSAL>);
    else if (a.dtype == GA_BF16) go(k_mass<D, GA_BF16, CAUSAL>);
    else go(k_mass<D, GA_MXFP4, CAUSAL>);
  };
  if (a.causal) type(std::true_type{});
  else type(std::false_type{});
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mass(const MassArgs& a, hipStream_t stream) {
  if (a.units == 0) return hipSuccess;
  if (a.head_dim == 64) return launch_t<64>(a, stream);
  if (a.head_dim == 128) return launch_t<128>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace ga
