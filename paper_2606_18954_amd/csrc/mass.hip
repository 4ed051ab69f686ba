// Attention mass of cached tokens: for every slot w of the plan's segments
//   out[w] = decay in[w] + sum over the query rows r that see w, and their q-heads h, of
//            exp(scale q[r,h] . k[w] - lse[r,h]),
// the softmax weights of a step that has been attended (lse is its result), summed per token.
//
// A slot belongs to one chain, so one workgroup that takes some pages of a chain with all of its rows
// and all kv-heads owns those slots: no atomics, one order of the sums, the same bits every time.  Its
// waves take different kv-heads first, and different pages where heads are few.
//   S = Q K^T (16 rows x 16 tokens per matrix tile), p = 2^(S scale log2 e - lse log2 e)
// A lane holds four rows' scores of one token, so a token's sum is three additions in the lane and two
// exchanges with the other lanes of the token; the kv-heads' sums meet in LDS.
//
// Few rows (up to kMassRows, most chains of a decode step): two tiles' queries stay in registers and
// the pages stream past, several of them on their way, once per two tiles (from the caches after the first
// time).  More rows: a few pages stay, as matrix operands, and the rows stream past, one tile's queries and the
// next one's row numbers on their way.  A great many (more than kMassHuge, a prompt's prefill): the same by
// workgroups of twelve (head_dim 64: sixteen) waves, which share the rows of their four pages; a kernel of its own.
// (24 prompts of up to 1700 tokens, MXFP4, with four waves | so: 28/4 heads x 128 555 | 404 us, 16/2 x 64 373 | 124;
// chains of fewer rows lose by it, their workgroups' starts are no longer hidden by each other: merged graphs
// with 16 queries a branch, up to 1800 rows, 431 | 570.  A wave's step, a tile of rows against four pages, then
// takes a memory latency, 2200 cycles at three waves per SIMD, where its instructions take 730 for all three.
// Without gain: rows from the last one down, which reads the queries from memory once and not three times; the
// mask only where it is needed; sixteen waves of fewer registers, which leave no next tile's queries on their way,
// 425.)
//
// What bounds it: reading K.  1024 branches of merged graphs, 28/4 heads x 128, MXFP4: 129 us, 0.65 GB read at
// 5.0 TB/s (0.50 GB of them once; the rest are scales' half lines, queries and last pages read again), vector
// unit busy 39%, matrix cores 13%.  16 step trees, bf16 (70 MB): 27 us, a chain of five dependent loads (chain,
// page words and branches, queries and pages) and few pages a workgroup.  Measured and not taken: non-temporal
// page loads (trees 28 -> 45 us: chains of more than two tiles read their pages again), three or six pages
// on their way in place of four (135.0 and 138.8 against 134.5 us), workgroups of at most 32 or 64 pages x pairs
// (no change), twice the workgroups (147 us).
#include "attn_dev.hpp"
#include "evict_internal.hpp"
#include "mxfp4.hpp"
#include "pool_load.hpp"

#include <type_traits>

namespace ga {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

// Waves of a workgroup, and waves per SIMD the registers are kept to.
constexpr int mass_wg_waves(int D, int kind) { return kind < 2 ? 4 : D == 64 ? 16 : 12; }
constexpr int mass_waves(int D, int type, int kind) {
  return D == 64 ? 4 : kind == 2 ? 3 : type == GA_F32 ? 2 : kind == 1 ? 3 : 4;
}
// Pages of a part of more than kMassHuge rows (mass_parts), at most.
constexpr int kMassHugePages = 4;
static_assert(kMassHuge / 32 >= kMassCost && kMassPages <= kMassHugePages);

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

template <bool F32> struct Op;
template <> struct Op<true> { float v; };
template <> struct Op<false> { bf16x8 v; };

// One page's K as loaded: token r16.  The order of the channels in the contraction is free, as long as Q's is
// the same: the 16-byte pieces 4 i + kg of a row, so that the four lanes of a row load 64 neighbouring bytes;
// MXFP4: the channels kg D / 4 ..+ D / 4 - 1, whose codes are one load.
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
#pragma unroll
    for (int i = 0; i < C::NW / 4; ++i) k.w[i] = load16(page, r16 * D * C::ELT + 64 * i + 16 * kg);
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
template <int D, int TYPE, bool F32 = TYPE == GA_F32>
__device__ __forceinline__ void load_row(Op<F32> (&op)[F32 ? D / 4 : D / 32], const unsigned char* p,
                                         int kg) {
  if constexpr (TYPE == GA_F32) {
#pragma unroll
    for (int s = 0; s < D / 16; ++s) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(p + 64 * s + 16 * kg);
#pragma unroll
      for (int i = 0; i < 4; ++i) op[4 * s + i].v = x[i];
    }
  } else {
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
      op[s].v = *reinterpret_cast<const bf16x8*>(
          p + (TYPE == GA_MXFP4 ? kg * (D / 2) + 16 * s : 64 * s + 16 * kg));
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

// KIND 0: no chain has more than kMassRows rows, 1: some have, up to kMassHuge, 2: the chains of more.  (Kind 0
// has a third fewer registers than 1, and so more waves to hide the loads of a workgroup's start: merged graphs
// of 1024 branches 135 us with kind 0, 145 with kind 1.)
template <int D, int TYPE, bool CAUSAL, int KIND>
__global__ __launch_bounds__(64 * mass_wg_waves(D, KIND), mass_waves(D, TYPE, KIND)) void k_mass(MassArgs a) {
  constexpr int NWV = mass_wg_waves(D, KIND);
  constexpr bool HUGE_ROWS = KIND == 2;
  using C = MCfg<D, TYPE>;
  using OpT = Op<C::F32>;
  extern __shared__ float s_mass[];                 // [kv-head slot (x split)][page][token]
  // (part by part: those that most chains do not have come last)
  const int part = (int)blockIdx.y, v = (int)blockIdx.x;
  const int np_all = (a.seg_len[v] + kPageTokens - 1) / kPageTokens;
  const int64_t page0 = a.seg_page_off[v], goff = a.grp_off[v];
  const int cnt = (int)(a.grp_off[v + 1] - goff);
  const int cw = CAUSAL ? a.seg_causal[v] : kNoCausal;
  const int rows = cnt * a.group;
  if (HUGE_ROWS != rows > kMassHuge) return;              // (the other kernel's)
  const int nparts = mass_parts(np_all, rows, a.cost);    // equal ones
  if (part >= nparts) return;
  const int per = (np_all + nparts - 1) / nparts;
  const int pg0 = part * per;
  const int npg = min(per, np_all - pg0);
  if (npg <= 0) return;
  const int32_t* words = a.seg_pages + page0 + pg0;
  const int32_t* branches = a.grp_br + goff;
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kg = lane >> 4;
  const int hs = a.Hkv >= 4 ? 4 : a.Hkv >= 2 ? 2 : 1;     // waves that take different kv-heads
  const int rs = NWV / hs;                                // waves that share a head: its pages, or its rows
  const int hslot = wave % hs, split = wave / hs;
  const unsigned char* q = static_cast<const unsigned char*>(a.q);
  const int pw0 = words[min(lane, npg - 1)], pw1 = words[min(64 + lane, npg - 1)];   // a lane per page
  const bool cm = CAUSAL && cw != kNoCausal;
  const int ntile = (rows + 15) >> 4;
  const unsigned magic = 0xffffffffu / (unsigned)a.group;
  // r / group and its remainder: the truncated reciprocal is at most one short.
  auto split_row = [&](int r, int& j, int& gi) {
    j = (int)__umulhi((unsigned)r, magic);
    gi = r - j * a.group;
    if (gi >= a.group) { gi -= a.group; ++j; }
  };
  const int stride = (HUGE_ROWS ? kMassHugePages : a.cost) * kPageTokens;
  // The waves of a head take different pages; of a chain with a great many rows, a part of which has few, those
  // left take different rows.
  int psplit = rs;
  if constexpr (HUGE_ROWS)
    while (psplit > 1 && (psplit / 2) * C::PG >= npg) psplit /= 2;
  const int rsplit = rs / psplit;
  float* region = s_mass + (hslot + split / psplit * hs) * stride;
  // The first tile with a row that sees the page (a newest segment: its last row sees every page).
  auto first_tile = [&](int page) {
    return cm ? (int)(((int64_t)max(0, kPageTokens * page - cw) * a.group) >> 4) : 0;
  };
  const int tile0 = first_tile(pg0);
  const unsigned shift = 8 * (scale_byte<D>(r16, kg) & 3);    // (MXFP4)

  for (int h = hslot; h < a.Hkv; h += hs) {
    const unsigned char* pool_h = static_cast<const unsigned char*>(a.pool) + (int64_t)h * C::HEAD;
    auto page_of = [&](int p) {
      const int x = min(p, npg - 1);
      const int word = x < 64 ? __builtin_amdgcn_readlane(pw0, x) : __builtin_amdgcn_readlane(pw1, x - 64);
      return page_at(pool_h + (int64_t)(word & kPageIdMask) * a.Hkv * C::HEAD, C::HEAD);
    };
    auto put = [&](int p, float x, bool fresh) {
      // the four lanes of a token
      const auto h2 = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x),
                                                       __builtin_bit_cast(unsigned, x), false, false);
      const unsigned lo = h2[0], hi = h2[1];
      x = __builtin_bit_cast(float, lo) + __builtin_bit_cast(float, hi);
      const auto q2 = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x),
                                                       __builtin_bit_cast(unsigned, x), false, false);
      const unsigned lo2 = q2[0], hi2 = q2[1];
      x = __builtin_bit_cast(float, lo2) + __builtin_bit_cast(float, hi2);
      if (lane < kPageTokens) {
        float* at = region + p * kPageTokens + lane;
        *at = fresh ? x : *at + x;
      }
    };
    // (A slot past the segment's end may hold anything: only its own sums see it, and they are not
    // stored.)
    auto few = [&](auto nt_tag, int t0, bool fresh) {
      constexpr int NT = decltype(nt_tag)::value;
      OpT qo[NT][C::OPS];
      float lse[NT], nl[NT][4];
      int rank[NT], lim[NT][4];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        int j, gi;
        split_row(min(16 * (t0 + t) + r16, rows - 1), j, gi);
        const int64_t row = (int64_t)branches[j] * a.Hq + h * a.group + gi;
        load_row<D, TYPE>(qo[t], q + row * D * C::ELT, kg);
        lse[t] = a.lse[row];
        rank[t] = j;
      }
      // (Behind the queries, whose wait then leaves the pages in flight.  The pages are loaded whether
      // or not they exist, the last one again, so that every path has the same loads outstanding, and
      // nothing of a page is touched before its turn: either would be waited for with vmcnt(0).)
      RawK<D, TYPE> buf[C::PF];
#pragma unroll
      for (int i = 0; i < C::PF; ++i) load_k<D, TYPE>(buf[i], page_of(split + rs * i), r16, kg);
      // The lane's scores are of rows 4 kg + i of a tile.
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const float nr = offset_of(lse[t], 16 * (t0 + t) + r16 < rows);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          nl[t][i] = __shfl(nr, 4 * kg + i);
          if constexpr (CAUSAL)                         // sees page p's token r16 for 16 p <= lim
            lim[t][i] = cw + __shfl(rank[t], 4 * kg + i) - kPageTokens * pg0 - r16;
        }
      }
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
            put(p, x, fresh);
          }
          load_k<D, TYPE>(buf[i], page_of(p + rs * C::PF), r16, kg);
        }
      }
    };
    auto many = [&] {
      for (int p0 = C::PG * (split % psplit); p0 < npg; p0 += C::PG * psplit) {
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
        // Row of the lane in tile x: its number in q (clamped to the last row), and its rank.
        auto row_of = [&](int x, int& j) {
          int gi;
          split_row(min(16 * x + r16, rows - 1), j, gi);
          return (int64_t)branches[j] * a.Hq + h * a.group + gi;
        };
        // The next tile's queries, and the row numbers of the one behind it, are on their way.
        int t = first_tile(pg0 + p0) + split / psplit, j0, j1, j2;
        OpT qo[C::OPS], qn[C::OPS];
        int64_t row = row_of(t, j0);
        float l0 = a.lse[row], l1;
        load_row<D, TYPE>(qo, q + row * D * C::ELT, kg);
        row = row_of(t + rsplit, j1);
        for (; t < ntile; t += rsplit) {
          load_row<D, TYPE>(qn, q + row * D * C::ELT, kg);
          l1 = a.lse[row];
          row = row_of(t + 2 * rsplit, j2);
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
          // (masked last: a row whose lse is NaN says nothing of a token that it does not see)
          auto add = [&](auto masked) {
            int lim[4];
            if constexpr (decltype(masked)::value)
#pragma unroll
              for (int i = 0; i < 4; ++i)
                lim[i] = cw + __shfl(j0, 4 * kg + i) - kPageTokens * (pg0 + p0) - r16;
#pragma unroll
            for (int g = 0; g < C::PG; ++g) {
              float e[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                float x = fmaf(S[g][i], a.scale_log2, nl[i]);
                if constexpr (decltype(masked)::value)
                  x = kPageTokens * g > lim[i] ? -__builtin_huge_valf() : x;
                e[i] = exp2_(x);
              }
              acc[g] += (e[0] + e[1]) + (e[2] + e[3]);
            }
          };
          if (CAUSAL && cm) add(std::true_type{});
          else add(std::false_type{});
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
    if (HUGE_ROWS || (KIND == 1 && rows > kMassRows)) {
      if constexpr (KIND > 0) many();
    } else if constexpr (!HUGE_ROWS) {
      int t = tile0;
      for (; t + 1 < ntile; t += 2) few(std::integral_constant<int, 2>{}, t, h == hslot && t == tile0);
      if (t < ntile) few(std::integral_constant<int, 1>{}, t, h == hslot && t == tile0);
    }
  }
  // The slots' earlier mass is on its way while the last waves come in.
  constexpr int PPI = 4 * NWV, IN = kMassCost / PPI;   // pages at a time
  float in[IN];
  int64_t slot[IN];
#pragma unroll
  for (int i = 0; i < IN; ++i) {
    const int p = i * PPI + (tid >> 4), tok = tid & 15;
    slot[i] = -1;
    in[i] = 0.f;
    if (i * PPI < npg && p < npg) {
      const int word = words[p];
      if (tok <= (int)((unsigned)word >> kPageValidShift)) {
        slot[i] = (int64_t)(word & kPageIdMask) * kPageTokens + tok;
        if (a.mass_in) in[i] = a.mass_in[slot[i]];
      }
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < IN; ++i) {
    if (slot[i] < 0) continue;
    const int p = i * PPI + (tid >> 4), tok = tid & 15;
    float sum = 0.f;
    for (int k = 0; k < hs * rsplit; ++k) sum += s_mass[k * stride + p * kPageTokens + tok];
    a.mass_out[slot[i]] = a.mass_in ? fmaf(a.decay, in[i], sum) : sum;
  }
}

template <int D>
hipError_t launch_t(const MassArgs& a, hipStream_t stream) {
  auto type = [&](auto causal, auto kind) {
    constexpr bool CAUSAL = decltype(causal)::value;
    constexpr int KIND = decltype(kind)::value, NWV = mass_wg_waves(D, KIND);
    const int parts = KIND == 2 ? a.parts_huge : a.parts;
    if (parts == 0) return;
    const unsigned lds = (KIND == 2 ? NWV * kMassHugePages : 4 * a.cost) * kPageTokens * sizeof(float);
    auto go = [&](auto kernel) {
      hipLaunchKernelGGL(kernel, dim3((unsigned)a.chains, (unsigned)parts), dim3(64 * NWV), lds, stream, a);
    };
    if (a.dtype == GA_F32) go(k_mass<D, GA_F32, CAUSAL, KIND>);
    else if (a.dtype == GA_BF16) go(k_mass<D, GA_BF16, CAUSAL, KIND>);
    else go(k_mass<D, GA_MXFP4, CAUSAL, KIND>);
  };
  auto kinds = [&](auto causal) {
    type(causal, std::integral_constant<int, 2>{});
    if (a.many) type(causal, std::integral_constant<int, 1>{});
    else type(causal, std::integral_constant<int, 0>{});
  };
  if (a.causal) kinds(std::true_type{});
  else kinds(std::false_type{});
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mass(const MassArgs& a, hipStream_t stream) {
  if (a.chains == 0) return hipSuccess;
  if (a.head_dim == 64) return launch_t<64>(a, stream);
  if (a.head_dim == 128) return launch_t<128>(a, stream);
  return hipErrorInvalidValue;
}

}  // namespace ga
