// Segment attention over MXFP4 pools (decode, and multi-query steps with few rows a page): one work item =
// (segment chain, page chunk, row block of up to 128 query rows, kv-head), as in seg_attn.hip, with the work
// list, the descriptors, the partial rows and the merge shared with it.
//
//   S^T = K Q^T   (16 tokens x 16 rows per matrix tile, contraction over head_dim)
//   O^T += V^T P^T (contraction over the 32 tokens of a pair of pages)
//
// A page of a kv-head is 17 D bytes (mxfp4.hpp), 17/64 of bf16's, so a page that few rows read
// is soon there and the instructions per page matter.  Three things keep them few:
// * The page goes from global memory into registers, in the lanes that need it: a lane's K
//   operand is D / 4 consecutive channels of one token (the channels' order in the contraction is
//   free as long as Q's is the same), its V operand four consecutive tokens of D / 16 channels.  No
//   LDS, no barrier and no transposition between the load and the matrix cores.
// * 4-bit codes become bf16 by one conversion per two values, their scale included.  K's pairs are
//   neighbouring channels, as the operand wants them; V's are as well, where the operand wants
//   neighbouring tokens: one byte permutation per two values puts them right.
// * A lane's scores are those of the tokens whose V it holds, so P needs no exchange either; and
//   its outputs are D / 4 consecutive columns of one row.
// The waves of a workgroup share a unit by its row tiles: up to two tiles, the waves take pairs of
// pages in turn, each with all rows; three or four, two groups of waves hold two tiles each; more,
// every wave holds its own tiles and sees every page (its second read comes from the caches).  A wave
// runs through its pages alone; only the end of a unit, where the waves' (m, l, O) are joined in LDS
// and the rows are written, needs barriers.
//
// Online softmax as in seg_attn.hip (log2 domain, lazily moved reference), float32 throughout;
// probabilities are rounded to bf16 for the second product (V's exponents need bf16's range).
//
// What bounds it.  Decode of 64 merged graphs, 1024 branches of 28/4 heads x 128 (449 K pages of a head, 0.98 GB):
// 237 us, 4.6 TB/s of reads and writes where pages alone, read in this pattern, come at 5.9; the vector unit is
// busy 58% of the time and the matrix cores 15%.  With the pages in the L2 the same instructions take 161 to
// 172 us, and reading the pages without them 165: neither is hidden whole by the other.  256 branches of
// 16384 tokens, 40/8 heads: 390 us, 4.7 TB/s.  16 step trees (38 MB): 18 us, one or two units a workgroup.
// Rejected, on the first of these (246 us then): four waves per SIMD, no change; two kv-heads a unit, no
// change, four slower (uneven ends); a unit's first pages loaded before the last one's rows are joined, no
// change; page loads that skip the last turns' duplicates, 259 us and spills; three pairs of pages in flight,
// slower.
#include "attn_dev.hpp"
#include "ga_internal.hpp"
#include "mxfp4.hpp"
#include "pool_load.hpp"

#include <hip/hip_ext.h>

#include <type_traits>

namespace ga {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <int D>
struct QCfg {
  static constexpr int LW = D / 32;                 // 32-bit words of K (or V) a lane holds per page
  static constexpr int QS = D / 32;                 // contraction steps of S^T = K Q^T
  static constexpr int NB = D / 16;                 // 16-column tiles of O^T
};

// One page as loaded: K and V codes, the word with K's scale, V's four scales.
template <int D>
struct Page {
  unsigned k[QCfg<D>::LW], v[QCfg<D>::LW];
  unsigned ks, vs;
};

template <int D>
__device__ __forceinline__ void load_words(unsigned (&w)[QCfg<D>::LW], page_t page, unsigned off) {
  if constexpr (D == 128) {
    const u32x4 x = load16(page, off);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = x[i];
  } else {
    const u32x2 x = load8(page, off);
    w[0] = x[0];
    w[1] = x[1];
  }
}

__device__ __forceinline__ float quad_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16));
  return fmaxf(v, __shfl_xor(v, 32));
}
__device__ __forceinline__ float quad_sum(float v) {
  v += __shfl_xor(v, 16);
  return v + __shfl_xor(v, 32);
}

// MAXNT: row tiles of a wave, one (steps with few rows a page: fewer registers, a workgroup more per CU) or two
// (a page is converted for twice the rows).  The line is 32 rows a page (us, two | one): merged graphs of 1024
// branches (16 rows) 258 | 250, 16 step trees (17 rows) 26.6 | 23.0, 30 prompts of 400 tokens with 10 branches of
// 28/4 heads (40 rows) 60.5 | 60.1, with 20 branches (75 rows) 80 | 86; against the rule only the long contexts
// above (12 rows, a fifth of the pages with 40), 390 | 402.
template <int D, bool CAUSAL, int MAXNT>
__global__ __launch_bounds__(kAttnThreads, fp4_wgs_per_cu(MAXNT == 1, D)) void k_fp4_attn(AttnArgs a) {
  using C = QCfg<D>;
  using F = Fp4<D>;
  constexpr int PF = MAXNT == 1 ? 2 : 3;            // pairs of pages in flight or in use per wave
  __shared__ __align__(1024) int s_desc[2][kDescMaxBytes / 4];
  __shared__ __align__(16) float s_o[4][16 * D];    // a row tile of each wave, chunks XOR-permuted
  __shared__ float s_m[4][16], s_l[4][16];
  __shared__ int s_next[2];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kg = lane >> 4;
  const int n_work = (int)(a.counters[0] * a.Hkv);
  const float NEG_INF = -__builtin_huge_valf();
  const unsigned char* pool = static_cast<const unsigned char*>(a.pool);
  const __bf16* qbase = static_cast<const __bf16*>(a.q);
  const unsigned lds_desc =
      (unsigned)(uintptr_t)(__attribute__((address_space(3))) int*)&s_desc[0][0];
  const int dins = (a.desc_words * 4 + 1023) / 1024;
  const int br_word = kDescHead + a.chunk_pages;

  auto fetch_desc = [&](int v, int nb) {
    const bool ok = v < n_work;
    if (lane == 0) s_next[nb] = ok ? v : -1;
    if (ok) {
      const int* src = a.desc + (int64_t)(v / a.Hkv) * a.desc_words;
      const unsigned dst = lds_desc + nb * kDescMaxBytes;
      for (int i = 0; i < dins; ++i)
        dma16(1024 * i + 16 * lane, src, __builtin_amdgcn_readfirstlane(dst + 1024 * i));
    }
  };

  // Work streams as in seg_attn.hip.
  const int ns = a.streams;
  const int per = a.Hkv / ns;
  const int n_str = (int)(a.counters[0] * per);
  int* heads = reinterpret_cast<int*>(a.counters + 4);
  auto gs = [&](int st) { return ((int)gridDim.x - st + ns - 1) / ns; };
  auto unit_of = [&](int j, int st) {
    return j < n_str ? (j / per) * a.Hkv + (j % per) * ns + st : n_work;
  };
  int cs = (int)blockIdx.x % ns;
  const int rank = (int)blockIdx.x / ns;
  if (wave == 0) {
    fetch_desc(unit_of(rank, cs), 0);
    wait_vmcnt(0);
  }
  __syncthreads();

  const int64_t blk_stride = (int64_t)a.Hkv * F::PAGE;
  // The lane's bytes of a page.
  const unsigned k_off = r16 * (D / 2) + kg * (D / 8);
  const unsigned v_off = F::V + lane * (D / 8);
  const unsigned ks_byte = r16 * F::NS + (kg * (D / 4)) / 32;
  const unsigned ks_off = F::KS + (ks_byte & ~3u), ks_shift = 8 * (ks_byte & 3);
  const unsigned vs_off = F::VS + (kg * F::NS + (r16 * F::SL) / 32) * 4;

  bool first = true;
  for (int b = 0;; b ^= 1) {
    const int w = __builtin_amdgcn_readfirstlane(s_next[b]);
    if (w < 0) break;
    const int* dsc = &s_desc[b][0];
    const int kvh = w % a.Hkv;
    const int np0 = __builtin_amdgcn_readfirstlane(dsc[0]);
    const int cw = __builtin_amdgcn_readfirstlane(dsc[1]);
    const int cnt = __builtin_amdgcn_readfirstlane(dsc[3]);
    const int row0 = __builtin_amdgcn_readfirstlane(dsc[4]) * kRowsPerBlock;
    const int prow_base = __builtin_amdgcn_readfirstlane(dsc[7]);
    const int R = min(kRowsPerBlock, cnt * a.group - row0);
    const int nrt = (R + 15) >> 4;
    const int j0 = row0 / a.group;
    const bool cm = CAUSAL && cw != kNoCausal;
    // Pages that some row of the unit sees (multi-query).
    int np = np0;
    if (cm) np = max(0, min(np0, (cw + (row0 + R - 1) / a.group + kPageTokens) / kPageTokens));
    const int npairs = (np + 1) >> 1;
    // Words of the pair's pages, a lane per pair (the second page of a last pair may not exist: the
    // first once more, masked).
    const int pk0 = dsc[kDescHead + max(0, min(2 * lane, np - 1))];
    const int pk1 = dsc[kDescHead + max(0, min(2 * lane + 1, np - 1))];

    const unsigned char* pool_h = (const unsigned char*)uniform64(
        (int64_t)(uintptr_t)(pool + (int64_t)kvh * F::PAGE));

    // One pass over the pages: ng groups of ks = 4 / ng waves.  The waves of a group share row tiles
    // (group g: tiles tile0 + g + ng t) and take pairs of pages in turn.
    auto run_pass = [&](auto nt_tag, int ng, int tile0) {
      constexpr int NT = decltype(nt_tag)::value;
      const int ks = 4 / ng;
      const int grp = wave % ng, split = wave / ng;
      const bool claims = tile0 == 0;                // (the unit's first pass)
      auto tile_of = [&](int g, int t) { return tile0 + g + ng * t; };
      auto load_page = [&](Page<D>& pg, int word) {
        const page_t page = page_at(pool_h + (int64_t)(word & kPageIdMask) * blk_stride, F::PAGE);
        load_words<D>(pg.k, page, k_off);
        load_words<D>(pg.v, page, v_off);
        pg.ks = load4(page, ks_off);
        pg.vs = load4(page, vs_off);
      };
      const int last_pair = max(npairs - 1, 0);
      auto load_pair = [&](Page<D> (&pp)[2], int p) {
        const int x = min(p, last_pair);
        load_page(pp[0], __builtin_amdgcn_readlane(pk0, x));
        load_page(pp[1], __builtin_amdgcn_readlane(pk1, x));
      };

      Page<D> buf[PF][2];
      bf16x8 qop[NT][C::QS];
      float m[NT], l[NT];
      f32x4 O[NT][C::NB];
      int cl[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        m[t] = NEG_INF;
        l[t] = 0.f;
#pragma unroll
        for (int n = 0; n < C::NB; ++n) O[t][n] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      int claim = 0;
      if (claims && !first && wave == 0 && lane == 0) claim = atomicAdd(&heads[cs], 1);
      // Q operand: lane holds row r16 of the tile, channels kg D / 4 + 8 s ..+ 7 at step s.
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const int r = tile_of(grp, t) * 16 + r16;
        const bool live = r < R;
        const __bf16* qp = qbase;
        if (live) {
          const int gr = row0 + r;
          const int j = gr / a.group;
          qp = qbase + ((int64_t)dsc[br_word + j - j0] * a.Hq + kvh * a.group + (gr - j * a.group)) * D;
        }
#pragma unroll
        for (int s = 0; s < C::QS; ++s) {
          bf16x8 v = {};
          if (live) v = *reinterpret_cast<const bf16x8*>(qp + kg * (D / 4) + 8 * s);
          qop[t][s] = v;
        }
        // The lane's row sees chunk token 16 p + 4 kg + i only for 16 p + i <= cl.
        cl[t] = cm ? cw + (row0 + r) / a.group - 4 * kg : 0x3fffffff;
      }
      // (The pages come behind the claim and the queries, whose waits then leave them in flight; they are
      // loaded whether or not they exist, the last pair again, so that every path has the same loads
      // outstanding.)
#pragma unroll
      for (int i = 0; i < PF; ++i) load_pair(buf[i], split + ks * i);
      // The next unit's descriptor is fetched while this one streams.
      if (claims && wave == 0) {
        int v;
        if (first) {
          v = unit_of(rank + gs(cs), cs);
        } else {
          int j = 2 * gs(cs) + __builtin_amdgcn_readfirstlane(claim);
          for (int t = 1; j >= n_str && t < ns; ++t) {
            cs = cs + 1 == ns ? 0 : cs + 1;
            int c = 0;
            if (lane == 0) c = atomicAdd(&heads[cs], 1);
            j = 2 * gs(cs) + __builtin_amdgcn_readfirstlane(c);
          }
          v = unit_of(j, cs);
        }
        fetch_desc(v, b ^ 1);
      }
      auto pair = [&](Page<D> (&pp)[2], int p) {
        f32x4 S[2][NT];
        int valid[2];
        valid[0] = (int)((unsigned)__builtin_amdgcn_readlane(pk0, p) >> kPageValidShift);
        valid[1] = 2 * p + 1 < np
                       ? (int)((unsigned)__builtin_amdgcn_readlane(pk1, p) >> kPageValidShift)
                       : -1;
        // Slots behind the segment's end may hold anything: their scores are replaced below, and
        // V's scales are cleared, so that no NaN meets a zero probability.
#pragma unroll
        for (int g = 0; g < 2; ++g) {
          if (valid[g] != kPageTokens - 1) {
            const int n = min(max(valid[g] + 1 - 4 * kg, 0), 4);
            pp[g].vs &= n == 4 ? 0xffffffffu : (1u << (8 * n)) - 1u;
          }
#pragma unroll
          for (int t = 0; t < NT; ++t) S[g][t] = f32x4{0.f, 0.f, 0.f, 0.f};
          const float sk = fp4_exp_at(pp[g].ks, ks_shift);
#pragma unroll
          for (int s = 0; s < C::QS; ++s) {
            u32x4 ka;
            ka[0] = fp4_pair<0>(pp[g].k[s], sk);
            ka[1] = fp4_pair<1>(pp[g].k[s], sk);
            ka[2] = fp4_pair<2>(pp[g].k[s], sk);
            ka[3] = fp4_pair<3>(pp[g].k[s], sk);
#pragma unroll
            for (int t = 0; t < NT; ++t)
              S[g][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, ka),
                                                                qop[t][s], S[g][t], 0, 0, 0);
          }
        }
        u32x4 pb[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          float lm = NEG_INF;
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            if (valid[g] != kPageTokens - 1) {
#pragma unroll
              for (int i = 0; i < 4; ++i)
                if (4 * kg + i > valid[g]) S[g][t][i] = NEG_INF;
            }
            if constexpr (CAUSAL) {
              const int thr = cl[t] - kPageTokens * (2 * p + g);
              if (cm) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                  if (i > thr) S[g][t][i] = NEG_INF;
              }
            }
            lm = fmaxf(lm, fmaxf(fmaxf(S[g][t][0], S[g][t][1]), fmaxf(S[g][t][2], S[g][t][3])));
          }
          lm *= a.scale_log2;
          if (__any(lm > m[t] + kTau)) {
            const float mn = fmaxf(m[t], quad_max(lm));
            const float alpha = mn == NEG_INF ? 1.f : exp2_(m[t] - mn);
            m[t] = mn;
            l[t] *= alpha;
#pragma unroll
            for (int n = 0; n < C::NB; ++n) O[t][n] *= alpha;
          }
          const float nm = m[t] == NEG_INF ? 0.f : -m[t];
          float e[2][4];
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) e[g][i] = exp2_(fmaf(S[g][t][i], a.scale_log2, nm));
          l[t] += ((e[0][0] + e[0][1]) + (e[0][2] + e[0][3])) +
                  ((e[1][0] + e[1][1]) + (e[1][2] + e[1][3]));
#pragma unroll
          for (int g = 0; g < 2; ++g)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              bf16x2_t x;
              x[0] = (__bf16)e[g][2 * i];
              x[1] = (__bf16)e[g][2 * i + 1];
              pb[t][2 * g + i] = __builtin_bit_cast(unsigned, x);
            }
        }
        // V: byte B of token j's slice holds channels 2 B and 2 B + 1; tile i of O^T has channel i
        // of every lane's slice.
        auto vtiles = [&](auto bt) {
          constexpr int B = decltype(bt)::value;
          u32x4 va[2];
#pragma unroll
          for (int g = 0; g < 2; ++g) {
            unsigned x[4];
            if constexpr (D == 128) {
              x[0] = fp4_pair<B>(pp[g].v[0], fp4_exp<0>(pp[g].vs));
              x[1] = fp4_pair<B>(pp[g].v[1], fp4_exp<1>(pp[g].vs));
              x[2] = fp4_pair<B>(pp[g].v[2], fp4_exp<2>(pp[g].vs));
              x[3] = fp4_pair<B>(pp[g].v[3], fp4_exp<3>(pp[g].vs));
            } else {
              x[0] = fp4_pair<B>(pp[g].v[0], fp4_exp<0>(pp[g].vs));
              x[1] = fp4_pair<B + 2>(pp[g].v[0], fp4_exp<1>(pp[g].vs));
              x[2] = fp4_pair<B>(pp[g].v[1], fp4_exp<2>(pp[g].vs));
              x[3] = fp4_pair<B + 2>(pp[g].v[1], fp4_exp<3>(pp[g].vs));
            }
            va[0][2 * g] = __builtin_amdgcn_perm(x[1], x[0], 0x05040100);
            va[0][2 * g + 1] = __builtin_amdgcn_perm(x[3], x[2], 0x05040100);
            va[1][2 * g] = __builtin_amdgcn_perm(x[1], x[0], 0x07060302);
            va[1][2 * g + 1] = __builtin_amdgcn_perm(x[3], x[2], 0x07060302);
          }
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int t = 0; t < NT; ++t)
              O[t][2 * B + i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  __builtin_bit_cast(bf16x8, va[i]), __builtin_bit_cast(bf16x8, pb[t]),
                  O[t][2 * B + i], 0, 0, 0);
        };
        vtiles(std::integral_constant<int, 0>{});
        vtiles(std::integral_constant<int, 1>{});
        if constexpr (D == 128) {
          vtiles(std::integral_constant<int, 2>{});
          vtiles(std::integral_constant<int, 3>{});
        }
      };
      for (int p = split; p < npairs; p += PF * ks) {
#pragma unroll
        for (int i = 0; i < PF; ++i) {
          const int x = p + ks * i;
          __builtin_amdgcn_sched_barrier(0);         // (nothing of a pair is touched before its turn)
          if (x < npairs) pair(buf[i], x);
          load_pair(buf[i], x + PF * ks);
        }
      }

      // End of the pass.
      if (wave == 0) wait_vmcnt(0);                  // (the next descriptor)
      int lane_e = lane;
      asm volatile("" : "+v"(lane_e));
      const int re = lane_e & 15, ke = lane_e >> 4;
      if (ks == 1) {
        // A wave that saw every page writes its rows itself: D / 4 consecutive columns a lane, column
        // e D / 16 + n of them in O[n][e].
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const int r = tile_of(grp, t) * 16 + re;
          const float L = quad_sum(l[t]);
          const float inv = L > 0.f ? 1.f / L : 0.f;
          const float lam = m[t] + log2_(L);
          float amax = 0.f;
          if (!a.out) {
#pragma unroll
            for (int n = 0; n < C::NB; ++n)
#pragma unroll
              for (int e = 0; e < 4; ++e) amax = fmaxf(amax, fabsf(O[t][n][e]));
            amax = quad_max(amax) * inv;
          }
          if (r < R) {
            const int gr = row0 + r;
            const int j = gr / a.group;
            const int h = kvh * a.group + (gr - j * a.group);
            if (a.out) {
              const int64_t orow = (int64_t)dsc[br_word + j - j0] * a.Hq + h;
              __bf16* dst = static_cast<__bf16*>(a.out) + orow * D + ke * (D / 4);
#pragma unroll
              for (int x = 0; x < D / 32; ++x) {
                bf16x8 v;
#pragma unroll
                for (int i = 0; i < 8; ++i)
                  v[i] = (__bf16)(O[t][(8 * x + i) % C::NB][(8 * x + i) / C::NB] * inv);
                *reinterpret_cast<bf16x8*>(dst + 8 * x) = v;
              }
              if (ke == 0) a.lse[orow] = lam * 0.69314718055994531f;
            } else {
              const int64_t prow = ((int64_t)prow_base + j) * a.Hq + h;
              const int e = max(__builtin_amdgcn_frexp_expf(amax), -100);
              const float up = __builtin_amdgcn_ldexpf(inv, kPartScaleBits - e);
              _Float16* dst = static_cast<_Float16*>(a.po) + prow * D;
              if constexpr (D == 128) {
                // Position 32 ke + 16 (x / 2) + 8 (x % 2) ..: columns 8 (x / 2) + 4 (x % 2) ..+ 3 of the
                // lane's, then those 16 further.
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                  f16x8 v;
#pragma unroll
                  for (int i = 0; i < 4; ++i) {
                    v[i] = (_Float16)(O[t][4 * (x & 1) + i][x >> 1] * up);
                    v[4 + i] = (_Float16)(O[t][4 * (x & 1) + i][(x >> 1) + 2] * up);
                  }
                  store_dev16(reinterpret_cast<f16x8*>(dst + 32 * ke + 8 * x), v);
                }
              } else {
                // Position 32 (ke / 2) + 8 x + 4 (ke % 2) ..: columns 4 x ..+ 3 of the lane's.
                typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                  f16x4 v;
#pragma unroll
                  for (int i = 0; i < 4; ++i) v[i] = (_Float16)(O[t][i][x] * up);
                  store_dev8(reinterpret_cast<f32x2*>(dst + 32 * (ke >> 1) + 8 * x + 4 * (ke & 1)),
                             __builtin_bit_cast(f32x2, v));
                }
              }
              if (ke == 0)
                store_dev8(reinterpret_cast<f32x2*>(a.plse + 2 * prow),
                           f32x2{lam, __builtin_amdgcn_ldexpf(1.f, e - kPartScaleBits)});
            }
          }
        }
        return;
      }
      // Otherwise tile t of every wave goes to LDS, and the threads join the splits' parts and write the
      // rows, D / 8 threads a row.
      const int nrounds = min(MAXNT, (nrt - tile0 + ng - 1) / ng);
#pragma unroll
      for (int t = 0; t < MAXNT; ++t) {
        if (t >= nrounds) break;
        lds_barrier();                               // the round before is read
        if (t < NT) {
          const int tt = t < NT ? t : 0;
          const float L = quad_sum(l[tt]);
          if (ke == 0) {
            s_m[wave][re] = m[tt];
            s_l[wave][re] = L;
          }
          float* so = s_o[wave] + re * D;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
#pragma unroll
            for (int c = 0; c < C::NB / 4; ++c) {
              // columns ke D / 4 + e D / 16 + 4 c .. + 3
              const int ch = ke * (D / 16) + e * (D / 64) + c;
              f32x4 x;
#pragma unroll
              for (int i = 0; i < 4; ++i) x[i] = O[tt][4 * c + i][e];
              *reinterpret_cast<f32x4*>(so + 4 * (ch ^ re)) = x;
            }
          }
        }
        lds_barrier();
        constexpr int TPR = D / 8;                   // threads of a row
        const int tasks = ng * 16 * TPR;
        for (int x = tid; x < tasks; x += kAttnThreads) {
          const int row = (x / TPR) & 15, gq = x / (16 * TPR), pc = x % TPR;
          const int r = tile_of(gq, t) * 16 + row;
          if (r < R) {                               // (the threads of a row go together)
            float M = NEG_INF;
            for (int s = 0; s < ks; ++s) M = fmaxf(M, s_m[gq + ng * s][row]);
            const float Ms = M == NEG_INF ? 0.f : M;
            float L = 0.f;
            f32x4 o0 = {0.f, 0.f, 0.f, 0.f}, o1 = {0.f, 0.f, 0.f, 0.f};
            // Partial rows: position 8 pc .. + 7 of the row holds two runs of four columns
            // (ga_internal.hpp); output rows: eight columns.
            const int c0 = a.out ? 2 * pc : 8 * (pc >> 2) + (pc & 3);
            const int c1 = a.out ? 2 * pc + 1 : c0 + 4;
            for (int s = 0; s < ks; ++s) {
              const int wv = gq + ng * s;
              const float wgt = exp2_(s_m[wv][row] - Ms);
              L += wgt * s_l[wv][row];
              const float* so = s_o[wv] + row * D;
              o0 += wgt * *reinterpret_cast<const f32x4*>(so + 4 * (c0 ^ row));
              o1 += wgt * *reinterpret_cast<const f32x4*>(so + 4 * (c1 ^ row));
            }
            // A row that saw no token of the chunk (multi-query) has o = 0, lambda = -inf.
            const float inv = L > 0.f ? 1.f / L : 0.f;
            const float lam = M + log2_(L);
            const int gr = row0 + r;
            const int j = gr / a.group;
            const int h = kvh * a.group + (gr - j * a.group);
            if (a.out) {
              const int64_t orow = (int64_t)dsc[br_word + j - j0] * a.Hq + h;
              bf16x8 v;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                v[i] = (__bf16)(o0[i] * inv);
                v[4 + i] = (__bf16)(o1[i] * inv);
              }
              *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(a.out) + orow * D + 8 * pc) = v;
              if (pc == 0) a.lse[orow] = lam * 0.69314718055994531f;
            } else {
              const int64_t prow = ((int64_t)prow_base + j) * a.Hq + h;
              float amax = 0.f;
#pragma unroll
              for (int i = 0; i < 4; ++i) amax = fmaxf(amax, fmaxf(fabsf(o0[i]), fabsf(o1[i])));
#pragma unroll
              for (int s = 1; s < TPR; s *= 2) amax = fmaxf(amax, __shfl_xor(amax, s));
              amax *= inv;
              const int e = max(__builtin_amdgcn_frexp_expf(amax), -100);
              const float up = __builtin_amdgcn_ldexpf(inv, kPartScaleBits - e);
              f16x8 v;
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                v[i] = (_Float16)(o0[i] * up);
                v[4 + i] = (_Float16)(o1[i] * up);
              }
              store_dev16(reinterpret_cast<f16x8*>(static_cast<_Float16*>(a.po) + prow * D + 8 * pc), v);
              if (pc == 0)
                store_dev8(reinterpret_cast<f32x2*>(a.plse + 2 * prow),
                           f32x2{lam, __builtin_amdgcn_ldexpf(1.f, e - kPartScaleBits)});
            }
          }
        }
      }
    };
    const std::integral_constant<int, 1> one{};
    if constexpr (MAXNT == 1) {
      const int ng = nrt <= 2 ? nrt : 4;
      for (int t0 = 0; t0 < nrt; t0 += ng)
        if (t0 + wave % ng < nrt) run_pass(one, ng, t0);
    } else {
      const int ng = nrt <= 2 ? 1 : nrt <= 4 ? 2 : 4;
      if (wave % ng + ng < nrt) run_pass(std::integral_constant<int, 2>{}, ng, 0);
      else run_pass(one, ng, 0);
    }
    first = false;
    lds_barrier();        // the rows are read from LDS, and nothing needs this unit's descriptor
  }
  // The work-stream heads are armed again by the merge, or, without one, by the last workgroup.
  if (a.out && tid == 0) {
    const int n_done = (int)__hip_atomic_fetch_add(reinterpret_cast<int*>(a.counters + 2), 1,
                                                   __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    if (n_done == (int)gridDim.x - 1) {
      for (int i = 0; i < kMaxStreams; ++i) heads[i] = 0;
      a.counters[2] = 0;
    }
  }
}

template <int D>
hipError_t launch_t(const AttnArgs& a, bool causal, int grid, hipStream_t stream, hipEvent_t t0,
                    hipEvent_t t1) {
  auto go = [&](auto kernel) {
    if (t0 || t1)
      hipExtLaunchKernelGGL(kernel, dim3(grid), dim3(kAttnThreads), 0, stream, t0, t1, 0, a);
    else
      hipLaunchKernelGGL(kernel, dim3(grid), dim3(kAttnThreads), 0, stream, a);
  };
  if (a.few_rows) {
    if (causal) go(k_fp4_attn<D, true, 1>);
    else go(k_fp4_attn<D, false, 1>);
  } else {
    if (causal) go(k_fp4_attn<D, true, 2>);
    else go(k_fp4_attn<D, false, 2>);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_fp4_attn(const AttnArgs& a, int head_dim, bool causal, int grid,
                           hipStream_t stream, hipEvent_t t0, hipEvent_t t1) {
  if (head_dim == 64) return launch_t<64>(a, causal, grid, stream, t0, t1);
  if (head_dim == 128) return launch_t<128>(a, causal, grid, stream, t0, t1);
  return hipErrorInvalidValue;
}

}  // namespace ga
