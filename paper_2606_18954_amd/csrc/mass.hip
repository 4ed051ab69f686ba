// Attention mass of cached tokens: for every slot w of the plan's segments
//   out[w] = decay in[w] + sum over the query rows r that see w, and their q-heads h, of
//            exp(scale q[r,h] . k[w] - lse[r,h]),
// the softmax weights of a step that has been attended (lse is its result), summed per token.
//
// A slot belongs to one chain, so one workgroup that takes some pages of a chain with all of its rows
// and all kv-heads owns those slots: no atomics, one order of the sums, the same bits every time.  The
// pages' K operands sit in registers (bf16; float32 for float32 pools) while the rows' queries stream
// past:  S = K Q^T in 16 x 16 tiles, p = 2^(S scale log2 e - lse log2 e), and each lane adds the p of its
// four tokens over its share of the rows.  The waves of a workgroup take different kv-heads first,
// and different rows where heads are few.
#include "attn_dev.hpp"
#include "evict_internal.hpp"
#include "mxfp4.hpp"

namespace ga {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

template <int D, int TYPE>
struct MCfg {
  static constexpr bool F32 = TYPE == GA_F32;
  static constexpr int PG = F32 ? 2 : 4;            // pages of a unit
  static constexpr int ELT = F32 ? 4 : 2;
  static constexpr int OPS = F32 ? D / 4 : D / 32;  // contraction steps
  static constexpr int HEAD = TYPE == GA_MXFP4 ? 17 * D : 32 * D * ELT;   // bytes of a page's head
};
template <bool F32> struct Op;
template <> struct Op<true> { float v; };
template <> struct Op<false> { bf16x8 v; };

// The lane's operand of one row of K or Q: channels kg D / 4 ..+ D / 4 - 1, in order.
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

template <int D, int TYPE>
__global__ __launch_bounds__(256) void k_mass(MassArgs a) {
  using C = MCfg<D, TYPE>;
  __shared__ float s_mass[4][C::PG * 16];
  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r16 = lane & 15, kg = lane >> 4;
  const float NEG_INF = -__builtin_huge_valf();
  const int hs = a.Hkv >= 4 ? 4 : a.Hkv >= 2 ? 2 : 1;     // waves that take different kv-heads
  const int rs = 4 / hs;                                  // waves that share a head's rows
  const unsigned char* pool = static_cast<const unsigned char*>(a.pool);
  const unsigned char* q = static_cast<const unsigned char*>(a.q);
  const int gpc = (a.chunk_pages + C::PG - 1) / C::PG;
  const int64_t total = a.counters[0] * gpc;
  const unsigned magic = (unsigned)(0xffffffffu / (unsigned)a.group);

  for (int64_t u = blockIdx.x; u < total; u += gridDim.x) {
    const int64_t item = u / gpc;
    const int pg0 = (int)(u - item * gpc) * C::PG;
    const int32_t* d = a.desc + item * a.desc_words;
    const int np = d[0], cw = d[1], cnt = d[3];
    const int goff = d[5];
    if (d[4] != 0 || pg0 >= np) continue;             // (the first row block's item takes all rows)
    const int npg = min(C::PG, np - pg0);
    const bool cm = a.causal && cw != kNoCausal;
    const int rows = cnt * a.group;
    int t0 = 0;                                       // the first tile with a row that sees the pages
    if (cm) t0 = (int)(((int64_t)max(0, kPageTokens * pg0 - cw) * a.group) >> 4);
    float acc[C::PG][4];
#pragma unroll
    for (int g = 0; g < C::PG; ++g)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[g][i] = 0.f;
    for (int h = wave % hs; h < a.Hkv; h += hs) {
      // K: token r16 of every page.  (A slot past the segment's end may hold anything: only its own
      // sums see it, and they are not stored.)
      Op<C::F32> ka[C::PG][C::OPS];
#pragma unroll
      for (int g = 0; g < C::PG; ++g) {
        const int word = d[kDescHead + pg0 + min(g, npg - 1)];
        const unsigned char* base =
            pool + ((int64_t)(word & kPageIdMask) * a.Hkv + h) * C::HEAD;
        if constexpr (TYPE == GA_MXFP4) {
          const float sk = __builtin_bit_cast(
              float, (unsigned)base[Fp4<D>::KS + r16 * Fp4<D>::NS + (kg * (D / 4)) / 32] << 23);
#pragma unroll
          for (int s = 0; s < D / 32; ++s) {
            const unsigned w =
                *reinterpret_cast<const unsigned*>(base + r16 * (D / 2) + kg * (D / 8) + 4 * s);
            const u32x4 x = {fp4_pair<0>(w, sk), fp4_pair<1>(w, sk), fp4_pair<2>(w, sk),
                             fp4_pair<3>(w, sk)};
            ka[g][s].v = __builtin_bit_cast(bf16x8, x);
          }
        } else {
          load_row<D, C::F32>(ka[g], base + r16 * D * C::ELT, kg);
        }
      }
      const int ntile = (rows + 15) >> 4;
      for (int t = t0 + wave / hs; t < ntile; t += rs) {
        const int r = 16 * t + r16;
        const bool live = r < rows;
        // r / group: the truncated reciprocal is at most one short
        const unsigned rr = (unsigned)min(r, rows - 1);
        int j = (int)__umulhi(rr, magic);
        int gi = (int)rr - j * a.group;
        if (gi >= a.group) { gi -= a.group; ++j; }
        const int64_t row = (int64_t)a.grp_br[goff + j] * a.Hq + h * a.group + gi;
        Op<C::F32> qo[C::OPS];
        load_row<D, C::F32>(qo, q + row * D * C::ELT, kg);
        const float lse = a.lse[row];
        // (a row without any weight counts for nothing)
        const float nl = live && fabsf(lse) != -NEG_INF ? -1.4426950408889634f * lse : NEG_INF;
        f32x4 S[C::PG];
#pragma unroll
        for (int g = 0; g < C::PG; ++g) S[g] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < C::OPS; ++s)
#pragma unroll
          for (int g = 0; g < C::PG; ++g) {
            if constexpr (C::F32)
              S[g] = __builtin_amdgcn_mfma_f32_16x16x4f32(ka[g][s].v, qo[s].v, S[g], 0, 0, 0);
            else
              S[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ka[g][s].v, qo[s].v, S[g], 0, 0, 0);
          }
        const int lim = cm ? cw + j - kPageTokens * pg0 - 4 * kg : 0x3fffffff;
#pragma unroll
        for (int g = 0; g < C::PG; ++g)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float p = exp2_(fmaf(S[g][i], a.scale_log2, nl));
            acc[g][i] += kPageTokens * g + i <= lim ? p : 0.f;
          }
      }
    }
#pragma unroll
    for (int g = 0; g < C::PG; ++g)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x = acc[g][i];
#pragma unroll
        for (int s = 1; s < 16; s *= 2) x += __shfl_xor(x, s);
        if (r16 == 0) s_mass[wave][16 * g + 4 * kg + i] = x;
      }
    __syncthreads();
    if (tid < C::PG * 16 && tid / 16 < npg) {
      const int word = d[kDescHead + pg0 + tid / 16];
      if ((tid & 15) <= (int)((unsigned)word >> kPageValidShift)) {
        const int64_t slot = (int64_t)(word & kPageIdMask) * kPageTokens + (tid & 15);
        const float sum = (s_mass[0][tid] + s_mass[1][tid]) + (s_mass[2][tid] + s_mass[3][tid]);
        a.mass_out[slot] = a.mass_in ? fmaf(a.decay, a.mass_in[slot], sum) : sum;
      }
    }
    __syncthreads();
  }
}

template <int D>
hipError_t launch_t(const MassArgs& a, hipStream_t stream) {
  auto go = [&](auto kernel, int pages) {
    const int64_t most = a.units * ((a.chunk_pages + pages - 1) / pages);
    const int64_t grid = most < 8LL * a.num_cus ? most : 8LL * a.num_cus;
    hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(256), 0, stream, a);
  };
  if (a.dtype == GA_F32) go(k_mass<D, GA_F32>, MCfg<D, GA_F32>::PG);
  else if (a.dtype == GA_BF16) go(k_mass<D, GA_BF16>, MCfg<D, GA_BF16>::PG);
  else go(k_mass<D, GA_MXFP4>, MCfg<D, GA_MXFP4>::PG);
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
