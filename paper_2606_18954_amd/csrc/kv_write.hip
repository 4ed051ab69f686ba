// Page-pool writes: storing new tokens' K and V in page slots (append) and moving tokens between
// page slots (copy); for MXFP4 pools also reading tokens back (read).
//
// A decode step extends every active branch's newest segment by the token it produced, and a
// state's continuation is split into step segments (Alg. S.1, Stage 1).  Since every segment
// starts at slot 0 of a page of its own, forking a state into children needs no copy (each child
// opens new pages); moving the tokens after a cut inside a page to fresh pages does.
//
// A slot word w names page w / 16, slot w % 16.  One thread moves 16 bytes: token j's data is
// Hkv x 2 x ROW bytes (ROW = D x element size), and piece p of it is kv-head p / (2 PR), K or V
// (p / PR) % 2, 16-byte chunk p % PR of the token row (PR = ROW / 16), so consecutive threads
// read and write contiguous runs of a row.  Words outside [0, num_pages x 16) skip the token:
// nothing outside the pool is ever written.
//
// MXFP4 pools: one thread takes 8 channels (16 bytes of bf16, 4 of codes), four threads a block of 32
// with its scale.  Append: a = max |x| over the block (two exchanges between the four lanes), e =
// floor(log2 a) - 2, one more where a >= 7 x 2^e (6 2^e is the largest value, and 7 2^e the border up to
// which rounding to it is as near as to the next one: no value is clipped by more than a rounding),
// kept in [-125, 125] so that every value of the block is a normal float32; x / 2^e is rounded to the
// nearest code, ties to the even one, by the conversion instruction.  A block with a NaN or an
// infinity has scale byte 255 and reads as NaN.  (Only the largest exponent leaves a value outside: from
// 7 x 2^125 on it becomes 6 x 2^125.)  Memory bounds it: 32768 tokens of 8 heads x 128, 169 MB and 27 us at
// 6.2 TB/s, in the order in which a prompt's tokens lie (whole pages, at random places) append 40.1 us, read 30.3,
// copy 25.8; with every token at a random slot 45.9, 38.3 and 44.3.  There V's runs of 4 bytes fill a quarter of
// the 64-byte pieces that reach memory: the append writes 98 MB where 36 are new, and moves 233 MB in all at
// 5.1 TB/s.  (The choices below were measured on random slots.)  The bf16 rows pass the caches by
// (non-temporal), so that a page's lines, which four tokens' V share, stay until all have come: with ordinary
// loads and stores append and read take 96 us, not 82.  Two tokens a thread (82 us) hide the latency of the
// words better than one (85) and leave a step's 1024 tokens more workgroups than four (a step's append and read
// 10.4 us, 12.0 with four).
#include "ga_internal.hpp"
#include "mxfp4.hpp"
#include "pool_load.hpp"

namespace ga {
namespace {

__device__ __forceinline__ int64_t slot_offset(int32_t w, int h, int kv, int Hkv, int row_bytes) {
  return ((((int64_t)(w >> 4) * Hkv + h) * 2 + kv) * kPageTokens + (w & 15)) * row_bytes;
}

__global__ __launch_bounds__(256) void k_kv_write(KvWriteArgs a) {
  const int64_t gid = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int pr = a.row_bytes / 16;
  const int ppt = a.Hkv * 2 * pr;
  const int64_t j = gid / ppt;
  if (j >= a.n) return;
  const int p = (int)(gid - j * ppt);
  const int h = p / (2 * pr), kv = (p / pr) & 1, c = p % pr;
  const int32_t dw = a.dst_words[j];
  if (dw < 0 || (int64_t)dw >= a.num_slots) return;
  const uint4* src;
  if (a.src_words) {
    const int32_t sw = a.src_words[j];
    if (sw < 0 || (int64_t)sw >= a.num_slots) return;
    src = reinterpret_cast<const uint4*>(a.pool + slot_offset(sw, h, kv, a.Hkv, a.row_bytes) +
                                         16 * c);
  } else {
    const unsigned char* base = kv ? a.v_new : a.k_new;
    src = reinterpret_cast<const uint4*>(base + (j * a.Hkv + h) * a.row_bytes + 16 * c);
  }
  *reinterpret_cast<uint4*>(a.pool + slot_offset(dw, h, kv, a.Hkv, a.row_bytes) + 16 * c) = *src;
}

// MODE 0: append, 1: copy, 2: read.  A thread takes 8 channels of kPieces tokens' K or V, which D / 8 threads
// share: each kind of load is issued for all of them before the first is used.
constexpr int kPieces = 2;

template <int D, int MODE>
__global__ __launch_bounds__(256) void k_kv_fp4(KvWriteArgs a) {
  constexpr int PR = D / 8, UB = 256 / PR;           // threads of a token's K or V, of which a block has UB
  const int per = 2 * a.Hkv, c = 8 * ((int)threadIdx.x % PR);
  const int64_t first = (int64_t)blockIdx.x * (kPieces * UB), j0 = first / per;
  const unsigned r0 = (unsigned)(first - j0 * per) + threadIdx.x / PR;
  int64_t row[kPieces];                              // of k_new / v_new, k_out / v_out
  int h[kPieces];
  bool v[kPieces], ok[kPieces];
  int32_t dw[kPieces], sw[kPieces];
  u32x4 x[kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const unsigned r = r0 + i * UB, dj = r / (unsigned)per, hv = r - dj * per;
    const int64_t j = j0 + dj;
    ok[i] = j < a.n;                                 // (the four lanes of a block go together)
    h[i] = (int)(hv >> 1);
    v[i] = hv & 1;
    row[i] = ((j * a.Hkv + h[i]) * D + c) * 2;
    dw[i] = ok[i] ? a.dst_words[j] : -1;
    if constexpr (MODE == 1) sw[i] = ok[i] ? a.src_words[j] : -1;
    if constexpr (MODE == 0)
      if (ok[i])
        x[i] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>((v[i] ? a.v_new : a.k_new) + row[i]));
  }
  auto block = [&](int32_t w, int i) {
    return a.pool + ((int64_t)(w >> 4) * a.Hkv + h[i]) * Fp4<D>::PAGE;
  };
  unsigned code[kPieces], byte[kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    ok[i] = dw[i] >= 0 && (int64_t)dw[i] < a.num_slots;
    if constexpr (MODE == 1) ok[i] = ok[i] && sw[i] >= 0 && (int64_t)sw[i] < a.num_slots;
    if constexpr (MODE != 0)
      if (ok[i]) {
        const int32_t w = MODE == 1 ? sw[i] : dw[i];
        const unsigned char* src = block(w, i);
        code[i] = load_codes<D>(src, w & 15, c, v[i]);
        byte[i] = src[fp4_scale<D>(w & 15, c, v[i])];
      }
  }
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    if (!ok[i]) continue;
    if constexpr (MODE == 0) {
      const unsigned w[4] = {x[i][0], x[i][1], x[i][2], x[i][3]};
      fp4_round(w, &code[i], &byte[i]);
    }
    if constexpr (MODE != 2) {
      unsigned char* dst = block(dw[i], i);
      store_codes<D>(dst, dw[i] & 15, c, v[i], code[i]);
      if ((c & 31) == 0) dst[fp4_scale<D>(dw[i] & 15, c, v[i])] = (unsigned char)byte[i];
    } else {
      const float s = __builtin_bit_cast(float, byte[i] << 23);
      __builtin_nontemporal_store(u32x4{fp4_pair<0>(code[i], s), fp4_pair<1>(code[i], s),
                                        fp4_pair<2>(code[i], s), fp4_pair<3>(code[i], s)},
                                  reinterpret_cast<u32x4*>((v[i] ? a.v_out : a.k_out) + row[i]));
    }
  }
}

// Reading a token of a pool of the other types.
__global__ __launch_bounds__(256) void k_kv_read(KvWriteArgs a) {
  const int64_t gid = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int pr = a.row_bytes / 16;
  const int ppt = a.Hkv * 2 * pr;
  const int64_t j = gid / ppt;
  if (j >= a.n) return;
  const int p = (int)(gid - j * ppt);
  const int h = p / (2 * pr), kv = (p / pr) & 1, c = p % pr;
  const int32_t w = a.dst_words[j];
  if (w < 0 || (int64_t)w >= a.num_slots) return;
  *reinterpret_cast<uint4*>((kv ? a.v_out : a.k_out) + (j * a.Hkv + h) * a.row_bytes + 16 * c) =
      *reinterpret_cast<const uint4*>(a.pool + slot_offset(w, h, kv, a.Hkv, a.row_bytes) + 16 * c);
}

template <int D>
void launch_fp4(const KvWriteArgs& a, unsigned grid, hipStream_t stream) {
  if (a.k_out)
    hipLaunchKernelGGL((k_kv_fp4<D, 2>), dim3(grid), dim3(256), 0, stream, a);
  else if (a.src_words)
    hipLaunchKernelGGL((k_kv_fp4<D, 1>), dim3(grid), dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((k_kv_fp4<D, 0>), dim3(grid), dim3(256), 0, stream, a);
}

}  // namespace

hipError_t launch_kv_write(const KvWriteArgs& a, hipStream_t stream) {
  const int64_t threads = (int64_t)a.n * a.Hkv * 2 * (a.fp4_dim ? a.fp4_dim / 8 : a.row_bytes / 16);
  const int64_t block = a.fp4_dim ? 256 * kPieces : 256;
  const int64_t grid = (threads + block - 1) / block;
  if (grid == 0) return hipSuccess;
  if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
  if (a.fp4_dim == 64) launch_fp4<64>(a, (unsigned)grid, stream);
  else if (a.fp4_dim) launch_fp4<128>(a, (unsigned)grid, stream);
  else if (a.k_out) hipLaunchKernelGGL(k_kv_read, dim3((unsigned)grid), dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(k_kv_write, dim3((unsigned)grid), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ga
