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
// infinity has scale byte 255 and reads as NaN.
#include "ga_internal.hpp"
#include "mxfp4.hpp"

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

// The codes of 8 channels from c on, in a page block.
template <int D>
__device__ __forceinline__ unsigned load_codes(const unsigned char* blk, int t, int c, bool v) {
  if constexpr (D == 128) {
    return *reinterpret_cast<const unsigned*>(blk + fp4_code<D>(t, c, v));
  } else {
    // (K: both halves side by side; V: two slices of four channels)
    const unsigned lo = *reinterpret_cast<const unsigned short*>(blk + fp4_code<D>(t, c, v));
    const unsigned hi = *reinterpret_cast<const unsigned short*>(blk + fp4_code<D>(t, c + 4, v));
    return lo | (hi << 16);
  }
}
template <int D>
__device__ __forceinline__ void store_codes(unsigned char* blk, int t, int c, bool v, unsigned w) {
  if constexpr (D == 128) {
    *reinterpret_cast<unsigned*>(blk + fp4_code<D>(t, c, v)) = w;
  } else {
    *reinterpret_cast<unsigned short*>(blk + fp4_code<D>(t, c, v)) = (unsigned short)w;
    *reinterpret_cast<unsigned short*>(blk + fp4_code<D>(t, c + 4, v)) = (unsigned short)(w >> 16);
  }
}

// MODE 0: append, 1: copy, 2: read.
template <int D, int MODE>
__global__ __launch_bounds__(256) void k_kv_fp4(KvWriteArgs a) {
  const int64_t gid = (int64_t)blockIdx.x * 256 + threadIdx.x;
  constexpr int PR = D / 8;                          // threads of a token's K or V
  const int ppt = a.Hkv * 2 * PR;
  const int64_t j = gid / ppt;
  if (j >= a.n) return;
  const int p = (int)(gid - j * ppt);
  const int h = p / (2 * PR), c = 8 * (p % PR);
  const bool v = (p / PR) & 1;
  const int32_t dw = a.dst_words[j];
  if (dw < 0 || (int64_t)dw >= a.num_slots) return;  // (the four lanes of a block go together)
  unsigned char* dst = a.pool + ((int64_t)(dw >> 4) * a.Hkv + h) * Fp4<D>::PAGE;
  const int td = dw & 15;
  const int64_t row = ((j * a.Hkv + h) * D + c) * 2; // of k_new / v_new, k_out / v_out
  if constexpr (MODE == 0) {
    const uint4 x = *reinterpret_cast<const uint4*>((v ? a.v_new : a.k_new) + row);
    const unsigned w[4] = {x.x, x.y, x.z, x.w};
    // bf16 magnitudes order like the integers they are.
    unsigned top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = max(top, max(w[i] & 0x7fffu, (w[i] >> 16) & 0x7fffu));
    top = max(top, (unsigned)__shfl_xor((int)top, 1));
    top = max(top, (unsigned)__shfl_xor((int)top, 2));
    // Exponent of a, plus one from mantissa 0.75 on; two below it is the scale.
    int byte = (int)((top + 0x20u) >> 7) - 2;
    byte = top >= 0x7f80u ? 255 : min(max(byte, 2), 252);
    unsigned code = 0;
    if (byte != 255) {
      const float s = __builtin_bit_cast(float, (unsigned)byte << 23);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2_t, w[0]), s, 0);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2_t, w[1]), s, 1);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2_t, w[2]), s, 2);
      code = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(code, __builtin_bit_cast(bf16x2_t, w[3]), s, 3);
    }
    store_codes<D>(dst, td, c, v, code);
    if ((c & 31) == 0) dst[fp4_scale<D>(td, c, v)] = (unsigned char)byte;
  } else if constexpr (MODE == 1) {
    const int32_t sw = a.src_words[j];
    if (sw < 0 || (int64_t)sw >= a.num_slots) return;
    const unsigned char* src = a.pool + ((int64_t)(sw >> 4) * a.Hkv + h) * Fp4<D>::PAGE;
    const int ts = sw & 15;
    store_codes<D>(dst, td, c, v, load_codes<D>(src, ts, c, v));
    if ((c & 31) == 0) dst[fp4_scale<D>(td, c, v)] = src[fp4_scale<D>(ts, c, v)];
  } else {
    const unsigned code = load_codes<D>(dst, td, c, v);
    const float s = __builtin_bit_cast(float, (unsigned)dst[fp4_scale<D>(td, c, v)] << 23);
    *reinterpret_cast<uint4*>((v ? a.v_out : a.k_out) + row) =
        make_uint4(fp4_pair<0>(code, s), fp4_pair<1>(code, s), fp4_pair<2>(code, s),
                   fp4_pair<3>(code, s));
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
  const int64_t grid = (threads + 255) / 256;
  if (grid == 0) return hipSuccess;
  if (grid > 0x7fffffffLL) return hipErrorInvalidValue;
  if (a.fp4_dim == 64) launch_fp4<64>(a, (unsigned)grid, stream);
  else if (a.fp4_dim) launch_fp4<128>(a, (unsigned)grid, stream);
  else if (a.k_out) hipLaunchKernelGGL(k_kv_read, dim3((unsigned)grid), dim3(256), 0, stream, a);
  else hipLaunchKernelGGL(k_kv_write, dim3((unsigned)grid), dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ga
