// Loads of a page by a wave: a buffer resource in scalar registers (the page) and 32-bit offsets in the
// lanes.  The page's address then costs scalar instructions only, where 64-bit lane addresses would cost
// a vector addition per load; a pool pointer rebuilt from scalar registers would even become a flat
// address, whose loads are waited for one by one.
#pragma once

#include "ga_internal.hpp"

namespace ga {
namespace {

typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
typedef __amdgpu_buffer_rsrc_t page_t;

// `bytes` of memory at `base` (the same in every lane).
__device__ __forceinline__ page_t page_at(const unsigned char* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<unsigned char*>(base), 0, bytes, 0x00020000);
}
__device__ __forceinline__ u32x4 load16(page_t p, unsigned off) {
  return __builtin_amdgcn_raw_buffer_load_b128(p, off, 0, 0);
}
__device__ __forceinline__ u32x2 load8(page_t p, unsigned off) {
  return __builtin_amdgcn_raw_buffer_load_b64(p, off, 0, 0);
}
__device__ __forceinline__ unsigned load4(page_t p, unsigned off) {
  return __builtin_amdgcn_raw_buffer_load_b32(p, off, 0, 0);
}

}  // namespace
}  // namespace ga
