// The device side of HIP on the CPU, as far as this repository's kernels use it, for builds of the kernels'
// own sources under AddressSanitizer: device memory is host memory of exactly the size asked for, a launch
// runs its workgroups one after another, and a thread runs until it needs the others of its wave (a ballot, a
// shuffle, a matrix product) or of its workgroup (a barrier).  Which wave goes on next is drawn from a seed.
//
// A copy to LDS written as inline assembly (dma16) is done when it is issued, or, with emu::late_copies, when
// its wave waits for it (vmcnt(0)): the first shows a copy that comes too early for a reader of what was there,
// the second a missing wait.  What this cannot show are the hardware's own wait states.
#pragma once
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <functional>
#include <type_traits>

#define __host__
#define __device__
#define __global__
#define __shared__ static
#define __forceinline__ inline
#define __launch_bounds__(...)
#define __align__(n) __attribute__((aligned(n)))
#define __HIP_MEMORY_SCOPE_AGENT 0

struct dim3 {
  unsigned x, y, z;
  dim3(unsigned x_ = 1, unsigned y_ = 1, unsigned z_ = 1) : x(x_), y(y_), z(z_) {}
};
struct alignas(16) int4 { int x, y, z, w; };
struct alignas(8) int2 { int x, y; };
struct alignas(16) uint4 { unsigned x, y, z, w; };
struct alignas(8) uint2 { unsigned x, y; };
inline int4 make_int4(int x, int y, int z, int w) { return {x, y, z, w}; }
inline int2 make_int2(int x, int y) { return {x, y}; }
inline uint2 make_uint2(unsigned x, unsigned y) { return {x, y}; }

namespace emu {

constexpr int kWave = 64;
struct Lane {
  void* sp = nullptr;
  char* stack = nullptr;
  dim3 tid;
  enum State { kReady, kWaveOp, kBarrier, kDone } state = kDone;
  long key = 0;                    // of the wave operation it waits at
  void (*resolve)(Lane** group, int n) = nullptr;
  const void* in = nullptr;
  void* out = nullptr;
};
extern Lane* cur;                  // the running thread
extern dim3 block, grid, threads;
extern int num_cus;
extern bool late_copies;
extern uint64_t seed;
extern long partial_ops;           // wave operations that not all 64 lanes took part in
void yield();
void launch(dim3 grid, dim3 threads, size_t lds, const std::function<void()>& kernel);
void* dynamic_lds();
void dma16(unsigned off, const void* base, unsigned lds_base);
void wait(int imm);
[[noreturn]] void fail(const char* what);

// One operation of a wave: f(in of every lane or nullptr, out of every lane).
template <class In, class Out, void (*F)(const In* const*, Out* const*)>
void resolve(Lane** group, int n) {
  const In* in[kWave] = {};
  Out* out[kWave] = {};
  for (int i = 0; i < n; ++i) {
    const int l = group[i]->tid.x % kWave;
    in[l] = static_cast<const In*>(group[i]->in);
    out[l] = static_cast<Out*>(group[i]->out);
  }
  F(in, out);
}
template <class In, class Out, void (*F)(const In* const*, Out* const*)>
Out wave_op(long key, const In& in) {
  Out out{};
  cur->in = &in;
  cur->out = &out;
  cur->key = key;
  cur->resolve = &resolve<In, Out, F>;
  cur->state = Lane::kWaveOp;
  yield();
  return out;
}
inline void barrier() {
  cur->state = Lane::kBarrier;
  yield();
}
inline void all64(const void* const* in, const char* what) {
  for (int l = 0; l < kWave; ++l)
    if (!in[l]) fail(what);
}

template <class T> struct Two { T v; int x; };
template <class T> void f_first(const T* const* in, T* const* out) {
  T v{};
  for (int l = kWave - 1; l >= 0; --l) if (in[l]) v = *in[l];
  for (int l = 0; l < kWave; ++l) if (out[l]) *out[l] = v;
}
template <class T> void f_lane(const Two<T>* const* in, T* const* out) {   // the value of lane x
  for (int l = 0; l < kWave; ++l)
    if (in[l]) {
      const int s = in[l]->x & 63;
      if (!in[s]) fail("a lane that is not there is read");
      *out[l] = in[s]->v;
    }
}
inline void f_ballot(const bool* const* in, uint64_t* const* out) {
  uint64_t m = 0;
  for (int l = 0; l < kWave; ++l) if (in[l] && *in[l]) m |= 1ull << l;
  for (int l = 0; l < kWave; ++l) if (out[l]) *out[l] = m;
}
struct Dpp { int old, src, ctrl, rows; bool zero; };
inline int dpp_source(int ctrl, int l) {                   // -1: none
  const int r = l & 15;
  if (ctrl < 0x100) return (l & ~3) + ((ctrl >> (2 * (l & 3))) & 3);
  if (ctrl > 0x110 && ctrl < 0x120) return r >= ctrl - 0x110 ? l - (ctrl - 0x110) : -1;
  if (ctrl == 0x140) return (l & ~15) + 15 - r;
  if (ctrl == 0x141) return (l & ~7) + 7 - (l & 7);
  if (ctrl == 0x142) return l >= 16 ? (l & ~15) - 1 : -1;
  if (ctrl == 0x143) return l >= 32 ? 31 : -1;
  fail("dpp control");
}
inline void f_dpp(const Dpp* const* in, int* const* out) {
  all64(reinterpret_cast<const void* const*>(in), "dpp in a part of a wave");
  for (int l = 0; l < kWave; ++l) {
    const Dpp& d = *in[l];
    const int s = dpp_source(d.ctrl, l);
    if (!((d.rows >> (l / 16)) & 1)) *out[l] = d.old;
    else *out[l] = s >= 0 ? in[s]->src : d.zero ? 0 : d.old;
  }
}
typedef unsigned u32x2_ __attribute__((ext_vector_type(2)));
inline void together() { wave_op<int, int, f_first<int>>(0, 0); }
struct Swap { unsigned a, b; };
template <int H> void f_swap(const Swap* const* in, u32x2_* const* out) {  // odd rows of a, even rows of b
  all64(reinterpret_cast<const void* const*>(in), "swap in a part of a wave");
  for (int l = 0; l < kWave; ++l) {
    const bool odd = (l / H) & 1;
    (*out[l])[0] = odd ? in[l - H]->b : in[l]->a;
    (*out[l])[1] = odd ? in[l]->b : in[l + H]->a;
  }
}

// Matrix products: a lane's column (row of A, column of B), and its first contraction index.
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16 __attribute__((ext_vector_type(16)));
template <class A, class C> struct Mm { A a, b; C c; };
template <int M, int K, class A, class C, class Get>
void product(const Mm<A, C>* const* in, C* const* out, Get get) {
  all64(reinterpret_cast<const void* const*>(in), "matrix product in a part of a wave");
  float a[M][64], b[M][64];
  constexpr int G = kWave / M, E = K / G;
  for (int l = 0; l < kWave; ++l)
    for (int j = 0; j < E; ++j) {
      a[l % M][E * (l / M) + j] = get(in[l]->a, j);
      b[l % M][E * (l / M) + j] = get(in[l]->b, j);
    }
  for (int l = 0; l < kWave; ++l) {
    C c = in[l]->c;
    constexpr int N = M * M / kWave;
    for (int i = 0; i < N; ++i) {
      const int row = M == 16 ? 4 * (l / 16) + i : 8 * (i / 4) + 4 * (l / 32) + i % 4;
      float s = 0.f;
      for (int k = 0; k < K; ++k) s += a[row][k] * b[l % M][k];
      c[i] += s;
    }
    *out[l] = c;
  }
}
inline float bits_to_bf16(short x) {
  const uint32_t w = (uint32_t)(uint16_t)x << 16;
  float f;
  std::memcpy(&f, &w, 4);
  return f;
}
inline void f_mm16(const Mm<bf8, f4>* const* in, f4* const* out) {
  product<16, 32>(in, out, [](const bf8& v, int j) { return (float)v[j]; });
}
inline void f_mm16_16(const Mm<s4, f4>* const* in, f4* const* out) {
  product<16, 16>(in, out, [](const s4& v, int j) { return bits_to_bf16(v[j]); });
}
inline void f_mm16_4(const Mm<float, f4>* const* in, f4* const* out) {
  product<16, 4>(in, out, [](float v, int) { return v; });
}
inline void f_mm32(const Mm<bf8, f16>* const* in, f16* const* out) {
  product<32, 16>(in, out, [](const bf8& v, int j) { return (float)v[j]; });
}
// Reads of four 16-bit values a lane, transposed among rows of 16 lanes: lane i gets the value i % 4 of lane
// 4 t + i / 4, for t = 0 .. 3.
inline void f_tr16(const s4* const* in, s4* const* out) {
  all64(reinterpret_cast<const void* const*>(in), "transposing read in a part of a wave");
  for (int l = 0; l < kWave; ++l)
    for (int t = 0; t < 4; ++t) (*out[l])[t] = (*in[(l & ~15) + 4 * t + (l & 15) / 4])[l & 3];
}

inline float fp4_value(unsigned code) {
  static const float mag[8] = {0.f, 0.5f, 1.f, 1.5f, 2.f, 3.f, 4.f, 6.f};
  return code & 8 ? -mag[code & 7] : mag[code & 7];
}
inline int scale_of(float s) {                             // the exponent byte
  uint32_t w;
  std::memcpy(&w, &s, 4);
  return (int)((w >> 23) & 255);
}
typedef __bf16 bf2 __attribute__((ext_vector_type(2)));
inline bf2 fp4_to_bf16(unsigned w, float s, int byte) {
  const unsigned b = (w >> (8 * byte)) & 255;
  const int e = scale_of(s);
  bf2 r;
  for (int i = 0; i < 2; ++i)
    r[i] = (__bf16)(e == 255 ? NAN : std::ldexp(fp4_value(i ? b >> 4 : b & 15), e - 127));
  return r;
}
inline unsigned bf16_to_fp4(unsigned old, bf2 x, float s, int byte) {
  unsigned b = 0;
  for (int i = 0; i < 2; ++i) {
    uint16_t h;                                      // (the sign by its bit: a negative zero has one)
    const __bf16 v = x[i];
    std::memcpy(&h, &v, 2);
    const float y = std::ldexp(bits_to_bf16((short)(h & 0x7fff)), 127 - scale_of(s));
    unsigned best = 0;
    for (unsigned c = 1; c < 8; ++c) {
      const float d = std::fabs(y - fp4_value(c)), e = std::fabs(y - fp4_value(best));
      if (d < e || (d == e && c % 2 == 0)) best = c;
    }
    b |= (best | (h & 0x8000 ? 8u : 0u)) << (4 * i);
  }
  return (old & ~(255u << (8 * byte))) | (b << (8 * byte));
}
struct Buffer { const unsigned char* base; int bytes; };
template <class T> T buffer_load(const Buffer& p, unsigned off) {
  T v{};
  if (off + sizeof(T) > (unsigned)p.bytes) fail("a load past its buffer's end");
  std::memcpy(&v, p.base + off, sizeof(T));
  return v;
}
inline unsigned perm(unsigned a, unsigned b, unsigned sel) {
  const uint64_t both = ((uint64_t)a << 32) | b;
  unsigned r = 0;
  for (int i = 0; i < 4; ++i) {
    const unsigned s = (sel >> (8 * i)) & 255;
    if (s > 7) fail("perm selector");
    r |= (unsigned)((both >> (8 * s)) & 255) << (8 * i);
  }
  return r;
}
inline int frexp_e(float x) {
  int e = 0;
  if (std::isfinite(x)) std::frexp(x, &e);
  return e;
}
template <class T> T add(T* p, T v) { const T o = *p; *p = o + v; return o; }

}  // namespace emu

#define threadIdx (emu::cur->tid)
#define blockIdx (emu::block)
#define gridDim (emu::grid)
#define blockDim (emu::threads)
#define EMU_KEY ((long)__LINE__)
#define __syncthreads() emu::barrier()
#define __builtin_amdgcn_s_barrier() emu::barrier()
#define __builtin_amdgcn_s_waitcnt(imm) emu::wait(imm)
#define __builtin_amdgcn_wave_barrier() ((void)emu::wave_op<int, int, emu::f_first<int>>(EMU_KEY, 0))
#define __builtin_amdgcn_fence(...) ((void)0)
#define __builtin_amdgcn_sched_barrier(m) ((void)0)
#define __builtin_amdgcn_sched_group_barrier(m, n, g) ((void)0)
template <class T> T emu_first(long key, T v) { return emu::wave_op<T, T, emu::f_first<T>>(key, v); }
template <class T> T emu_lane(long key, T v, int l) {
  return emu::wave_op<emu::Two<T>, T, emu::f_lane<T>>(key, emu::Two<T>{v, l});
}
inline int emu_me() { return (int)(emu::cur->tid.x % emu::kWave); }
#define __builtin_amdgcn_readfirstlane(v) emu_first<int>(EMU_KEY, (int)(v))
#define __builtin_amdgcn_readlane(v, l) emu_lane<int>(EMU_KEY, (int)(v), (l))
#define __shfl(v, l) emu_lane(EMU_KEY, (v), (l))
#define __shfl_xor(v, m) emu_lane(EMU_KEY, (v), emu_me() ^ (m))
#define __shfl_up(v, d) emu_lane(EMU_KEY, (v), emu_me() >= (d) ? emu_me() - (d) : emu_me())
#define __ballot(p) emu::wave_op<bool, uint64_t, emu::f_ballot>(EMU_KEY, (bool)(p))
#define __any(p) (__ballot(p) != 0)
#define __builtin_amdgcn_update_dpp(old, src, ctrl, rows, banks, zero) \
  emu::wave_op<emu::Dpp, int, emu::f_dpp>(EMU_KEY, emu::Dpp{(int)(old), (int)(src), ctrl, rows, zero})
#define __builtin_amdgcn_mov_dpp(src, ctrl, rows, banks, zero) \
  __builtin_amdgcn_update_dpp(0, src, ctrl, rows, banks, zero)
#define __builtin_amdgcn_permlane32_swap(a, b, x, y) \
  emu::wave_op<emu::Swap, emu::u32x2_, emu::f_swap<32>>(EMU_KEY, emu::Swap{(a), (b)})
#define __builtin_amdgcn_permlane16_swap(a, b, x, y) \
  emu::wave_op<emu::Swap, emu::u32x2_, emu::f_swap<16>>(EMU_KEY, emu::Swap{(a), (b)})
#define __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, x, y, z) \
  emu::wave_op<emu::Mm<emu::bf8, emu::f4>, emu::f4, emu::f_mm16>(EMU_KEY, emu::Mm<emu::bf8, emu::f4>{(a), (b), (c)})
#define __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(a, b, c, x, y, z) \
  emu::wave_op<emu::Mm<emu::s4, emu::f4>, emu::f4, emu::f_mm16_16>(EMU_KEY, emu::Mm<emu::s4, emu::f4>{(a), (b), (c)})
#define __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, x, y, z) \
  emu::wave_op<emu::Mm<float, emu::f4>, emu::f4, emu::f_mm16_4>(EMU_KEY, emu::Mm<float, emu::f4>{(a), (b), (c)})
#define __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, x, y, z) \
  emu::wave_op<emu::Mm<emu::bf8, emu::f16>, emu::f16, emu::f_mm32>(EMU_KEY, emu::Mm<emu::bf8, emu::f16>{(a), (b), (c)})
#define __builtin_amdgcn_ds_read_tr16_b64_v4i16(p) \
  emu::wave_op<emu::s4, emu::s4, emu::f_tr16>(EMU_KEY, *(const emu::s4*)(p))
#define __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, b) emu::fp4_to_bf16(w, s, b)
#define __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(o, x, s, b) emu::bf16_to_fp4(o, x, s, b)
#define __amdgpu_buffer_rsrc_t emu::Buffer
#define __builtin_amdgcn_make_buffer_rsrc(p, stride, n, flags) (emu::Buffer{(p), (n)})
#define __builtin_amdgcn_raw_buffer_load_b128(p, off, s, a) emu::buffer_load<u32x4>(p, off)
#define __builtin_amdgcn_raw_buffer_load_b64(p, off, s, a) emu::buffer_load<u32x2>(p, off)
#define __builtin_amdgcn_raw_buffer_load_b32(p, off, s, a) emu::buffer_load<unsigned>(p, off)
#define __builtin_amdgcn_perm(a, b, s) emu::perm(a, b, s)
#define __builtin_amdgcn_ubfe(w, o, n) (((unsigned)(w) >> (o)) & ((1u << (n)) - 1u))
#define __builtin_amdgcn_exp2f(x) exp2f(x)
#define __builtin_amdgcn_logf(x) log2f(x)
#define __builtin_amdgcn_rcpf(x) (1.f / (x))
#define __builtin_amdgcn_ldexpf(x, e) ldexpf(x, e)
#define __builtin_amdgcn_frexp_expf(x) emu::frexp_e(x)
#define __builtin_amdgcn_mbcnt_lo(m, c) \
  ((c) + __builtin_popcount((m) & (emu_me() >= 32 ? ~0u : (1u << emu_me()) - 1u)))
#define __builtin_amdgcn_mbcnt_hi(m, c) \
  ((c) + __builtin_popcount((m) & (emu_me() < 32 ? 0u : (1u << (emu_me() - 32)) - 1u)))
#define __hip_atomic_fetch_add(p, v, order, scope) emu::add(p, v)
#define __popcll(x) __builtin_popcountll(x)
template <class T> T atomicAdd(T* p, T v) { return emu::add(p, v); }
template <class T> T atomicMin(T* p, T v) { const T o = *p; if (v < o) *p = v; return o; }
template <class T> T atomicMax(T* p, T v) { const T o = *p; if (v > o) *p = v; return o; }
inline unsigned __umulhi(unsigned a, unsigned b) { return (unsigned)(((uint64_t)a * b) >> 32); }
template <class A, class B, class = std::enable_if_t<std::is_arithmetic_v<A> && std::is_arithmetic_v<B>>>
constexpr std::common_type_t<A, B> min(A a, B b) { return (std::common_type_t<A, B>)b < a ? b : a; }
template <class A, class B, class = std::enable_if_t<std::is_arithmetic_v<A> && std::is_arithmetic_v<B>>>
constexpr std::common_type_t<A, B> max(A a, B b) { return (std::common_type_t<A, B>)a < b ? b : a; }

// The host side.
typedef int hipError_t;
typedef void* hipStream_t;
typedef void* hipEvent_t;
enum { hipSuccess = 0, hipErrorInvalidValue = 1 };
enum { hipMemcpyHostToDevice, hipMemcpyDeviceToHost, hipEventDisableTiming, hipDeviceAttributeMultiprocessorCount };
inline hipError_t hipMalloc(void** p, size_t n) {
  if (posix_memalign(p, 256, n ? n : 1)) return 2;
  std::memset(*p, 0xA7, n);                          // (what nobody wrote is nobody's page or branch)
  return 0;
}
inline hipError_t hipHostMalloc(void** p, size_t n) { return hipMalloc(p, n); }
inline hipError_t hipFree(void* p) { std::free(p); return 0; }
inline hipError_t hipHostFree(void* p) { std::free(p); return 0; }
inline hipError_t hipMemcpy(void* d, const void* s, size_t n, int) { std::memcpy(d, s, n); return 0; }
inline hipError_t hipMemcpyAsync(void* d, const void* s, size_t n, int, hipStream_t) { std::memcpy(d, s, n); return 0; }
inline hipError_t hipGetLastError() { return 0; }
inline const char* hipGetErrorString(hipError_t) { return ""; }
inline hipError_t hipGetDevice(int* d) { *d = 0; return 0; }
inline hipError_t hipDeviceGetAttribute(int* v, int, int) { *v = emu::num_cus; return 0; }
inline hipError_t hipDeviceSynchronize() { return 0; }
inline hipError_t hipStreamSynchronize(hipStream_t) { return 0; }
inline hipError_t hipStreamWaitEvent(hipStream_t, hipEvent_t, unsigned) { return 0; }
inline hipError_t hipEventCreate(hipEvent_t* e) { *e = e; return 0; }
inline hipError_t hipEventCreateWithFlags(hipEvent_t* e, unsigned) { *e = e; return 0; }
inline hipError_t hipEventRecord(hipEvent_t, hipStream_t) { return 0; }
inline hipError_t hipEventSynchronize(hipEvent_t) { return 0; }
inline hipError_t hipEventDestroy(hipEvent_t) { return 0; }
inline hipError_t hipEventElapsedTime(float* f, hipEvent_t, hipEvent_t) { *f = 0.f; return 0; }
#define HIP_SYMBOL(x) (x)
template <class T> hipError_t hipGetSymbolAddress(void** p, T& s) { *p = &s; return 0; }
template <class K, class... A>
void hipLaunchKernelGGL(K k, dim3 g, dim3 b, size_t lds, hipStream_t, A... a) {
  emu::launch(g, b, lds, [=] { k(a...); });
}
template <class K, class... A>
void hipExtLaunchKernelGGL(K k, dim3 g, dim3 b, size_t lds, hipStream_t, hipEvent_t, hipEvent_t, unsigned, A... a) {
  emu::launch(g, b, lds, [=] { k(a...); });
}
