// The scheduler of the CPU model of the device (hip/hip_runtime.h).
#include <hip/hip_runtime.h>

#include <sys/mman.h>

#include <algorithm>
#include <vector>

extern "C" void emu_switch(void** save, void* to);
asm(R"(
.text
.globl emu_switch
emu_switch:
  push %rbp
  push %rbx
  push %r12
  push %r13
  push %r14
  push %r15
  mov %rsp, (%rdi)
  mov %rsi, %rsp
  pop %r15
  pop %r14
  pop %r13
  pop %r12
  pop %rbx
  pop %rbp
  ret
)");

// Conversions that the compiler calls on CPUs without instructions for them.
extern "C" __bf16 __truncsfbf2(float f) {
  uint32_t w;
  std::memcpy(&w, &f, 4);
  uint16_t h;
  if (f != f) h = (uint16_t)((w >> 16) | 0x40);
  else h = (uint16_t)((w + 0x7fff + ((w >> 16) & 1)) >> 16);
  __bf16 r;
  std::memcpy(&r, &h, 2);
  return r;
}

namespace emu {

Lane* cur = nullptr;
dim3 block, grid, threads;
int num_cus = 256;
bool late_copies = false;
uint64_t seed = 1;
long partial_ops = 0;

namespace {
constexpr size_t kStack = 256 << 10;
constexpr int kMost = 1024;
Lane lanes[kMost];
void* main_sp = nullptr;
const std::function<void()>* body = nullptr;
std::vector<char> lds;
char* lds_at = nullptr;
struct Copy { const char* src; char* dst; };
std::vector<Copy> copies[kMost];

uint64_t draw() {
  seed ^= seed << 13;
  seed ^= seed >> 7;
  seed ^= seed << 17;
  return seed;
}
void entry() {
  (*body)();
  cur->state = Lane::kDone;
  emu_switch(&cur->sp, main_sp);
  __builtin_trap();
}
void start(Lane& l) {
  if (!l.stack) {
    l.stack = static_cast<char*>(mmap(nullptr, kStack, PROT_READ | PROT_WRITE, MAP_PRIVATE | MAP_ANONYMOUS, -1, 0));
    mprotect(l.stack, 4096, PROT_NONE);
  }
  void** sp = reinterpret_cast<void**>(l.stack + kStack) - 2;
  *sp = reinterpret_cast<void*>(&entry);             // (the stack is 16-byte aligned behind the return)
  for (int i = 0; i < 6; ++i) *--sp = nullptr;
  l.sp = sp;
  l.state = Lane::kReady;
}
void go(Lane& l) {
  cur = &l;
  emu_switch(&main_sp, l.sp);
  cur = nullptr;
}
// Runs wave w until all of its lanes are at a barrier or done; a wave operation at a time.
bool step(int w, int n) {
  Lane* wave = lanes + w * kWave;
  const int m = std::min(kWave, n - w * kWave);
  bool ran = false;
  for (int i = 0; i < m; ++i)
    if (wave[i].state == Lane::kReady) {
      go(wave[i]);
      ran = true;
    }
  Lane* group[kWave];
  int k = 0;
  long key = 0;
  void (*f)(Lane**, int) = nullptr;
  for (int i = 0; i < m; ++i)
    if (wave[i].state == Lane::kWaveOp && (!f || wave[i].key < key)) {
      key = wave[i].key;
      f = wave[i].resolve;
    }
  if (!f) return ran;
  for (int i = 0; i < m; ++i)
    if (wave[i].state == Lane::kWaveOp && wave[i].key == key && wave[i].resolve == f) group[k++] = &wave[i];
  partial_ops += k != kWave;
  f(group, k);
  for (int i = 0; i < k; ++i) group[i]->state = Lane::kReady;
  return true;
}
}  // namespace

void fail(const char* what) {
  std::fprintf(stderr, "model: %s (block %u %u, thread %u)\n", what, block.x, block.y, cur ? cur->tid.x : 0u);
  std::abort();
}
void yield() { emu_switch(&cur->sp, main_sp); }
void* dynamic_lds() { return lds_at; }

void dma16(unsigned off, const void* base, unsigned lds_base) {
  const Copy c{static_cast<const char*>(base) + off,
               reinterpret_cast<char*>((uintptr_t)lds_base + 16 * (cur->tid.x % kWave))};
  if (late_copies) copies[cur->tid.x].push_back(c);
  else std::memcpy(c.dst, c.src, 16);
}
void wait(int imm) {
  if ((imm & 15) | (imm >> 14 & 3)) return;          // (not vmcnt(0))
  for (const Copy& c : copies[cur->tid.x]) std::memcpy(c.dst, c.src, 16);
  copies[cur->tid.x].clear();
}

void launch(dim3 g, dim3 b, size_t bytes, const std::function<void()>& kernel) {
  if (b.x > kMost || b.y != 1 || b.z != 1 || g.z != 1) fail("launch shape");
  if (g.x == 0 || g.y == 0) fail("empty grid");
  body = &kernel;
  grid = g;
  threads = b;
  const int n = (int)b.x, waves = (n + kWave - 1) / kWave;
  for (unsigned y = 0; y < g.y; ++y)
    for (unsigned x = 0; x < g.x; ++x) {
      block = dim3(x, y, 0);
      // (a fresh allocation of exactly the size asked for, so that its ends are watched)
      lds_at = bytes ? static_cast<char*>(std::malloc(bytes)) : nullptr;
      if (bytes) std::memset(lds_at, 0xA7, bytes);
      for (int i = 0; i < n; ++i) {
        lanes[i].tid = dim3(i, 0, 0);
        copies[i].clear();
        start(lanes[i]);
      }
      for (;;) {
        bool ran = false;
        const int first = (int)(draw() % waves);
        // (some waves run ahead of others by a drawn number of steps)
        for (int k = 0; k < waves; ++k) {
          const int w = (first + k) % waves;
          for (uint64_t s = draw() % 8; s + 1 > 0; --s) {
            const bool r = step(w, n);
            ran = ran || r;
            if (!r || s == 0) break;
          }
        }
        if (ran) continue;
        int at = 0, done = 0;
        for (int i = 0; i < n; ++i) {
          at += lanes[i].state == Lane::kBarrier;
          done += lanes[i].state == Lane::kDone;
        }
        if (done == n) break;
        if (at + done != n) fail("deadlock");
        // (a wave's lanes wait together)
        for (int w = 0; w < waves; ++w) {
          int d = 0;
          const int m = std::min(kWave, n - w * kWave);
          for (int i = 0; i < m; ++i) d += lanes[w * kWave + i].state == Lane::kDone;
          if (d != 0 && d != m) fail("a wave partly ended before a barrier");
        }
        for (int i = 0; i < n; ++i)
          if (lanes[i].state == Lane::kBarrier) lanes[i].state = Lane::kReady;
      }
      for (int i = 0; i < n; ++i)
        if (!copies[i].empty()) fail("a copy to LDS that no wait covered");
      std::free(lds_at);
    }
}

}  // namespace emu
