// Runs calls of graphattn_step.h on the CPU model of the device: a file of cases in, their outputs out.  Every array
// is an allocation of exactly its size.  A case is a list of blobs (int64 bytes, then the bytes); the first holds the
// call's number and its sizes as int64.
#include <hip/hip_runtime.h>

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <string>
#include <vector>

#include "graphattn_step.h"

namespace ga {
static std::string error;
ga_status host_fail(ga_status st, const char* msg) { error = msg; return st; }
ga_status host_hip_fail(hipError_t, const char* what) { error = what; return GA_EHIP; }
void host_clear_error() { error.clear(); }
ga_status host_check_params(const ga_params*) { return GA_OK; }
}  // namespace ga

struct Blob {
  void* p = nullptr;
  int64_t bytes = 0;
};

static bool read_blob(FILE* f, Blob* b) {
  if (std::fread(&b->bytes, 8, 1, f) != 1) return false;
  b->p = nullptr;
  if (b->bytes > 0) {
    // (aligned as the calls ask for, and no byte longer than the array)
    if (posix_memalign(&b->p, 16, b->bytes)) std::abort();
    if ((int64_t)std::fread(b->p, 1, b->bytes, f) != b->bytes) std::abort();
  }
  return true;
}
static void write_blob(FILE* f, const Blob& b) {
  std::fwrite(&b.bytes, 8, 1, f);
  if (b.bytes) std::fwrite(b.p, 1, b.bytes, f);
}

template <class T> static T* as(const Blob& b) { return static_cast<T*>(b.p); }

int main(int argc, char** argv) {
  FILE* in = std::fopen(argv[1], "rb");
  FILE* out = std::fopen(argv[2], "wb");
  emu::seed = argc > 3 ? std::strtoull(argv[3], nullptr, 10) : 1;
  if (argc > 4) emu::num_cus = std::atoi(argv[4]);
  if (!in || !out) return 2;
  Blob head;
  int done = 0;
  while (read_blob(in, &head)) {
    const int64_t* s = as<int64_t>(head);
    std::vector<Blob> b(s[1]);
    for (auto& x : b)
      if (!read_blob(in, &x)) std::abort();
    const int op = (int)s[0];
    s += 2;
    ga_status st = GA_EINVAL;
    std::vector<int> outs;
    auto graph_at = [&](int i, const int64_t* z) {
      return ga_device_graph{(int32_t)z[0], (int32_t)z[1], z[2], z[3], z[4], as<int32_t>(b[i]), as<int64_t>(b[i + 1]),
                             as<int32_t>(b[i + 2]), as<int64_t>(b[i + 3]), as<int32_t>(b[i + 4])};
    };
    if (op == 0) {
      st = graphattn_page_table(as<int32_t>(b[0]), (int32_t)s[0], (int32_t)s[1], as<int64_t>(b[1]), as<int32_t>(b[2]),
                                (int32_t)s[2], s[3], as<int32_t>(b[3]), s[4], as<int64_t>(b[4]), as<int32_t>(b[5]), s[5],
                                nullptr);
      outs = {4, 5};
    } else if (op == 1) {
      const ga_device_graph g = graph_at(0, s);
      st = graphattn_slot_map(&g, as<int32_t>(b[5]), as<int32_t>(b[6]), as<int32_t>(b[7]), as<int32_t>(b[8]),
                              as<int32_t>(b[9]), (int32_t)s[5], nullptr);
      outs = {6, 7, 8, 9};
    } else if (op == 2) {
      const double* f = as<double>(b[0]);
      ga_params p{(int32_t)s[1], (int32_t)s[2], (int32_t)s[3], 16, s[5], (int32_t)s[4], 0.f, 0};
      ga_qk_transform t{(int32_t)s[9], (int32_t)s[10], (float)f[0], (float)f[1], as<double>(b[8]), as<float>(b[9]),
                        as<float>(b[10])};
      st = graphattn_qkv_append(b[1].p, b[2].p, b[3].p, b[4].p, s[6], s[7], s[8], as<int32_t>(b[5]), as<int32_t>(b[6]),
                                (int32_t)s[0], s[11] ? b[2].p : b[7].p, &t, &p, nullptr);
      outs = {1, s[11] ? 2 : 7};
    } else {
      ga_logit_rules r{};
      r.repetition = as<float>(b[10]);
      r.frequency = as<float>(b[11]);
      r.presence = as<float>(b[12]);
      r.temperature = as<float>(b[13]);
      r.prompt_segments = (int32_t)s[6];
      r.bias_offsets = as<int64_t>(b[14]);
      r.bias_tokens = as<int32_t>(b[15]);
      r.bias_values = as<float>(b[16]);
      r.num_bias = s[7];
      r.masks = as<uint32_t>(b[17]);
      r.num_masks = (int32_t)s[8];
      r.mask_words = s[9];
      r.row_mask = as<int32_t>(b[18]);
      const ga_device_graph g = graph_at(2, s + 10);
      void* o = s[15] ? b[0].p : b[1].p;
      st = graphattn_process_logits(b[0].p, s[4], (int32_t)s[0], (int32_t)s[1], (int32_t)s[2], &r, s[16] ? &g : nullptr,
                                    as<int32_t>(b[7]), as<int32_t>(b[8]), as<int32_t>(b[9]), o, s[5], (int32_t)s[3],
                                    nullptr);
      outs = {s[15] ? 0 : 1};
    }
    if (st != GA_OK) {
      std::printf("case %d: %d %s\n", done, (int)st, ga::error.c_str());
      return 1;
    }
    for (int i : outs) write_blob(out, b[i]);
    for (auto& x : b) std::free(x.p);
    std::free(head.p);
    ++done;
  }
  std::fclose(in);
  std::fclose(out);
  std::printf("ok, %d cases\n", done);
  return 0;
}
