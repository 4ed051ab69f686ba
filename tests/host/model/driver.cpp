// Random calls of the compressed cache on the CPU model of the device (hip/hip_runtime.h): rollout graphs of the
// shapes that rollouts have, attended, gathered and evicted, every array of exactly the size the headers ask
// for.  Results are compared with sums in 64 bits; AddressSanitizer watches the addresses.
//
//   driver KIND CASES SEED     KIND: attn, mass, evict or cache
//   driver file PATH           a given graph, for its addresses alone (its sums in 64 bits would take too long):
//                              every page is a table's, every row and slot of an output is written
#include <hip/hip_runtime.h>

#include <algorithm>
#include <random>
#include <string>
#include <vector>

#include "graphattn_cache.h"

namespace {

typedef std::vector<int32_t> Ints;
std::mt19937 rng;
int U(int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); }
int spread(int lo, int hi) {
  return (int)std::lround(std::exp(std::uniform_real_distribution<double>(std::log(lo), std::log(hi))(rng)));
}
double normal() { return std::normal_distribution<double>()(rng); }

// Device memory of exactly n values.
template <class T> struct Dev {
  T* p = nullptr;
  size_t n;
  explicit Dev(size_t n_) : n(n_) { void* v; hipMalloc(&v, n * sizeof(T)); p = static_cast<T*>(v); }
  Dev(const Dev&) = delete;
  ~Dev() { hipFree(p); }
  T& operator[](size_t i) { return p[i]; }
};

void must(ga_status rc, const char* what) {
  if (rc == GA_OK) return;
  std::fprintf(stderr, "%s: %d %s\n", what, (int)rc, graphattn_last_error());
  std::exit(1);
}

uint16_t to_bf16(double x) {
  const float f = (float)x;
  uint32_t w;
  std::memcpy(&w, &f, 4);
  return (uint16_t)((w + 0x7fff + ((w >> 16) & 1)) >> 16);
}
double of_bf16(uint16_t h) { return emu::bits_to_bf16((short)h); }

struct Graph {
  Ints len, pages, segs, counts;
  std::vector<int64_t> off{0}, poff{0};
  std::vector<Ints> paths;
  int64_t num_pages = 0;
  int rows = 0;
  ga_segment_table table() const { return {(int32_t)len.size(), len.data(), off.data(), pages.data()}; }
  ga_branch_paths branches() const { return {(int32_t)paths.size(), poff.data(), segs.data()}; }
};

int fill(Graph& g, int n) { g.len.push_back(n); return (int)g.len.size() - 1; }

// kind 0 fan, 1 step trees and merged graphs, 2 long chains with a shared trunk, 3 single chains, 4 prompts
Graph draw_graph(int kind, bool queries, int most, int spare) {
  Graph g;
  const int prompts = spread(1, kind == 1 ? 3 : 8);
  for (int p = 0; p < prompts; ++p) {
    if (kind == 0) {
      const int t = spread(1, most / 8 + 1), root = fill(g, 4 * t), fan = spread(1, 40);
      for (int b = 0; b < fan; ++b) g.paths.push_back({root, fill(g, t)});
    } else if (kind == 1) {
      std::vector<Ints> front{{fill(g, U(1, most / 4 + 1))}};
      const bool dag = U(0, 1);
      for (int fan : {2, 2, 2, 1}) {
        std::vector<Ints> next;
        std::vector<Ints> kids(front.size());
        for (size_t i = 0; i < front.size(); ++i) {
          if (dag && i && U(0, 3) == 0) kids[i] = kids[U(0, (int)i - 1)];
          else for (int k = 0; k < fan; ++k) kids[i].push_back(fill(g, U(1, most / 8 + 1)));
          for (int k : kids[i]) { next.push_back(front[i]); next.back().push_back(k); }
        }
        front = next;
      }
      g.paths.insert(g.paths.end(), front.begin(), front.end());
    } else if (kind == 2) {
      Ints trunk;
      for (int i = U(1, 4); i > 0; --i) trunk.push_back(fill(g, U(1, most)));
      for (int b = U(2, 8); b > 0; --b) {
        Ints path = trunk;
        for (int i = U(1, 3); i > 0; --i) path.push_back(fill(g, U(1, most / 2 + 1)));
        g.paths.push_back(path);
      }
    } else {
      g.paths.push_back({fill(g, spread(1, most))});
    }
  }
  for (auto& path : g.paths) {
    int n = 1;
    if (kind == 4) n = U(0, 3) ? g.len[path.back()] : U(1, g.len[path.back()]);
    else if (queries) {
      const int t = U(1, 40);
      path.push_back(fill(g, t));
      n = U(0, 2) ? t : U(1, t);
    }
    g.counts.push_back(n);
    g.rows += n;
    g.segs.insert(g.segs.end(), path.begin(), path.end());
    g.poff.push_back((int64_t)g.segs.size());
  }
  for (int n : g.len) g.off.push_back(g.off.back() + (n + 15) / 16 + (spare ? U(0, spare) : 0));
  g.num_pages = g.off.back() + U(0, 3);
  Ints order((size_t)g.num_pages);
  for (size_t i = 0; i < order.size(); ++i) order[i] = (int32_t)i;
  std::shuffle(order.begin(), order.end(), rng);
  g.pages.assign(order.begin(), order.begin() + g.off.back());
  return g;
}

// A pool with values in the slots of the graph's tokens and NaN elsewhere, and the values.
struct Pool {
  ga_params p;
  Dev<unsigned char> mem;
  std::vector<double> v[2];                          // [slot][Hkv][D]
  explicit Pool(const ga_params& p_) : p(p_), mem((size_t)(graphattn_kv_page_bytes(&p_) * p_.num_pages)) {
    for (auto& x : v) x.assign((size_t)(p.num_pages * 16 * p.num_kv_heads * p.head_dim), NAN);
    const size_t values = (size_t)(p.num_pages * p.num_kv_heads * 32 * p.head_dim);
    if (p.dtype == GA_F32) for (size_t i = 0; i < values; ++i) reinterpret_cast<float*>(mem.p)[i] = NAN;
    if (p.dtype == GA_BF16) for (size_t i = 0; i < values; ++i) reinterpret_cast<uint16_t*>(mem.p)[i] = 0x7fc0;
    if (p.dtype == GA_MXFP4) std::memset(mem.p, 0xff, mem.n);
  }
  size_t at(int64_t slot, int h, int c) const { return ((size_t)slot * p.num_kv_heads + h) * p.head_dim + c; }
  void put(int64_t slot) {
    const int D = p.head_dim, t = (int)(slot % 16);
    for (int h = 0; h < p.num_kv_heads; ++h)
      for (int kv = 0; kv < 2; ++kv)
        for (int c = 0; c < D; ++c) {
          double x = normal();
          const size_t blk = (size_t)(slot / 16 * p.num_kv_heads + h);
          if (p.dtype == GA_F32) {
            reinterpret_cast<float*>(mem.p)[(blk * 2 + kv) * 16 * D + t * D + c] = (float)x;
            x = (float)x;
          } else if (p.dtype == GA_BF16) {
            reinterpret_cast<uint16_t*>(mem.p)[(blk * 2 + kv) * 16 * D + t * D + c] = to_bf16(x);
            x = of_bf16(to_bf16(x));
          } else {
            unsigned char* b = mem.p + blk * 17 * D;
            const int w = D / 16;
            const int code = kv ? 8 * D + ((t / 4 * 16 + c / w) * 4 + t % 4) * (w / 2) + c % w / 2 : t * (D / 2) + c / 2;
            const int scale = kv ? 16 * D + D / 2 + (t / 4 * (D / 32) + c / 32) * 4 + t % 4 : 16 * D + t * (D / 32) + c / 32;
            if (c % 32 == 0) b[scale] = (unsigned char)U(125, 126);
            const unsigned q = (unsigned)U(0, 15);
            b[code] = (unsigned char)(c & 1 ? (b[code] & 15) | (q << 4) : (b[code] & 0xf0) | q);
            x = std::ldexp((double)emu::fp4_value(q), b[scale] - 127);
          }
          v[kv][at(slot, h, c)] = x;
        }
  }
};

struct Case {
  Graph g;
  ga_params p;
  bool many;                                         // a multi-query plan
  std::vector<std::vector<int64_t>> ctx;             // slots of every branch's tokens
  void contexts() {
    ctx.clear();
    for (const auto& path : g.paths) {
      std::vector<int64_t> c;
      for (int s : path)
        for (int t = 0; t < g.len[s]; ++t) c.push_back((int64_t)g.pages[g.off[s] + t / 16] * 16 + t % 16);
      ctx.push_back(c);
    }
  }
};

struct Result { std::vector<double> out, lse, bound, lse_bound, mass, mass_bound; };

// out, lse and the masses of the rows, in 64 bits; q [rows][Hq][D].  odd [rows][Hq]: an lse to gather the masses
// with in place of the row's own, where it is not 0.
Result reference(const Case& c, const Pool& pool, const std::vector<double>& q, const std::vector<double>& odd) {
  const int Hq = c.p.num_q_heads, G = Hq / c.p.num_kv_heads, D = c.p.head_dim;
  Result r;
  r.mass.assign((size_t)(16 * c.p.num_pages), 0.);
  r.mass_bound = r.mass;
  size_t row = 0;
  std::vector<double> s, reach;
  for (size_t b = 0; b < c.ctx.size(); ++b)
    for (int i = 0; i < c.g.counts[b]; ++i, ++row) {
      const size_t n = c.ctx[b].size() - c.g.counts[b] + i + 1;
      for (int h = 0; h < Hq; ++h) {
        const double* qr = &q[(row * Hq + h) * D];
        s.assign(n, 0.);
        reach.assign(n, 0.);
        double top = -INFINITY, far = 0.;
        for (size_t t = 0; t < n; ++t) {
          const double* k = &pool.v[0][pool.at(c.ctx[b][t], h / G, 0)];
          for (int x = 0; x < D; ++x) { s[t] += qr[x] * k[x]; reach[t] += std::fabs(qr[x] * k[x]); }
          s[t] /= std::sqrt((double)D);
          reach[t] /= std::sqrt((double)D);
          top = std::max(top, s[t]);
          far = std::max(far, reach[t]);
        }
        double l = 0.;
        for (size_t t = 0; t < n; ++t) l += std::exp(s[t] - top);
        const double lse = top + std::log(l);
        r.lse.push_back(lse);
        // (float32 scores: half a step an addition; a few steps of the sum and its logarithm)
        r.lse_bound.push_back((D + 8) * std::ldexp(1., -24) * far + std::ldexp(1., -20) * (1. + std::fabs(lse)));
        std::vector<double> o(D, 0.), w(D, 0.);
        double vmax = 0.;
        for (size_t t = 0; t < n; ++t) {
          const double e = std::exp(s[t] - lse);
          const int64_t slot = c.ctx[b][t];
          const double given = odd[row * Hq + h];
          // (an infinite lse: the row counts for nothing; NaN: for every token that it sees, and no other)
          r.mass[slot] += given == 0. ? e : std::isnan(given) ? NAN : 0.;
          r.mass_bound[slot] += e * ((D + 8) * std::ldexp(1., -24) * reach[t] +
                                     std::ldexp(1., -22) * (2. + reach[t] + std::fabs(lse)) + std::ldexp(1., -16));
          const double* v = &pool.v[1][pool.at(slot, h / G, 0)];
          for (int x = 0; x < D; ++x) { o[x] += e * v[x]; w[x] += e * std::fabs(v[x]); vmax = std::max(vmax, std::fabs(v[x])); }
        }
        for (int x = 0; x < D; ++x) {
          // (probabilities to bf16, partial rows to fp16 of their largest value, the result to bf16)
          const double part = std::ldexp(w[x], -8) + std::ldexp(vmax, -11) + std::ldexp(vmax, -18);
          r.out.push_back(o[x]);
          r.bound.push_back(c.p.out_f32 ? part : part + std::ldexp(std::fabs(o[x]) + part, -8));
        }
      }
    }
  return r;
}

void compare(const char* what, const std::vector<double>& got, const std::vector<double>& want,
             const std::vector<double>& bound) {
  double worst = 0.;
  for (size_t i = 0; i < want.size(); ++i) {
    const double d = std::isnan(want[i]) && std::isnan(got[i]) ? 0. : std::fabs(got[i] - want[i]);
    if (!(d <= bound[i] || (d == 0. && std::isnan(want[i])))) {
      std::fprintf(stderr, "%s[%zu]: %g, not %g (off %g, may be %g)\n", what, i, got[i], want[i], d, bound[i]);
      std::exit(1);
    }
    if (bound[i] > 0) worst = std::max(worst, d / bound[i]);
  }
  std::printf(" %s %.3f", what, worst);
}

// (of the last two a prompt's rows pass the 4096 from which on the mass shares them among more waves)
const int kHeads[][3] = {{28, 4, 128}, {40, 8, 128}, {32, 8, 128}, {16, 2, 64}, {12, 12, 64}, {8, 2, 64},
                         {12, 3, 128}, {4, 1, 64}, {4, 1, 128}, {64, 1, 64}, {64, 1, 128}};

void attend(bool mass_of_it, int number) {
  Case c;
  const int kind = U(0, 4), hd = U(0, mass_of_it ? 10 : 8);
  c.many = kind == 4 || U(0, 1);
  emu::num_cus = spread(4, 64);                     // (a workgroup for every work stream at least)
  const int most = spread(8, kind == 1 ? 700 : 1500);
  c.g = draw_graph(kind, c.many, most, U(0, 3) == 0 ? 3 : 0);
  while ((int64_t)c.g.rows * kHeads[hd][0] * most > (mass_of_it ? 3000000 : 1500000) || c.g.num_pages * kHeads[hd][1] > 6000)
    c.g = draw_graph(kind, c.many, most / 4 + 1, 0);
  const int types[3] = {GA_MXFP4, GA_BF16, GA_F32};
  const int type = mass_of_it ? types[U(0, 2)] : GA_MXFP4;
  c.p = {kHeads[hd][0], kHeads[hd][1], kHeads[hd][2], 16, c.g.num_pages, type, 0.f, !mass_of_it && U(0, 4) == 0};
  c.contexts();
  std::printf("%d: kind %d, %zu branches, %d rows, %lld pages, %d/%d x %d, type %d, %s, %d CUs", number, kind, c.g.paths.size(),
              c.g.rows, (long long)c.g.num_pages, c.p.num_q_heads, c.p.num_kv_heads, c.p.head_dim, type,
              c.many ? "multi-query" : "decode", emu::num_cus);
  std::fflush(stdout);
  Pool pool(c.p);
  std::vector<char> used((size_t)(16 * c.g.num_pages), 0);
  for (const auto& x : c.ctx)
    for (int64_t s : x)
      if (!used[s]) { used[s] = 1; pool.put(s); }
  const size_t nq = (size_t)c.g.rows * c.p.num_q_heads, D = c.p.head_dim;
  std::vector<double> q(nq * D);
  Dev<unsigned char> dq(nq * D * (type == GA_F32 ? 4 : 2));
  for (size_t i = 0; i < q.size(); ++i) {
    if (type == GA_F32) q[i] = reinterpret_cast<float*>(dq.p)[i] = (float)normal();
    else q[i] = of_bf16(reinterpret_cast<uint16_t*>(dq.p)[i] = to_bf16(normal()));
  }
  const ga_segment_table st = c.g.table();
  const ga_branch_paths bp = c.g.branches();
  ga_plan* plan = nullptr;
  if (c.many) must(graphattn_plan_create_extend(&st, &bp, c.g.counts.data(), &c.p, nullptr, &plan), "plan");
  else must(graphattn_plan_create(&st, &bp, &c.p, nullptr, &plan), "plan");
  std::vector<double> odd(nq, 0.);
  if (mass_of_it && U(0, 2) == 0)
    for (int i = U(1, 3); i > 0; --i) odd[U(0, (int)nq - 1)] = U(0, 2) ? NAN : U(0, 1) ? INFINITY : -INFINITY;
  Result want = reference(c, pool, q, odd);
  for (int pass = 0; pass < 2; ++pass) {
    emu::late_copies = pass;
    emu::seed = 88172645463325252ull + 2 * rng() + 1;
    if (!mass_of_it) {
      Dev<unsigned char> out(nq * D * (c.p.out_f32 ? 4 : 2));
      Dev<float> lse(nq);
      must(graphattn_run(plan, dq.p, pool.mem.p, out.p, lse.p, nullptr), "run");
      std::vector<double> o(nq * D), l(lse.p, lse.p + nq);
      for (size_t i = 0; i < o.size(); ++i)
        o[i] = c.p.out_f32 ? reinterpret_cast<float*>(out.p)[i] : of_bf16(reinterpret_cast<uint16_t*>(out.p)[i]);
      compare("out", o, want.out, want.bound);
      compare("lse", l, want.lse, want.lse_bound);
    } else {
      Dev<float> lse(nq), in((size_t)(16 * c.g.num_pages)), out((size_t)(16 * c.g.num_pages));
      for (size_t i = 0; i < nq; ++i) lse[i] = (float)(odd[i] != 0. ? odd[i] : want.lse[i]);
      for (size_t i = 0; i < in.n; ++i) { in[i] = (float)U(0, 9); out[i] = -7.f; }
      const bool with = U(0, 2);
      must(graphattn_run_mass(plan, dq.p, pool.mem.p, lse.p, with ? in.p : nullptr, 0.5f, out.p, nullptr), "mass");
      std::vector<double> got(out.p, out.p + out.n), w(out.n, -7.), bound(out.n, 0.);
      for (size_t i = 0; i < w.size(); ++i)
        if (used[i]) {
          w[i] = want.mass[i] + (with ? 0.5 * in[i] : 0.);
          bound[i] = want.mass_bound[i] + std::ldexp(w[i], -20);
        }
      compare("mass", got, w, bound);
    }
    if (pass == 0 && U(0, 1)) {
      // New lengths, where the segments own more pages, and fewer tokens elsewhere.
      for (size_t s = 0; s < c.g.len.size(); ++s)
        if (U(0, 1)) c.g.len[s] = U(1, (int)(16 * (c.g.off[s + 1] - c.g.off[s])));
      if (c.many)
        for (size_t b = 0; b < c.g.paths.size(); ++b)
          c.g.len[c.g.paths[b].back()] = std::max(c.g.len[c.g.paths[b].back()], c.g.counts[b]);
      must(graphattn_plan_set_lengths(plan, c.g.len.data(), nullptr), "lengths");
      c.contexts();
      std::fill(used.begin(), used.end(), 0);
      for (const auto& x : c.ctx)
        for (int64_t s : x)
          if (!used[s]) { used[s] = 1; pool.put(s); }
      want = reference(c, pool, q, odd);
    }
  }
  ga_plan_info info;
  must(graphattn_plan_info(plan, &info), "info");
  std::printf(", chunks of %d pages\n", info.chunk_pages);
  graphattn_plan_destroy(plan);
}

// int64 values: operation (0 attention, 1 mass, 2 eviction), Hq, Hkv, D, type, pages, segments, branches, then the
// table's lengths, offsets and pages, the paths' offsets and segments, and the branches' query counts (0: decode) or
// the segments' keep counts, first and recent tokens.
void given(const char* path) {
  FILE* f = std::fopen(path, "rb");
  if (!f) { std::perror(path); std::exit(2); }
  auto take = [&](size_t n) {
    std::vector<int64_t> v(n);
    if (n && std::fread(v.data(), 8, n, f) != n) { std::fprintf(stderr, "%s is short\n", path); std::exit(2); }
    return v;
  };
  auto ints = [&](size_t n) { const auto v = take(n); return Ints(v.begin(), v.end()); };
  const auto h = take(8);
  Graph g;
  g.num_pages = h[5];
  g.len = ints(h[6]);
  g.off = take(h[6] + 1);
  g.pages = ints(g.off.back());
  const ga_segment_table st = g.table();
  emu::num_cus = 256;
  emu::seed = 88172645463325252ull;
  const int64_t slots = 16 * g.num_pages;
  if (h[0] == 2) {
    const Ints keep = ints(h[6]);
    const auto safe = take(2);
    size_t total = 0;
    for (int n : keep) total += n;
    Dev<float> mass(slots);
    for (int64_t i = 0; i < slots; ++i) mass[i] = U(0, 19) ? (float)std::exp(2 * normal() - 3) : 0.f;
    Dev<int32_t> pos(total), words(total);
    ga_evict* e = nullptr;
    must(graphattn_evict_create(&st, keep.data(), safe[0], safe[1], g.num_pages, nullptr, &e), "evict_create");
    must(graphattn_evict_select(e, mass.p, pos.p, words.p, nullptr), "evict_select");
    size_t at = 0;
    for (size_t s = 0; s < g.len.size(); ++s)
      for (int k = 0; k < keep[s]; ++k, ++at) {
        const int t = pos[at];
        if (t < 0 || t >= g.len[s] || (k && t <= pos[at - 1]) ||
            words[at] != g.pages[g.off[s] + t / 16] * 16 + t % 16) {
          std::fprintf(stderr, "segment %zu: position %d at %d\n", s, t, k);
          std::exit(1);
        }
      }
    graphattn_evict_destroy(e);
  } else {
    g.poff = take(h[7] + 1);
    g.segs = ints(g.poff.back());
    g.counts = ints(h[7]);
    g.paths.resize(h[7]);
    const bool many = h[7] && g.counts[0] > 0;
    int64_t rows = 0;
    for (int n : g.counts) rows += many ? n : 1;
    const ga_params p{(int32_t)h[1], (int32_t)h[2], (int32_t)h[3], 16, g.num_pages, (int32_t)h[4], 0.f, 0};
    const ga_branch_paths bp = g.branches();
    ga_plan* plan = nullptr;
    if (many) must(graphattn_plan_create_extend(&st, &bp, g.counts.data(), &p, nullptr, &plan), "plan");
    else must(graphattn_plan_create(&st, &bp, &p, nullptr, &plan), "plan");
    // (zeros: values are of no matter here)
    const size_t nq = (size_t)rows * p.num_q_heads, qb = nq * p.head_dim * (p.dtype == GA_F32 ? 4 : 2);
    Dev<unsigned char> pool((size_t)(graphattn_kv_page_bytes(&p) * g.num_pages)), q(qb), out(qb);
    Dev<float> lse(nq), mass(slots);
    std::memset(pool.p, 0, pool.n);
    std::memset(q.p, 0, q.n);
    for (int pass = 0; pass < 2; ++pass) {
      emu::late_copies = pass;
      if (h[0] == 0) {
        std::memset(out.p, 0xA7, out.n);
        std::memset(lse.p, 0xA7, 4 * lse.n);
        must(graphattn_run(plan, q.p, pool.p, out.p, lse.p, nullptr), "run");
        for (size_t i = 0; i < out.n; ++i)
          if (out[i]) { std::fprintf(stderr, "byte %zu of the output is %02x\n", i, out[i]); std::exit(1); }
        // (all scores are 0: lse is the logarithm of the tokens that the row sees)
        size_t r = 0;
        for (int64_t b = 0; b < h[7]; ++b) {
          int64_t n = 0;
          for (int64_t e = g.poff[b]; e < g.poff[b + 1]; ++e) n += g.len[g.segs[e]];
          const int c = many ? g.counts[b] : 1;
          for (int i = 0; i < c; ++i)
            for (int x = 0; x < p.num_q_heads; ++x, ++r)
              if (!(std::fabs(lse[r] - std::log((double)(n - c + i + 1))) < 1e-4)) {
                std::fprintf(stderr, "lse[%zu] is %g, of %lld tokens\n", r, lse[r], (long long)(n - c + i + 1));
                std::exit(1);
              }
        }
      } else {
        for (size_t i = 0; i < nq; ++i) lse[i] = 0.f;
        for (int64_t i = 0; i < slots; ++i) mass[i] = -1.f;
        must(graphattn_run_mass(plan, q.p, pool.p, lse.p, nullptr, 1.f, mass.p, nullptr), "mass");
        // (every weight is 1: a slot counts the rows and heads that see it)
        std::vector<double> want(slots, 0.);
        for (int64_t b = 0; b < h[7]; ++b) {
          const int c = many ? g.counts[b] : 1;
          for (int64_t e = g.poff[b]; e < g.poff[b + 1]; ++e) {
            const int s = g.segs[e];
            for (int t = 0; t < g.len[s]; ++t) {
              const int late = e + 1 == g.poff[b + 1] ? std::max(0, t - (g.len[s] - c)) : 0;
              want[(int64_t)g.pages[g.off[s] + t / 16] * 16 + t % 16] += (double)(c - late) * p.num_q_heads;
            }
          }
        }
        for (int64_t i = 0; i < slots; ++i)
          if (mass[i] != (want[i] ? want[i] : -1.)) {
            std::fprintf(stderr, "mass[%lld] is %g, not %g\n", (long long)i, mass[i], want[i]);
            std::exit(1);
          }
      }
      if (h[0] == 1 || graphattn_kv_page_bytes(&p) * g.num_pages > (64 << 20)) break;
    }
    graphattn_plan_destroy(plan);
  }
  std::fclose(f);
  std::printf("ok %s\n", path);
}

void evict(int number) {
  const int S = spread(1, 12);
  Graph g;
  for (int s = 0; s < S; ++s) fill(g, U(0, 5) ? spread(1, 3000) : spread(1, 40000));
  for (int n : g.len) g.off.push_back(g.off.back() + (n + 15) / 16);
  g.num_pages = g.off.back() + U(0, 2);
  Ints order((size_t)g.num_pages);
  for (size_t i = 0; i < order.size(); ++i) order[i] = (int32_t)i;
  std::shuffle(order.begin(), order.end(), rng);
  g.pages.assign(order.begin(), order.begin() + g.off.back());
  const int first = U(0, 2) ? U(0, 20) : U(0, 2000), recent = U(0, 2) ? U(0, 300) : U(0, 3000);
  Ints keep;
  size_t total = 0;
  for (int n : g.len) {
    keep.push_back(U(std::min(n, first + recent), n));
    total += keep.back();
  }
  Dev<float> mass((size_t)(16 * g.num_pages));
  const int values = U(0, 4);
  for (size_t i = 0; i < mass.n; ++i) {
    const int r = U(0, 99);
    mass[i] = values == 0 ? (float)U(0, 3) : values == 1 ? (float)std::exp(3 * normal()) : values == 2 ? (float)normal()
              : values == 3 ? (r < 60 ? 0.f : (float)std::exp(20 * normal())) : 1.f;
    if (values == 2 && r < 3) mass[i] = r == 0 ? NAN : r == 1 ? INFINITY : -INFINITY;
    if (values == 0 && r < 3) mass[i] = -0.f;
  }
  Dev<int32_t> pos(total), words(total);
  const ga_segment_table st = g.table();
  ga_evict* h = nullptr;
  must(graphattn_evict_create(&st, keep.data(), first, recent, g.num_pages, nullptr, &h), "evict_create");
  emu::seed = 88172645463325252ull + 2 * rng() + 1;
  must(graphattn_evict_select(h, mass.p, pos.p, words.p, nullptr), "evict_select");
  size_t at = 0;
  for (int s = 0; s < S; ++s) {
    Ints order2(g.len[s]);
    for (int t = 0; t < g.len[s]; ++t) order2[t] = t;
    auto key = [&](int t) -> double {
      if (t < first || t >= g.len[s] - recent) return 1e300;
      const float m = mass[(size_t)g.pages[g.off[s] + t / 16] * 16 + t % 16];
      return std::isnan(m) ? 1e299 : std::isinf(m) ? (m > 0 ? 1e298 : -1e298) : m;
    };
    std::stable_sort(order2.begin(), order2.end(), [&](int a, int b) { return key(a) > key(b); });
    order2.resize(keep[s]);
    std::sort(order2.begin(), order2.end());
    for (int t : order2) {
      if (pos[at] != t || words[at] != g.pages[g.off[s] + t / 16] * 16 + t % 16) {
        std::fprintf(stderr, "segment %d of %d tokens: %d at %zu, not %d\n", s, g.len[s], pos[at], at, t);
        std::exit(1);
      }
      ++at;
    }
  }
  graphattn_evict_destroy(h);
  std::printf("%d: %d segments, %zu of %lld slots stay\n", number, S, total, (long long)(16 * g.num_pages));
}

void cache(int number) {
  const int hd = U(0, 8), D = kHeads[hd][2], H = kHeads[hd][1], n = spread(1, 400);
  const ga_params p{H, H, D, 16, n / 8 + 3, U(0, 3) ? GA_MXFP4 : U(0, 1) ? GA_BF16 : GA_F32, 0.f, 0};
  Pool pool(p);
  const size_t elt = p.dtype == GA_F32 ? 4 : 2;
  Ints order((size_t)(p.num_pages * 16));
  for (size_t i = 0; i < order.size(); ++i) order[i] = (int32_t)i;
  std::shuffle(order.begin(), order.end(), rng);
  for (int i = 0; i < n; ++i) pool.put(order[i]);
  Dev<int32_t> src(n), dst(n);
  for (int i = 0; i < n; ++i) { src[i] = order[i]; dst[i] = order[n + i]; }
  const int bad = U(0, n - 1);
  const int32_t outside[4] = {-1, (int32_t)(p.num_pages * 16), INT32_MIN, INT32_MAX};
  dst[bad] = outside[U(0, 3)];
  Dev<unsigned char> k((size_t)n * H * D * elt), v(k.n), k2(k.n), v2(k.n);
  emu::seed = 88172645463325252ull + 2 * rng() + 1;
  // Read, moved, read again, appended elsewhere from what was read, read a third time: the same bits.
  must(graphattn_kv_read(pool.mem.p, src.p, n, k.p, v.p, &p, nullptr), "read");
  must(graphattn_kv_copy(pool.mem.p, src.p, dst.p, n, &p, nullptr), "copy");
  for (int pass = 0; pass < 2; ++pass) {
    std::memcpy(k2.p, k.p, k.n);
    std::memcpy(v2.p, v.p, v.n);
    const size_t row = (size_t)H * D * elt;
    for (int i = 0; i < n; ++i)
      if (i != bad) { std::memset(k2.p + i * row, 1, row); std::memset(v2.p + i * row, 1, row); }
    must(graphattn_kv_read(pool.mem.p, dst.p, n, k2.p, v2.p, &p, nullptr), "read");
    if (std::memcmp(k.p, k2.p, k.n) || std::memcmp(v.p, v2.p, v.n)) {
      for (size_t i = 0; i < k.n; ++i)
        if (k[i] != k2[i] || v[i] != v2[i]) {
          std::fprintf(stderr, "%d tokens of %d x %d, type %d, bad %d: byte %zu is %02x %02x, not %02x %02x\n", n, H, D, p.dtype, bad, i,
                       k2[i], v2[i], k[i], v[i]);
          break;
        }
      std::fprintf(stderr, "tokens differ after pass %d\n", pass);
      std::exit(1);
    }
    if (pass) break;
    std::memset(pool.mem.p, 0x5a, pool.mem.n);
    must(graphattn_kv_append(pool.mem.p, k.p, v.p, dst.p, n, &p, nullptr), "append");
  }
  for (int i = 0; i < n; ++i)
    for (int h = 0; h < H; ++h)
      for (int c = 0; c < D; ++c)
        for (int kv = 0; kv < 2; ++kv) {
          const unsigned char* b = (kv ? v.p : k.p) + ((size_t)(i * H + h) * D + c) * elt;
          const double x = elt == 4 ? *reinterpret_cast<const float*>(b) : of_bf16(*reinterpret_cast<const uint16_t*>(b));
          if (x != pool.v[kv][pool.at(src[i], h, c)]) { std::fprintf(stderr, "token %d differs\n", i); std::exit(1); }
        }
  std::printf("%d: %d tokens of %d x %d, type %d\n", number, n, H, D, p.dtype);
}

}  // namespace

int main(int argc, char** argv) {
  const std::string kind = argc > 1 ? argv[1] : "attn";
  if (kind == "file") {
    given(argv[2]);
    return 0;
  }
  const int cases = argc > 2 ? std::atoi(argv[2]) : 5, seed = argc > 3 ? std::atoi(argv[3]) : 1;
  for (int i = 0; i < cases; ++i) {
    rng.seed(1000 * seed + i);
    if (kind == "attn") attend(false, i);
    else if (kind == "mass") attend(true, i);
    else if (kind == "evict") evict(i);
    else cache(i);
  }
  std::printf("ok, %ld operations of a part of a wave\n", emu::partial_ops);
}
