// Plans of the 8-bit cache with random scores, host-only, under sanitizers: every item within its request, every new slot in
// one block of the append, in order; every allocation of such a plan failing once.  And whether two sets of rows meet, as the
// rotary positions' call decides it, against every byte.
#include "rope_host.cpp"
#include "q4.h"
#include "q8.h"
#include "wavepp_q8.h"

#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <set>
#include <vector>

namespace wavepp {
hipError_t launch_q8_append(const DevPlan&, const Q8Dev&, const void*, const void*, void*, void*, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_q8_read(const DevPlan&, const Q8Dev&, const void*, const void*, void*, void*, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_q8_attention(const DevPlan&, const Q8Dev&, int32_t, const void*, const void*, const void*, void*, float*, hipStream_t) {
  return hipErrorNotSupported;
}
hipError_t launch_rope(const DevPlan&, const RopeDev&, const double*, hipStream_t) { return hipErrorNotSupported; }
}  // namespace wavepp

static long left = -1;                               // allocations until the one that fails; < 0: none does
static bool fails() { return left >= 0 && left-- == 0; }
void* operator new(size_t n) {
  if (fails()) throw std::bad_alloc();
  if (void* p = malloc(n ? n : 1)) return p;
  throw std::bad_alloc();
}
void* operator new(size_t n, const std::nothrow_t&) noexcept { return fails() ? nullptr : malloc(n ? n : 1); }
void operator delete(void* p) noexcept { free(p); }
void operator delete(void* p, size_t) noexcept { free(p); }

#define CHECK(x) \
  if (!(x)) { printf("failed: %s (line %d)\n", #x, __LINE__); return 1; }

static int plans(std::mt19937& g, bool memory) {
  auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(g); };
  const int kv = pick(1, 4), G = pick(1, 12), D = pick(0, 1) ? 64 : 128, B = pick(0, 1) ? 16 : 64, R = memory ? 4 : pick(0, 8);
  std::vector<int32_t> prefix, chunk, begin, end, table;
  std::vector<float> slopes;
  int longest = 1, T = 0;
  for (int r = 0; r < R; ++r) {
    prefix.push_back(pick(0, 1) ? pick(0, 40) : pick(0, 9000));
    chunk.push_back(pick(0, 2) ? pick(0, 4) : pick(0, 400));
    longest = std::max(longest, prefix[r] + chunk[r]);
    for (int i = 0; i < chunk[r]; ++i, ++T) {
      const int n = prefix[r] + chunk[r];
      begin.push_back(pick(0, n));
      end.push_back(pick(0, n));
    }
  }
  for (int h = 0; h < kv * G; ++h) slopes.push_back(0.01f * float(h));
  const int stride = (longest + B - 1) / B + pick(0, 2);
  for (int i = 0; i < R * stride; ++i) table.push_back(i);
  for (int i = R * stride - 1; i > 0; --i) std::swap(table[i], table[pick(0, i)]);
  const wavepp_attn_shape s{kv * G, kv, D, D, B, std::max(1, R * stride), 0, 0.1f};
  const wavepp_batch b{R, prefix.data(), chunk.data(), table.data(), stride};
  wavepp_q8_scores sc{pick(0, 1) ? 30.0f : 0.0f, pick(0, 1) ? slopes.data() : nullptr, pick(0, 1) ? begin.data() : nullptr,
                      pick(0, 1) ? end.data() : nullptr};
  const int splits = pick(0, 4);
  if (memory) {
    for (long n = 0; n < 100000; ++n) {
      wavepp_plan* p = nullptr;
      left = n;
      const int st = wavepp_q8_plan(&s, &b, &sc, splits, &p);
      const bool all = left >= 0;
      left = -1;
      CHECK(st == WAVEPP_OK || (st == WAVEPP_EINVAL && !p));
      if (p) wavepp_plan_destroy(p);
      if (all) return st == WAVEPP_OK ? 0 : 1;
    }
    return 1;
  }
  wavepp_plan* p = nullptr;
  CHECK(wavepp_q8_plan(&s, &b, pick(0, 3) ? &sc : nullptr, splits, &p) == WAVEPP_OK && p->total_tokens == T);
  for (const WorkItem& w : p->items) {
    if (w.rows == 0) continue;
    CHECK(w.req >= 0 && w.req < R && w.row0 >= 0 && w.row0 + w.rows <= chunk[w.req] * G);
    CHECK(w.kv_begin >= 0 && w.kv_end <= prefix[w.req] + chunk[w.req] && (w.kv_begin < w.kv_end || w.kv_end == 0));
    CHECK(w.part < 0 || w.part + w.rows <= p->partial_rows);
  }
  const auto* blocks = reinterpret_cast<const Q8Block*>(p->blob.data() + p->off_blocks);
  int at = 0;
  for (int r = 0, cu = 0; r < R; cu += chunk[r], ++r)
    for (int i = 0; i < chunk[r];) {
      CHECK(at < p->num_blocks);
      const Q8Block& x = blocks[at++];
      const int pos = prefix[r] + i, lo = x.span & 255, hi = x.span >> 8;
      CHECK(x.page == table[r * stride + pos / B] && x.slot % kQ8Block == 0 && x.slot + lo == pos % B && x.token == cu + i);
      CHECK(lo < hi && hi <= kQ8Block && (hi == kQ8Block || i + hi - lo == chunk[r]));
      i += hi - lo;
    }
  CHECK(at == p->num_blocks && p->off_blocks + sizeof(Q8Block) * size_t(at) <= p->blob.size());
  wavepp_plan_destroy(p);
  return 0;
}

static int meeting(std::mt19937& g) {
  auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(g); };
  for (int n = 0; n < 20000; ++n) {
    const int wa = pick(1, 9), wb = pick(1, 9), sa = pick(wa, 20), sb = pick(0, 3) ? std::max(sa, wb) : pick(wb, 20), T = pick(1, 6);
    const int a = 200 + pick(-60, 60), b = 200 + pick(-60, 60);
    std::set<int> bytes;
    for (int i = 0; i < T; ++i)
      for (int k = 0; k < wa; ++k) bytes.insert(a + i * sa + k);
    bool met = false;
    for (int i = 0; i < T; ++i)
      for (int k = 0; k < wb; ++k) met = met || bytes.count(b + i * sb + k);
    const bool says = rows_meet(uintptr_t(a), sa, wa, uintptr_t(b), sb, wb, T);
    CHECK(sa == sb ? says == met : says || !met);
  }
  return 0;
}

int main() {
  std::mt19937 g(7);
  for (int i = 0; i < 400; ++i)
    if (plans(g, false)) return 1;
  for (int i = 0; i < 6; ++i)
    if (plans(g, true)) return 1;
  if (meeting(g)) return 1;
  printf("q8_rope_fuzz ok\n");
  return 0;
}
