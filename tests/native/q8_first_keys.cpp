// The first key that a work item of the 8-bit cache loads is the first that one of its queries sees, and its request's span the
// one it was planned for: random waves, tokens beside chunks, with random intervals.  Host-only, under sanitizers.
#include "plan.h"
#include "q8.h"
#include "wavepp_q8.h"

#include <algorithm>
#include <cstdio>
#include <random>
#include <vector>

namespace wavepp {
hipError_t launch_q8_append(const DevPlan&, const Q8Dev&, const void*, const void*, void*, void*, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_q8_read(const DevPlan&, const Q8Dev&, const void*, const void*, void*, void*, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_q8_attention(const DevPlan&, const Q8Dev&, int32_t, const void*, const void*, const void*, void*, float*, hipStream_t) {
  return hipErrorNotSupported;
}
}  // namespace wavepp

using namespace wavepp;

#define CHECK(x) \
  if (!(x)) { printf("failed: %s (line %d)\n", #x, __LINE__); return 1; }

static int wave(std::mt19937& g) {
  auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(g); };
  const int kv = pick(1, 3), G = pick(1, 12), D = pick(0, 1) ? 64 : 128, B = pick(0, 1) ? 16 : 64, R = pick(1, 8);
  std::vector<int32_t> prefix, chunk, cu, begin, end, table;
  int longest = 1;
  for (int r = 0; r < R; ++r) {
    prefix.push_back(pick(0, 1) ? pick(0, 40) : pick(0, 9000));
    chunk.push_back(pick(0, 2) ? pick(0, 4) : pick(0, 400));
    cu.push_back(int32_t(begin.size()));
    const int n = prefix[r] + chunk[r], window = pick(1, 2000);
    longest = std::max(longest, n);
    const bool any = pick(0, 1);
    for (int i = 0; i < chunk[r]; ++i) {
      begin.push_back(any ? pick(0, n) : std::max(0, prefix[r] + i + 1 - window));
      end.push_back(any ? pick(0, n) : prefix[r] + i + 1);
    }
  }
  const int stride = (longest + B - 1) / B;
  for (int i = 0; i < R * stride; ++i) table.push_back(i);
  const wavepp_attn_shape s{kv * G, kv, D, D, B, R * stride, 0, 0.1f};
  const wavepp_batch b{R, prefix.data(), chunk.data(), table.data(), stride};
  const bool causal = pick(0, 4) == 0;
  const wavepp_q8_scores sc{pick(0, 1) ? 30.0f : 0.0f, nullptr, causal ? nullptr : begin.data(), causal ? nullptr : end.data()};
  wavepp_plan* p = nullptr;
  CHECK(wavepp_q8_plan(&s, &b, &sc, pick(0, 4), &p) == WAVEPP_OK);
  const auto* at = reinterpret_cast<const Q8ItemReq*>(p->blob.data() + p->off_item_reqs);
  CHECK(p->off_item_reqs + sizeof(Q8ItemReq) * p->items.size() <= p->blob.size());
  for (size_t i = 0; i < p->items.size(); ++i) {
    const WorkItem& w = p->items[i];
    if (w.rows == 0) continue;
    CHECK(at[i].prefix == prefix[w.req] && at[i].cu == cu[w.req] && at[i].bt_row == w.req * stride);
    int first = causal ? 0 : INT32_MAX, last = 0;
    for (int t = w.row0 / G; !causal && t <= (w.row0 + w.rows - 1) / G; ++t) {
      const int x = begin[size_t(cu[w.req] + t)], y = end[size_t(cu[w.req] + t)];
      if (x < y) first = std::min(first, x), last = std::max(last, y);
    }
    if (first == INT32_MAX) {
      CHECK(w.kv_begin == 0 && w.kv_end == 0);
      continue;
    }
    CHECK(at[i].first == first && (causal || w.kv_end <= last) && w.kv_begin < w.kv_end);
    CHECK(first / B < stride && (w.kv_end - 1) / B < stride && first < w.kv_end);       // what the loads are kept within
  }
  wavepp_plan_destroy(p);
  return 0;
}

int main() {
  std::mt19937 g(11);
  for (int i = 0; i < 600; ++i)
    if (wave(g)) return 1;
  printf("q8_first_keys ok\n");
  return 0;
}
