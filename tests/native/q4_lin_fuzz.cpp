// Plans of the 4-bit cache and of linear attention over seeded random waves, host-only, under sanitizers: every item of an
// accepted plan within its request, all of a request's tokens and keys covered once, in order.
#include "lin_host.cpp"
#include "q4.h"
#include "wavepp_q4.h"

#include <cstdio>
#include <cstdlib>
#include <random>

namespace wavepp {
hipError_t launch_lin(const LinDevPlan&, const void*, const void*, const void*, const float*, float*, void*, hipStream_t) {
  return hipErrorNotSupported;
}
hipError_t launch_q4_append(const DevPlan&, const void*, const void*, void*, void*, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_q4_read(const DevPlan&, const void*, const void*, void*, void*, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_q4_attention(const DevPlan&, int32_t, const void*, const void*, const void*, void*, float*, hipStream_t) {
  return hipErrorNotSupported;
}
}  // namespace wavepp

#define CHECK(x) \
  if (!(x)) { printf("failed: %s (line %d)\n", #x, __LINE__); return 1; }

static int lin(std::mt19937& g) {
  auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(g); };
  const int qk = pick(1, 8), R = pick(0, 9), dims[2] = {64, 128};
  wavepp_lin_shape s{qk * pick(1, 8), qk, dims[pick(0, 1)], dims[pick(0, 1)], 2 * R + 1, pick(0, 1), 0.5f};
  std::vector<int32_t> len, in, out;
  int64_t tokens = 0;
  for (int r = 0; r < R; ++r) {
    len.push_back(pick(0, 3) == 0 ? pick(0, 12) : pick(0, 1) ? pick(0, 300) : pick(0, 40000));
    out.push_back(r);
    in.push_back(pick(0, 2) == 0 ? -1 : pick(0, 1) ? r : R + r);
    tokens += len.back();
  }
  wavepp_lin_batch b{R, len.data(), in.data(), out.data()};
  wavepp_lin_plan_t* p = nullptr;
  CHECK(wavepp_lin_plan(&s, &b, &p) == WAVEPP_OK && p->total_tokens == tokens);
  std::vector<int> used(size_t(p->num_parts), 0), start(size_t(p->num_parts), 0);
  int64_t cu = 0;
  CHECK(std::is_partitioned(p->segments.begin(), p->segments.end(), [](const LinItem& x) { return x.part_out >= 0; }));
  for (int i = 0; i < int(p->segments.size()); ++i) CHECK((p->segments[i].part_out >= 0) == (i < p->num_ahead));
  for (int r = 0; r < R; cu += len[r], ++r) {
    int64_t at = cu;
    int32_t before = -1;
    bool ended = len[r] == 0;
    while (at < cu + len[r]) {
      const LinItem* found = nullptr;
      for (const auto* v : {&p->steps, &p->segments})
        for (const LinItem& x : *v)
          if (x.cu == at) found = &x;
      CHECK(found && found->len > 0 && at + found->len <= cu + len[r]);
      if (at == cu) {
        CHECK(found->part_in >= 0 ? in[r] == out[r] && ++start[size_t(found->part_in)] == 1 : found->state_in == in[r]);
      } else {
        CHECK(found->part_in >= 0 && found->part_in == before && found->state_in == -1);
      }
      before = found->part_out;
      at += found->len;
      if (before >= 0) CHECK(found->len % kLinBlock == 0 && found->state_out == -1 && ++used[size_t(before)] == 1);
      if (before < 0) {
        CHECK(at == cu + len[r] && found->state_out == out[r]);
        ended = true;
      }
    }
    CHECK(ended);
  }
  for (const LinScan& sc : p->scans) {
    CHECK(sc.count > 0 && sc.first_part >= 0 && sc.first_part + sc.count <= p->num_parts);
    for (int i = 0; i < sc.count; ++i) CHECK(used[size_t(sc.first_part + i)]++ == 1);
    if (sc.start_part >= 0) CHECK(start[size_t(sc.start_part)]++ == 1);
  }
  for (size_t i = 0; i < used.size(); ++i) CHECK(used[i] + start[i] == 2);
  wavepp_lin_info info;
  CHECK(wavepp_lin_get_info(p, &info) == WAVEPP_OK && size_t(info.workspace_bytes) == wavepp_lin_workspace_bytes(p));
  wavepp_lin_destroy(p);
  return 0;
}

static int q4(std::mt19937& g) {
  auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(g); };
  const int kv = pick(1, 8), G = pick(1, 33), R = pick(1, 40), B = pick(0, 1) ? 16 : 64, D = pick(0, 1) ? 64 : 128;
  std::vector<int32_t> pre, len, table;
  int longest = 1;
  const int most = pick(0, 1) ? 4 : 200, far = pick(0, 1) ? 300 : 40000;
  for (int r = 0; r < R; ++r) {
    pre.push_back(pick(0, far));
    len.push_back(pick(0, most));
    longest = std::max(longest, pre.back() + len.back());
  }
  const int stride = (longest + B - 1) / B;
  for (int i = 0; i < R * stride; ++i) table.push_back(i);
  wavepp_attn_shape s{G * kv, kv, D, D, B, R * stride, 0, 0.1f};
  wavepp_batch b{R, pre.data(), len.data(), table.data(), stride};
  wavepp_plan* p = nullptr;
  CHECK(wavepp_q4_plan(&s, &b, pick(0, 2) ? 0 : pick(1, 9), &p) == WAVEPP_OK);
  wavepp_plan_info info;
  wavepp_plan_get_info(p, &info);
  std::vector<int32_t> items(8 * size_t(info.num_items) + 8);
  const int n = wavepp_plan_get_items(p, items.data(), info.num_items);
  std::vector<int64_t> pairs(size_t(R), 0);
  for (int i = 0; i < n; ++i) {
    const int32_t* w = &items[8 * size_t(i)];
    if (w[3] == 0) continue;
    CHECK(w[0] >= 0 && w[0] < R && w[1] >= 0 && w[1] < kv && w[2] >= 0 && w[3] > 0 && w[3] <= info.rows_per_item);
    CHECK(int64_t(w[2]) + w[3] <= int64_t(len[w[0]]) * G && w[4] >= 0 && w[4] < w[5] && w[4] % info.kv_tile == 0);
    CHECK(w[5] <= pre[w[0]] + (w[2] + w[3] - 1) / G + 1);
    CHECK(w[6] == -1 || int64_t(w[6]) + w[3] <= info.partial_rows);
    pairs[size_t(w[0])] += int64_t(w[3]) * (w[5] - w[4]);
  }
  for (int r = 0; r < R; ++r) {                      // rows x keys of all items: each row tile up to its last row's key
    int64_t want = 0;
    for (int64_t row = 0; row < int64_t(len[r]) * G; row += info.rows_per_item) {
      const int64_t rows = std::min<int64_t>(info.rows_per_item, int64_t(len[r]) * G - row);
      want += rows * (pre[r] + (row + rows - 1) / G + 1);
    }
    CHECK(pairs[size_t(r)] == want * kv);
  }
  wavepp_plan_destroy(p);
  return 0;
}

int main() {
  std::mt19937 g(7);
  for (int i = 0; i < 1500; ++i)
    if (lin(g) || q4(g)) {
      printf("wave %d\n", i);
      return 1;
    }
  puts("q4_lin_fuzz ok");
  return 0;
}
