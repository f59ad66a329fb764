// Whether a plan of the 8-bit cache loads tokens' pages past the caches: where hardly a page that its queries read is read by
// two requests.  Host-only, under sanitizers.
#include "plan.h"
#include "q8.h"
#include "wavepp_q8.h"

#include <algorithm>
#include <cstdio>
#include <vector>

namespace wavepp {
hipError_t launch_q8_append(const DevPlan&, const Q8Dev&, const void*, const void*, void*, void*, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_q8_read(const DevPlan&, const Q8Dev&, const void*, const void*, void*, void*, hipStream_t) { return hipErrorNotSupported; }
hipError_t launch_q8_attention(const DevPlan&, const Q8Dev&, int32_t, const void*, const void*, const void*, void*, float*, hipStream_t) {
  return hipErrorNotSupported;
}
}  // namespace wavepp

static bool bad = false;

// R requests of one token behind `pages` cached pages of 64, the first `shared` of which are the same ones (page 0 alone where
// `one`), with a window of so many keys (0: none).
static void expect(bool stream, int R, int pages, int shared, bool one, int window, int line) {
  const int stride = pages + 1;
  std::vector<int32_t> prefix(R, 64 * pages), chunk(R, 1), table(size_t(R) * stride), begin(R, std::max(0, 64 * pages + 1 - window));
  int next = shared + 1;
  for (int r = 0; r < R; ++r)
    for (int b = 0; b < stride; ++b) table[size_t(r) * stride + b] = b < shared ? (one ? 0 : b) : next++;
  const wavepp_attn_shape s{32, 8, 128, 128, 64, next, 0, 0.1f};
  const wavepp_batch batch{R, prefix.data(), chunk.data(), table.data(), stride};
  const wavepp_q8_scores sc{0.0f, nullptr, begin.data(), nullptr};
  wavepp_plan* p = nullptr;
  if (wavepp_q8_plan(&s, &batch, window ? &sc : nullptr, 0, &p) != WAVEPP_OK) {
    printf("line %d: no plan: %s\n", line, wavepp_last_error());
    bad = true;
    return;
  }
  if (p->stream != stream) {
    printf("line %d: past the caches: %d\n", line, p->stream);
    bad = true;
  }
  wavepp_plan_destroy(p);
}
#define EXPECT(...) expect(__VA_ARGS__, __LINE__)

int main() {
  EXPECT(true, 16, 40, 0, false, 0);             // pages of their own
  EXPECT(false, 16, 40, 30, false, 0);           // a shared prompt
  EXPECT(true, 1, 40, 30, false, 0);             // of one request
  EXPECT(true, 16, 40, 30, false, 500);          // a window that has left it
  EXPECT(true, 16, 40, 30, true, 500);           // or one page that stands for all that it has left
  EXPECT(false, 16, 40, 38, false, 500);         // a window that still reads it
  EXPECT(false, 16, 40, 30, false, 64 * 40 + 1); // a window over everything
  EXPECT(true, 16, 40, 0, false, 64 * 40 + 1);
  EXPECT(true, 16, 40, 40, false, 1);            // which reads the new token alone
  if (!bad) printf("q8_shared_pages ok\n");
  return bad;
}
