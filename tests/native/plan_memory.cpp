// Every host allocation of a wave's plan, one at a time, fails: the entry points say so and never throw into their C
// callers, and nothing that they had allocated by then is lost (the sanitizer's leak check).
#include "lin.h"
#include "q4.h"
#include "wavepp_kda.h"
#include "wavepp_lin.h"
#include "wavepp_q4.h"

#include <cstdio>
#include <cstdlib>
#include <new>
#include <vector>

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

template <typename Make>
static int each_allocation(const char* name, Make make) {
  long refused = 0;
  for (long n = 0; n < 100000; ++n) {
    left = n;
    const int st = make();
    const bool all = left >= 0;                      // no allocation failed
    left = -1;
    if (all) {
      printf("%s: %ld allocations\n", name, n);
      return st == WAVEPP_OK && refused > 3 ? 0 : 1;
    }
    refused += st != WAVEPP_OK;
    if (st != WAVEPP_EINVAL && st != WAVEPP_OK) {    // (a stable sort does without its buffer)
      printf("%s: allocation %ld failed, status %d\n", name, n, st);
      return 1;
    }
  }
  return 1;
}

int main() {
  std::vector<int32_t> prefix{9000, 300, 40, 0}, chunk{1, 700, 12, 200}, table(4 * 200), in{-1, 1, 2, -1}, out{0, 1, 3, 4};
  for (size_t i = 0; i < table.size(); ++i) table[i] = int32_t(i);
  wavepp_batch batch{4, prefix.data(), chunk.data(), table.data(), 200};
  wavepp_attn_shape grouped{16, 2, 128, 128, 64, 800, 0, 0.1f}, latent{16, 1, 576, 512, 64, 800, 1, 0.1f};
  auto attn = [&](auto entry, const wavepp_attn_shape& s) {
    wavepp_plan* p = nullptr;
    const int st = entry(&s, &batch, 0, &p);
    if ((st == WAVEPP_OK) != (p != nullptr)) abort();
    wavepp_plan_destroy(p);
    return st;
  };
  int bad = each_allocation("wavepp_attn_plan", [&] { return attn(wavepp_attn_plan, grouped); });
  bad |= each_allocation("wavepp_attn_plan, latent", [&] { return attn(wavepp_attn_plan, latent); });
  bad |= each_allocation("wavepp_q4_plan", [&] { return attn(wavepp_q4_plan, grouped); });
  bad |= each_allocation("wavepp_lin_plan", [&] {
    wavepp_lin_shape s{8, 4, 128, 64, 5, 1, 0.5f};
    wavepp_lin_batch b{4, chunk.data(), in.data(), out.data()};
    wavepp_lin_plan_t* p = nullptr;
    const int st = wavepp_lin_plan(&s, &b, &p);
    if ((st == WAVEPP_OK) != (p != nullptr)) abort();
    wavepp_lin_destroy(p);
    return st;
  });
  std::vector<int32_t> lens, from, to;                // enough chains of unlike lengths that they are given out by load
  for (int r = 0; r < 12; ++r) lens.push_back(64 * (r + 1)), from.push_back(-1), to.push_back(r);
  bad |= each_allocation("wavepp_kda_plan", [&] {
    wavepp_kda_shape s{64, 128, 128, 12};
    wavepp_kda_batch b{12, lens.data(), from.data(), to.data()};
    wavepp_kda_plan_t* p = nullptr;
    const int st = wavepp_kda_plan(&s, &b, &p);
    if ((st == WAVEPP_OK) != (p != nullptr)) abort();
    wavepp_kda_destroy(p);
    return st;
  });
  if (bad) return 1;
  puts("plan_memory ok");
  return 0;
}
