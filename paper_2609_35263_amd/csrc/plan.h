// The plan of an attention wave, as the host code of the bf16 cache (host.cpp), of the 4-bit cache (q4_host.cpp) and of the
// 8-bit cache (q8_host.cpp) share it.  Not part of the public ABI.
#pragma once

#include "wavepp_attn.h"
#include "internal.h"

#include <vector>

namespace wavepp {

enum class Cache { bf16, q4, q8 };    // what the wave's pages hold

// Scores other than the causal ones of wavepp_attn.h, all host memory: see wavepp_q8.h.
struct PlanScores {
  float cap = 0.0f;
  const float* slopes = nullptr;
  const int32_t *key_begin = nullptr, *key_end = nullptr;
};

}  // namespace wavepp

struct wavepp_plan {
  wavepp_attn_shape shape;
  wavepp::Cache cache = wavepp::Cache::bf16;
  int32_t num_requests = 0;
  int32_t bt_stride = 0;
  int64_t total_tokens = 0;
  uint32_t serial = 0;
  int32_t rows_per_item = 0;
  int32_t kv_tile = 0;
  int32_t max_splits_used = 1;
  int32_t num_real_items = 0;
  int32_t num_few = 0;                // the last items, which run with few rows over 4-bit or 8-bit pages
  int32_t few_rows = 0;               // most rows of such an item
  bool stream = false;                // 8-bit pages: hardly a page is in two requests
  std::vector<wavepp::WorkItem> items;
  std::vector<wavepp::MergeItem> merges;      // those that merge_wide_kernel takes first
  int32_t num_merge_wide = 0, merge_rows = 0;
  int64_t partial_rows = 0;
  // metadata blob (uploaded as is) and its sub-array offsets
  std::vector<unsigned char> blob;
  size_t off_reqs = 0, off_bt = 0, off_items = 0, off_merges = 0;
  // 8-bit pages: the blocks that the wave's tokens touch, every item's request; the scores' arrays, 0 where the plan has none
  size_t off_blocks = 0, off_item_reqs = 0, off_ranges = 0, off_slopes = 0;
  int32_t num_blocks = 0;
  float cap = 0.0f;
  size_t meta_bytes = 0;       // blob size rounded up to 256
  size_t off_opart = 0, off_lpart = 0;
  size_t workspace_bytes = 0;
};

namespace wavepp {

// Validates a wave and plans it for pages of that kind; scores may be NULL and are of 8-bit pages alone.
int plan_wave(const wavepp_attn_shape* shape, const wavepp_batch* batch, int32_t max_splits, Cache cache,
              const PlanScores* scores, wavepp_plan** out);
int check_workspace(const wavepp_plan* plan, void* ws, size_t ws_bytes);
// Everything a launch needs, with the plan's metadata and partials at `ws`.
DevPlan make_dev(const wavepp_plan* plan, void* ws);
// WAVEPP_EINVAL where the plan is of another kind of cache, whose pages have another size.
int require_cache(const wavepp_plan* plan, Cache cache);

}  // namespace wavepp
