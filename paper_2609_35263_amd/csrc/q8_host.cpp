// Host side of the 8-bit paged cache: its plans, checks of arguments and launches.
#include "wavepp_q8.h"
#include "internal.h"
#include "plan.h"
#include "q8.h"

using namespace wavepp;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// Whether the launches can have as many workgroups as the wave needs.
int check_moves(const wavepp_plan* plan) {
  const int64_t n = q8_moves(plan->num_blocks, plan->shape.num_kv_heads);
  return n <= kQ8MostMoves ? WAVEPP_OK
                           : set_error(WAVEPP_EUNSUPPORTED, "the wave touches %d blocks of 16 slots in %d KV heads: store or read it in parts",
                                       plan->num_blocks, plan->shape.num_kv_heads);
}
int check_items(const wavepp_plan* plan) {
  const int64_t few = plan->num_few, many = int64_t(plan->items.size()) - few;
  return few <= kQ8MostFew && many <= kQ8MostMany
             ? WAVEPP_OK
             : set_error(WAVEPP_EUNSUPPORTED, "the wave has %lld tiles of few rows and %lld of many: plan it in parts", (long long)few,
                         (long long)many);
}

// What every call on a plan checks first.  *run: whether there is anything to enqueue.
int check_call(const wavepp_plan* plan, void* workspace, size_t ws_bytes, int (*check_size)(const wavepp_plan*), bool* run) {
  clear_error();
  *run = false;
  if (!plan) return set_error(WAVEPP_EINVAL, "plan is NULL");
  int st = require_cache(plan, Cache::q8);
  if (!st) st = check_workspace(plan, workspace, ws_bytes);
  if (st || plan->total_tokens == 0) return st;
  if ((st = check_size(plan))) return st;
  *run = true;
  return require_upload(workspace, plan->serial, "wavepp_attn_plan_upload");
}

int check_buffers(const void* a, const void* b, const void* c, const void* d) {
  if (!a || !b || !c || !d) return set_error(WAVEPP_EINVAL, "a device buffer is NULL");
  if (!aligned16(a) || !aligned16(b) || !aligned16(c) || !aligned16(d))
    return set_error(WAVEPP_EINVAL, "device buffers must be 16-byte aligned");
  return WAVEPP_OK;
}

Q8Dev make_q8(const wavepp_plan* plan, void* ws) {
  auto* base = static_cast<unsigned char*>(ws);
  Q8Dev x{};
  x.blocks = reinterpret_cast<const Q8Block*>(base + plan->off_blocks);
  x.item_reqs = reinterpret_cast<const Q8ItemReq*>(base + plan->off_item_reqs);
  x.num_blocks = plan->num_blocks;
  x.few_rows = plan->few_rows;
  x.stream = plan->stream;
  if (plan->off_ranges) x.ranges = reinterpret_cast<const TokenRange*>(base + plan->off_ranges);
  if (plan->off_slopes) x.slopes = reinterpret_cast<const float*>(base + plan->off_slopes);
  x.cap = plan->cap;
  return x;
}

}  // namespace

extern "C" {

size_t wavepp_q8_page_bytes(int32_t head_dim, int32_t page_size) {
  if ((head_dim != 64 && head_dim != 128) || (page_size != 16 && page_size != 64)) return 0;
  return size_t(page_size) * head_dim + kQ8ScaleBytes;
}

int wavepp_q8_plan(const wavepp_attn_shape* shape, const wavepp_batch* batch, const wavepp_q8_scores* scores,
                   int32_t max_splits, wavepp_plan** out) {
  return guarded([&] {
    PlanScores s;
    if (scores) s = {scores->cap, scores->slopes, scores->key_begin, scores->key_end};
    return plan_wave(shape, batch, max_splits, Cache::q8, scores ? &s : nullptr, out);
  });
}

int wavepp_q8_append_kv(const wavepp_plan* plan, const void* k_new, const void* v_new, void* k_pool, void* v_pool,
                        void* workspace, size_t ws_bytes, hipStream_t stream) {
  bool run;
  int st = check_call(plan, workspace, ws_bytes, check_moves, &run);
  if (st || !run) return st;
  st = check_buffers(k_new, v_new, k_pool, v_pool);
  if (st) return st;
  const hipError_t e = launch_q8_append(make_dev(plan, workspace), make_q8(plan, workspace), k_new, v_new, k_pool, v_pool, stream);
  return e == hipSuccess ? WAVEPP_OK : set_hip_error(e, "q8_append_kv launch");
}

int wavepp_q8_read_kv(const wavepp_plan* plan, const void* k_pool, const void* v_pool, void* k_out, void* v_out,
                      void* workspace, size_t ws_bytes, hipStream_t stream) {
  bool run;
  int st = check_call(plan, workspace, ws_bytes, check_moves, &run);
  if (st || !run) return st;
  st = check_buffers(k_pool, v_pool, k_out, v_out);
  if (st) return st;
  const hipError_t e = launch_q8_read(make_dev(plan, workspace), make_q8(plan, workspace), k_pool, v_pool, k_out, v_out, stream);
  return e == hipSuccess ? WAVEPP_OK : set_hip_error(e, "q8_read_kv launch");
}

int wavepp_q8_chunked_prefill(const wavepp_plan* plan, const void* q, const void* k_pool, const void* v_pool, void* out,
                              float* lse, void* workspace, size_t ws_bytes, hipStream_t stream) {
  bool run;
  int st = check_call(plan, workspace, ws_bytes, check_items, &run);
  if (st || !run) return st;
  st = check_buffers(q, k_pool, v_pool, out);
  if (st) return st;
  if (reinterpret_cast<uintptr_t>(lse) & 3) return set_error(WAVEPP_EINVAL, "lse must be 4-byte aligned");
  const DevPlan d = make_dev(plan, workspace);
  hipError_t e = launch_q8_attention(d, make_q8(plan, workspace), plan->num_few, q, k_pool, v_pool, out, lse, stream);
  if (e != hipSuccess) return set_hip_error(e, "q8 attention launch");
  if (!plan->merges.empty()) {
    e = launch_merge(d, out, lse, stream);
    if (e != hipSuccess) return set_hip_error(e, "merge launch");
  }
  return WAVEPP_OK;
}

}  // extern "C"
