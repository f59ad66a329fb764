// Host side of the 4-bit paged cache: its plans, checks of arguments and launches.
#include "wavepp_q4.h"
#include "internal.h"
#include "plan.h"
#include "q4.h"

using namespace wavepp;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

// What every call on a plan checks first.  *run: whether there is anything to enqueue.
int check_call(const wavepp_plan* plan, void* workspace, size_t ws_bytes, bool* run) {
  clear_error();
  *run = false;
  if (!plan) return set_error(WAVEPP_EINVAL, "plan is NULL");
  int st = require_cache(plan, true);
  if (!st) st = check_workspace(plan, workspace, ws_bytes);
  if (st || plan->total_tokens == 0) return st;
  *run = true;
  return require_upload(workspace, plan->serial, "wavepp_attn_plan_upload");
}

int check_buffers(const void* a, const void* b, const void* c, const void* d) {
  if (!a || !b || !c || !d) return set_error(WAVEPP_EINVAL, "a device buffer is NULL");
  if (!aligned16(a) || !aligned16(b) || !aligned16(c) || !aligned16(d))
    return set_error(WAVEPP_EINVAL, "device buffers must be 16-byte aligned");
  return WAVEPP_OK;
}

}  // namespace

extern "C" {

size_t wavepp_q4_page_bytes(int32_t head_dim, int32_t page_size) {
  if ((head_dim != 64 && head_dim != 128) || (page_size != 16 && page_size != 64)) return 0;
  return size_t(page_size) * (head_dim / 2 + head_dim / kQ4Block);
}

int wavepp_q4_plan(const wavepp_attn_shape* shape, const wavepp_batch* batch, int32_t max_splits, wavepp_plan** out) {
  return guarded([&] { return plan_wave(shape, batch, max_splits, true, out); });
}

int wavepp_q4_append_kv(const wavepp_plan* plan, const void* k_new, const void* v_new, void* k_pool, void* v_pool,
                        void* workspace, size_t ws_bytes, hipStream_t stream) {
  bool run;
  int st = check_call(plan, workspace, ws_bytes, &run);
  if (st || !run) return st;
  st = check_buffers(k_new, v_new, k_pool, v_pool);
  if (st) return st;
  const hipError_t e = launch_q4_append(make_dev(plan, workspace), k_new, v_new, k_pool, v_pool, stream);
  return e == hipSuccess ? WAVEPP_OK : set_hip_error(e, "q4_append_kv launch");
}

int wavepp_q4_read_kv(const wavepp_plan* plan, const void* k_pool, const void* v_pool, void* k_out, void* v_out,
                      void* workspace, size_t ws_bytes, hipStream_t stream) {
  bool run;
  int st = check_call(plan, workspace, ws_bytes, &run);
  if (st || !run) return st;
  st = check_buffers(k_pool, v_pool, k_out, v_out);
  if (st) return st;
  const hipError_t e = launch_q4_read(make_dev(plan, workspace), k_pool, v_pool, k_out, v_out, stream);
  return e == hipSuccess ? WAVEPP_OK : set_hip_error(e, "q4_read_kv launch");
}

int wavepp_q4_chunked_prefill(const wavepp_plan* plan, const void* q, const void* k_pool, const void* v_pool, void* out,
                              float* lse, void* workspace, size_t ws_bytes, hipStream_t stream) {
  bool run;
  int st = check_call(plan, workspace, ws_bytes, &run);
  if (st || !run) return st;
  st = check_buffers(q, k_pool, v_pool, out);
  if (st) return st;
  if (reinterpret_cast<uintptr_t>(lse) & 3) return set_error(WAVEPP_EINVAL, "lse must be 4-byte aligned");
  const DevPlan d = make_dev(plan, workspace);
  hipError_t e = launch_q4_attention(d, plan->num_few, q, k_pool, v_pool, out, lse, stream);
  if (e != hipSuccess) return set_hip_error(e, "q4 attention launch");
  if (!plan->merges.empty()) {
    e = launch_merge(d, out, lse, stream);
    if (e != hipSuccess) return set_hip_error(e, "merge launch");
  }
  return WAVEPP_OK;
}

}  // extern "C"
