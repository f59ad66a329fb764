// Host side of linear attention with a decay for each head: validation of the wave, the work list and the launch.
//
// Resume semantics and the rules for slots are those of the KDA layers (kda_host.cpp): a wave's workgroups run
// concurrently, so a slot that one request writes may be neither read nor written by another.
#include "wavepp_lin.h"
#include "lin.h"

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstring>
#include <functional>
#include <memory>
#include <new>
#include <numeric>
#include <vector>

using namespace wavepp;

struct wavepp_lin_plan_s {
  wavepp_lin_shape shape;
  int64_t total_tokens = 0;
  uint32_t serial = 0;
  std::vector<LinItem> steps, segments;
  std::vector<LinScan> scans;
  int32_t num_parts = 0, num_ahead = 0;     // partial states, and segments whose own state is computed ahead
  std::vector<unsigned char> blob;
  size_t off_steps = 0, off_segments = 0, off_scans = 0, off_parts = 0, off_decay = 0;
  size_t workspace_bytes = 0;
};

namespace {

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
// Constants of the model below, in blocks of the main kernel (about 3.5 us): what a workgroup takes besides its blocks in
// either kernel, a block of the kernel that runs ahead, the scan's launch and one of its states of 128 x 128, and the
// memory's time for a block of 128 + 128 columns.  Measured over forced cuts of seven waves (us, forced best / chosen):
// 32 heads of 128 x 64, one by one, 4,627 + 4,948 + 6,968 tokens: 390 whole, 128 / 128; 64 of 128 x 128, 16,384 tokens: 912
// whole, 380 / 380; 16 of 64 x 64, 2 x 8,000: 329 whole, 55 / 55; 8 of 128 x 128, 16,384: 798 whole, 70 / 70.
// All with a head a workgroup: the two heads of a paired workgroup are modelled as two chains on a slot each, which was not
// measured over forced cuts, and three workgroups of 64 x 64 heads fit on a CU where the model has two.
constexpr double kMainOverhead = 3.0, kAheadOverhead = 2.0, kAheadBlock = 0.5, kScanBase = 1.5, kScanBlock = 0.01;
constexpr double kMemoryBlock = 0.0046;

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

int check_ws(const wavepp_lin_plan_t* plan, void* ws, size_t ws_bytes) {
  if (!ws) return set_error(WAVEPP_EINVAL, "workspace is NULL");
  if (reinterpret_cast<uintptr_t>(ws) % 256) return set_error(WAVEPP_EINVAL, "workspace must be 256-byte aligned");
  if (ws_bytes < plan->workspace_bytes)
    return set_error(WAVEPP_ENOSPACE, "workspace has %zu bytes, plan needs %zu", ws_bytes, plan->workspace_bytes);
  return WAVEPP_OK;
}

// How a chunk of n blocks is cut into at most `pieces` segments of equal length, the last shorter: blocks of one, their number.
struct Cut {
  int64_t each, count;
  Cut(int64_t n, int64_t pieces) : each(ceil_div(n, std::max<int64_t>(1, std::min(n, pieces)))), count(ceil_div(n, each)) {}
};

// Workgroups of the main kernel that run at once, in the model of the time.
int64_t main_slots(const wavepp_lin_shape& s) { return kNumCu * (s.head_dim_v == 64 ? 2 : 1); }

// The time at which the last of `runs` (length, how many) ends, longest first on `slots` workgroups that run one
// after another; every one takes `overhead` besides its length.  Runs of one length end in the order in which they are given
// out, so the next slot to be free is the first of two ascending lists: those before the length, and those of it.
double makespan(std::vector<std::pair<int64_t, int64_t>> runs, int64_t slots, double overhead) {
  std::sort(runs.rbegin(), runs.rend());
  std::vector<double> busy(size_t(slots), 0.0), ends, next;
  double longest = 0.0;
  for (size_t i = 0; i < runs.size();) {
    const int64_t length = runs[i].first;
    int64_t n = 0;
    for (; i < runs.size() && runs[i].first == length; ++i) n += runs[i].second;
    ends.resize(size_t(n));
    const double each = double(length) + overhead;
    size_t a = 0, b = 0;
    for (size_t k = 0; k < size_t(n); ++k) {
      const bool old = a < busy.size() && (b == k || busy[a] <= ends[b]);
      ends[k] = (old ? busy[a++] : ends[b++]) + each;
    }
    if (n) longest = std::max(longest, ends.back());
    next.resize(busy.size());
    std::merge(busy.begin() + a, busy.end(), ends.begin() + b, ends.end(), next.begin());
    busy.swap(next);
  }
  return longest;
}

// Modelled time, in blocks of the main kernel, of chunks of `blocks` (one for each of `heads` chains), cut so that
// no segment is longer than `most`; some number no less than `best` where it cannot beat that.
double cut_cost(const wavepp_lin_shape& s, const std::vector<int64_t>& blocks, int64_t most, double best) {
  const int64_t slots = main_slots(s), H = s.num_heads;
  // what memory takes for a block: rows of q, k, v and out in the main kernel, of k and v in the one that runs ahead; heads
  // that share q and k read them from one L2
  const double traffic = kMemoryBlock * (double(s.head_dim_k) * s.num_qk_heads / s.num_heads + s.head_dim_v) / 256.0;
  std::vector<std::pair<int64_t, int64_t>> all, ahead;
  int64_t parts = 0, total = 0, early = 0, count = 0;
  for (int64_t n : blocks) {
    const Cut c(n, ceil_div(n, most));
    total += n * H;
    count += c.count * H;
    all.push_back({n - c.each * (c.count - 1), H});
    if (c.count == 1) continue;
    all.push_back({c.each, (c.count - 1) * H});
    ahead.push_back({c.each, (c.count - 1) * H});
    early += c.each * (c.count - 1) * H;
    parts += c.count - 1;
  }
  const double scan = parts ? kScanBase + kScanBlock * double(parts) * H * (s.head_dim_k * s.head_dim_v / 16384.0) : 0.0;
  const double bound = std::max((double(total) + kMainOverhead * double(count)) / double(slots), traffic * double(total)) + scan;
  if (bound >= best) return bound;
  double t = scan + std::max(makespan(std::move(all), slots, kMainOverhead), traffic * double(total));
  if (parts)
    t += std::max(kAheadBlock * makespan(std::move(ahead), 2 * kNumCu, kAheadOverhead), 0.5 * traffic * double(early));
  return t;
}

// The longest segment, in blocks: a chunk whole where the chains are many and have work for two rounds of the longest, so
// that it ends among the others; else what cut_cost likes best.  64 heads of 128 x 128, 16,384 tokens beside 15 chunks of
// 64: 880 us whole, 447 cut, and beside 40 895 and 512; 32/8 of 128 x 64, 9,000 beside 31: 508 and 96.  Of 44 drawn waves of
// 1,024 chains and more that are cut for their longest chunk none got slower, the median 1.8 times as fast.
int64_t segment_blocks(const wavepp_lin_shape& s, const std::vector<int64_t>& blocks) {
  const int64_t longest = *std::max_element(blocks.begin(), blocks.end());
  const int64_t chains = int64_t(blocks.size()) * s.num_heads;
  const int64_t work = std::accumulate(blocks.begin(), blocks.end(), int64_t(0)) * s.num_heads;
  if (chains >= 4 * kNumCu && work >= 2 * longest * main_slots(s)) return longest;
  int64_t best = longest;
  double least = cut_cost(s, blocks, longest, INFINITY);
  for (int64_t pieces = 2, last = longest; pieces <= 2 * kNumCu && last > 2; ++pieces) {
    const int64_t most = ceil_div(longest, pieces);
    if (most == last) continue;
    last = most;
    int64_t count = 0;
    for (int64_t n : blocks) count += Cut(n, ceil_div(n, most)).count;
    if (count * s.num_heads > std::max<int64_t>(8 * kNumCu, chains + 4 * kNumCu)) break;   // rounds enough for any unevenness
    const double t = cut_cost(s, blocks, most, least);
    if (t < least) least = t, best = most;
  }
  return best;
}

int make_plan(const wavepp_lin_shape* shape, const wavepp_lin_batch* batch, wavepp_lin_plan_t** out) {
  clear_error();
  if (!shape || !batch || !out) return set_error(WAVEPP_EINVAL, "null argument");
  *out = nullptr;
  const wavepp_lin_shape s = *shape;
  if (s.num_heads <= 0 || s.num_qk_heads <= 0 || s.head_dim_k <= 0 || s.head_dim_v <= 0 || s.num_state_slots < 0)
    return set_error(WAVEPP_EINVAL, "non-positive shape field");
  if (s.num_heads % s.num_qk_heads)
    return set_error(WAVEPP_EINVAL, "num_heads (%d) is not a multiple of num_qk_heads (%d)", s.num_heads, s.num_qk_heads);
  if (s.alpha_per_token != 0 && s.alpha_per_token != 1) return set_error(WAVEPP_EINVAL, "alpha_per_token must be 0 or 1");
  if (!std::isfinite(s.scale)) return set_error(WAVEPP_EINVAL, "scale must be finite");
  if ((s.head_dim_k != 64 && s.head_dim_k != 128) || (s.head_dim_v != 64 && s.head_dim_v != 128))
    return set_error(WAVEPP_EUNSUPPORTED, "unsupported head dims (d_k=%d, d_v=%d): each 64 or 128", s.head_dim_k, s.head_dim_v);
  if (s.num_heads > 65535) return set_error(WAVEPP_EINVAL, "too many heads");   // a block of rows stays within 32-bit offsets
  const int32_t R = batch->num_requests;
  if (R < 0) return set_error(WAVEPP_EINVAL, "num_requests < 0");
  if (R > 0 && (!batch->chunk_lens || !batch->state_in || !batch->state_out))
    return set_error(WAVEPP_EINVAL, "null chunk_lens / state_in / state_out");

  int64_t total = 0;
  std::vector<int32_t> writer(size_t(s.num_state_slots), -1);
  for (int32_t r = 0; r < R; ++r) {
    const int32_t c = batch->chunk_lens[r];
    if (c < 0) return set_error(WAVEPP_EINVAL, "request %d: negative chunk length %d", r, c);
    total += c;
    if (total > INT32_MAX / 2) return set_error(WAVEPP_EINVAL, "too many tokens in the wave");
    if (c == 0) continue;
    const int32_t si = batch->state_in[r], so = batch->state_out[r];
    if (si < -1 || si >= s.num_state_slots)
      return set_error(WAVEPP_ERANGE, "request %d: state_in %d outside [-1, %d)", r, si, s.num_state_slots);
    if (so < 0 || so >= s.num_state_slots)
      return set_error(WAVEPP_ERANGE, "request %d: state_out %d outside [0, %d)", r, so, s.num_state_slots);
    if (writer[so] >= 0)
      return set_error(WAVEPP_EALIAS, "requests %d and %d both write snapshot slot %d", writer[so], r, so);
    writer[so] = r;
  }
  for (int32_t r = 0; r < R; ++r) {
    if (batch->chunk_lens[r] == 0) continue;
    const int32_t si = batch->state_in[r];
    if (si >= 0 && writer[si] >= 0 && writer[si] != r)
      return set_error(WAVEPP_EALIAS, "request %d resumes from slot %d, which request %d writes", r, si, writer[si]);
  }

  std::unique_ptr<wavepp_lin_plan_t> plan(new (std::nothrow) wavepp_lin_plan_t());
  if (!plan) return set_error(WAVEPP_EINVAL, "out of host memory");
  plan->shape = s;
  plan->total_tokens = total;
  plan->serial = next_serial();
  std::vector<int64_t> blocks;
  for (int32_t r = 0; r < R; ++r)
    if (batch->chunk_lens[r] > kLinStepTokens) blocks.push_back(ceil_div(batch->chunk_lens[r], kLinBlock));
  const int64_t per = blocks.empty() ? 1 : segment_blocks(s, blocks);
  std::vector<LinItem> last;            // segments without a partial state of their own
  int64_t cu = 0, parts = 0;
  for (int32_t r = 0; r < R; ++r) {
    const int64_t c = batch->chunk_lens[r];
    LinItem it{};
    it.cu = int32_t(cu);
    it.len = int32_t(c);
    it.state_in = batch->state_in ? batch->state_in[r] : -1;
    it.state_out = batch->state_out ? batch->state_out[r] : -1;
    it.part_in = it.part_out = -1;
    cu += c;
    if (c == 0) continue;
    if (c <= kLinStepTokens) {
      plan->steps.push_back(it);
      continue;
    }
    const int64_t n = ceil_div(c, kLinBlock);
    const Cut cut(n, ceil_div(n, per));
    const int64_t each = cut.each, count = cut.count;
    // the last segment may end before the first has read its start, so a slot that is resumed in place is copied first
    const bool copied = count > 1 && it.state_in >= 0 && it.state_in == it.state_out;
    const int32_t start = copied ? int32_t(parts + count - 1) : -1;
    if (count > 1) plan->scans.push_back(LinScan{it.state_in, int32_t(parts), int32_t(count - 1), start});
    for (int64_t g = 0; g < count; ++g) {
      LinItem x = it;
      x.cu = int32_t(it.cu + g * each * kLinBlock);
      x.len = int32_t(std::min(c - g * each * kLinBlock, each * kLinBlock));
      if (g > 0 || copied) {
        x.state_in = -1;
        x.part_in = g > 0 ? int32_t(parts + g - 1) : start;
      }
      if (g + 1 < count) {
        x.state_out = -1;
        x.part_out = int32_t(parts + g);
        plan->segments.push_back(x);
      } else {
        last.push_back(x);
      }
    }
    parts += count - 1 + copied;
    if (parts > INT32_MAX / 4) return set_error(WAVEPP_EINVAL, "wave too large");
  }
  plan->num_parts = int32_t(parts);
  plan->num_ahead = int32_t(plan->segments.size());
  // longest first within each kind, so that the last workgroups to start are short
  const auto longer = [](const LinItem& a, const LinItem& b) { return a.len > b.len; };
  std::stable_sort(plan->segments.begin(), plan->segments.end(), longer);
  std::stable_sort(last.begin(), last.end(), longer);
  std::stable_sort(plan->steps.begin(), plan->steps.end(), longer);
  plan->segments.insert(plan->segments.end(), last.begin(), last.end());
  const int64_t most = std::max({int64_t(plan->segments.size()), int64_t(plan->steps.size())});
  if (most * s.num_heads >= 1 << 22) return set_error(WAVEPP_EINVAL, "too many workgroups");   // 2^32 threads a launch

  plan->off_steps = sizeof(LinHeader);
  plan->off_segments = plan->off_steps + sizeof(LinItem) * plan->steps.size();
  plan->off_scans = plan->off_segments + sizeof(LinItem) * plan->segments.size();
  plan->blob.assign(plan->off_scans + sizeof(LinScan) * plan->scans.size(), 0);
  LinHeader h{kLinMagic, plan->serial, int32_t(plan->steps.size()), int32_t(plan->segments.size())};
  memcpy(plan->blob.data(), &h, sizeof(h));
  auto put = [&](size_t off, const auto& v) {
    if (!v.empty()) memcpy(plan->blob.data() + off, v.data(), sizeof(v[0]) * v.size());
  };
  put(plan->off_steps, plan->steps);
  put(plan->off_segments, plan->segments);
  put(plan->off_scans, plan->scans);
  plan->off_parts = align_up(plan->blob.size(), 256);
  const size_t states = size_t(parts) * size_t(s.num_heads);
  plan->off_decay = plan->off_parts + align_up(states * size_t(s.head_dim_k) * size_t(s.head_dim_v) * sizeof(float), 256);
  plan->workspace_bytes = plan->off_decay + align_up(states * sizeof(float), 256);
  *out = plan.release();
  return WAVEPP_OK;
}

}  // namespace

extern "C" {

int wavepp_lin_plan(const wavepp_lin_shape* shape, const wavepp_lin_batch* batch, wavepp_lin_plan_t** out) {
  return guarded([&] { return make_plan(shape, batch, out); });
}

size_t wavepp_lin_workspace_bytes(const wavepp_lin_plan_t* plan) { return plan ? plan->workspace_bytes : 0; }

int wavepp_lin_get_info(const wavepp_lin_plan_t* plan, wavepp_lin_info* info) {
  if (!plan || !info) return set_error(WAVEPP_EINVAL, "null argument");
  info->total_tokens = plan->total_tokens;
  info->num_step_items = int32_t(plan->steps.size());
  info->num_segments = int32_t(plan->segments.size());
  info->num_partials = plan->num_parts;
  info->block_tokens = kLinBlock;
  info->metadata_bytes = int64_t(plan->blob.size());
  info->workspace_bytes = int64_t(plan->workspace_bytes);
  return WAVEPP_OK;
}

int wavepp_lin_upload(const wavepp_lin_plan_t* plan, void* workspace, size_t ws_bytes, hipStream_t stream) {
  clear_error();
  if (!plan) return set_error(WAVEPP_EINVAL, "plan is NULL");
  int st = check_ws(plan, workspace, ws_bytes);
  if (st) return st;
  return upload_plan(plan->blob.data(), plan->blob.size(), plan->serial, workspace, stream);
}

int wavepp_lin_chunked_prefill(const wavepp_lin_plan_t* plan, const void* q, const void* k, const void* v,
                               const float* alpha, float* state_pool, void* out, void* workspace, size_t ws_bytes,
                               hipStream_t stream) {
  clear_error();
  if (!plan) return set_error(WAVEPP_EINVAL, "plan is NULL");
  int st = check_ws(plan, workspace, ws_bytes);
  if (st) return st;
  if (plan->total_tokens == 0) return WAVEPP_OK;
  st = require_upload(workspace, plan->serial, "wavepp_lin_upload");
  if (st) return st;
  if (!q || !k || !v || !alpha || !state_pool || !out)
    return set_error(WAVEPP_EINVAL, "q / k / v / alpha / state_pool / out is NULL");
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(state_pool) || !aligned16(out) ||
      (reinterpret_cast<uintptr_t>(alpha) & 3))
    return set_error(WAVEPP_EINVAL, "device buffers must be 16-byte aligned (alpha 4-byte)");
  auto* base = static_cast<unsigned char*>(workspace);
  LinDevPlan d{};
  d.hdr = reinterpret_cast<const LinHeader*>(base);
  d.steps = reinterpret_cast<const LinItem*>(base + plan->off_steps);
  d.segments = reinterpret_cast<const LinItem*>(base + plan->off_segments);
  d.scans = reinterpret_cast<const LinScan*>(base + plan->off_scans);
  d.parts = reinterpret_cast<float*>(base + plan->off_parts);
  d.part_decay = reinterpret_cast<float*>(base + plan->off_decay);
  d.serial = plan->serial;
  d.num_steps = int32_t(plan->steps.size());
  d.num_segments = int32_t(plan->segments.size());
  d.num_ahead = plan->num_ahead;
  d.num_scans = int32_t(plan->scans.size());
  d.num_heads = plan->shape.num_heads;
  d.num_qk_heads = plan->shape.num_qk_heads;
  d.head_dim_k = plan->shape.head_dim_k;
  d.head_dim_v = plan->shape.head_dim_v;
  d.alpha_per_token = plan->shape.alpha_per_token;
  d.scale = plan->shape.scale;
  const hipError_t e = launch_lin(d, q, k, v, alpha, state_pool, out, stream);
  return e == hipSuccess ? WAVEPP_OK : set_hip_error(e, "linear attention launch");
}

void wavepp_lin_destroy(wavepp_lin_plan_t* plan) { delete plan; }

}  // extern "C"
