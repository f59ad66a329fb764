// Host side of rotary positions: the frequencies, checks of arguments and the launch.
#include "wavepp_rope.h"
#include "internal.h"
#include "plan.h"
#include "rope.h"

#include <algorithm>
#include <cmath>
#include <memory>
#include <new>

using namespace wavepp;

struct wavepp_rope {
  int32_t pairs = 0, offset = 0, interleaved = 0;
  float magnitude = 1.0f;
  double frequencies[kRopeMaxPairs] = {}, turns[kRopeMaxPairs] = {};
  void take_turns();
};

namespace {

constexpr double kTurn = 6.283185307179586476925286766559;

int64_t floor_div(int64_t a, int64_t b) { return a / b - (a % b < 0); }

// Whether one of T rows of `w` bytes at b, b + s, ... has a byte of [lo, hi): row j does where j s lies in (lo - b - w, hi - b).
bool row_meets(int64_t lo, int64_t hi, uintptr_t b, int64_t s, int64_t w, int64_t T) {
  const int64_t first = floor_div(lo - int64_t(b) - w, s) + 1, last = floor_div(hi - int64_t(b) - 1, s);
  return std::max<int64_t>(first, 0) <= std::min<int64_t>(last, T - 1);
}

// Whether two sets of T rows share a byte: rows of `wa` bytes at a, a + sa, ..., and of `wb` at b, b + sb, ...
bool rows_meet(uintptr_t a, int64_t sa, int64_t wa, uintptr_t b, int64_t sb, int64_t wb, int64_t T) {
  const int64_t d = int64_t(b) - int64_t(a);
  if (d >= (T - 1) * sa + wa || -d >= (T - 1) * sb + wb) return false;        // one ends before the other
  if (sa != sb) {                                                             // row by row: rare, as both lie in each other's gaps
    for (int64_t i = 0; i < T; ++i)
      if (row_meets(int64_t(a) + i * sa, int64_t(a) + i * sa + wa, b, sb, wb, T)) return true;
    return false;
  }
  // row j of b lies d + (j - i) s from row i of a: whether that is in (-wb, wa) for a difference below T
  const int64_t near = -d / sa;
  for (int64_t k = near - 1; k <= near + 1; ++k)
    if (k > -T && k < T && d + k * sa > -wb && d + k * sa < wa) return true;
  return false;
}

struct Rows {
  const char* name;
  uintptr_t at;
  int64_t stride, width;             // bytes
};

// The most elements from one token to the next: a call's 2^24 tokens of them in bytes lie well within 63 bits.
constexpr int64_t kMostStride = int64_t(1) << 30;

bool positive(double x) { return x > 0.0 && std::isfinite(x); }

// The largest frequency: at any position of 32 bits its angle is under 2^128 turns, and what fp64 leaves of one after whole
// turns are taken off, rounded or not before that, is under 2^76: a number of fp32, whose cosine is one too.
constexpr double kMostFrequency = 1e30;
int check_frequency(int32_t i, double f) {
  return std::fabs(f) <= kMostFrequency ? WAVEPP_OK : set_error(WAVEPP_EINVAL, "frequency %d must be a number within [-1e30, 1e30]", i);
}

}  // namespace

void wavepp_rope::take_turns() {
  for (int32_t i = 0; i < pairs; ++i) turns[i] = frequencies[i] / kTurn;
}

extern "C" {

int wavepp_rope_create(const wavepp_rope_spec* spec, wavepp_rope** out) {
  clear_error();
  if (!spec || !out) return set_error(WAVEPP_EINVAL, "null argument");
  *out = nullptr;
  const wavepp_rope_spec& s = *spec;
  if (s.rot_dim < 2 || s.rot_dim % 2) return set_error(WAVEPP_EINVAL, "rot_dim must be even and positive");
  if (s.rot_dim > 2 * kRopeMaxPairs) return set_error(WAVEPP_EUNSUPPORTED, "rot_dim is over %d", 2 * kRopeMaxPairs);
  if (s.rot_offset < 0) return set_error(WAVEPP_EINVAL, "rot_offset is negative");
  if (s.interleaved != 0 && s.interleaved != 1) return set_error(WAVEPP_EINVAL, "interleaved must be 0 or 1");
  if (!positive(s.magnitude) || !std::isfinite(float(s.magnitude)) || float(s.magnitude) == 0.0f)
    return set_error(WAVEPP_EINVAL, "magnitude must be positive and finite");
  std::unique_ptr<wavepp_rope> rope(new (std::nothrow) wavepp_rope());
  if (!rope) return set_error(WAVEPP_EINVAL, "out of host memory");
  rope->pairs = s.rot_dim / 2;
  rope->offset = s.rot_offset;
  rope->interleaved = s.interleaved;
  rope->magnitude = float(s.magnitude);
  if (s.frequencies) {
    for (int32_t i = 0; i < rope->pairs; ++i) {
      if (int st = check_frequency(i, s.frequencies[i])) return st;
      rope->frequencies[i] = s.frequencies[i];
    }
    rope->take_turns();
    *out = rope.release();
    return WAVEPP_OK;
  }
  if (!(s.base > 1.0) || !std::isfinite(s.base)) return set_error(WAVEPP_EINVAL, "base must be over 1 and finite");
  if (s.scaling < WAVEPP_ROPE_PLAIN || s.scaling > WAVEPP_ROPE_INDEX) return set_error(WAVEPP_EINVAL, "no such scaling: %d", s.scaling);
  if (s.scaling != WAVEPP_ROPE_PLAIN && !positive(s.factor)) return set_error(WAVEPP_EINVAL, "factor must be positive and finite");
  const bool ramp = s.scaling == WAVEPP_ROPE_TURNS || s.scaling == WAVEPP_ROPE_INDEX;
  if (ramp && (!positive(s.original_length) || !positive(s.slow_turns) || !positive(s.fast_turns) || s.slow_turns >= s.fast_turns))
    return set_error(WAVEPP_EINVAL, "original_length and 0 < slow_turns < fast_turns must be positive and finite");
  double lo = 0.0, hi = 0.0;
  if (s.scaling == WAVEPP_ROPE_INDEX) {
    auto at = [&](double turns) { return s.rot_dim * std::log(s.original_length / (kTurn * turns)) / (2.0 * std::log(s.base)); };
    lo = std::max(0.0, std::floor(at(s.fast_turns)));
    hi = std::min(double(s.rot_dim - 1), std::ceil(at(s.slow_turns)));
  }
  for (int32_t i = 0; i < rope->pairs; ++i) {
    const double f = std::pow(s.base, -2.0 * i / s.rot_dim);
    double w = 1.0;                                    // how much of the pair keeps its frequency
    if (s.scaling == WAVEPP_ROPE_LINEAR)
      w = 0.0;
    else if (s.scaling == WAVEPP_ROPE_TURNS)
      w = (s.original_length * f / kTurn - s.slow_turns) / (s.fast_turns - s.slow_turns);
    else if (s.scaling == WAVEPP_ROPE_INDEX)
      w = 1.0 - (i - lo) / std::max(hi - lo, 1e-3);
    w = std::min(1.0, std::max(0.0, w));
    rope->frequencies[i] = w == 1.0 ? f : w * f + (1.0 - w) * f / s.factor;
    if (int st = check_frequency(i, rope->frequencies[i])) return st;
  }
  rope->take_turns();
  *out = rope.release();
  return WAVEPP_OK;
}

int wavepp_rope_frequencies(const wavepp_rope* rope, double* out, int32_t capacity) {
  clear_error();
  if (!rope || capacity < 0 || (!out && capacity > 0)) return set_error(WAVEPP_EINVAL, "bad argument");
  const int32_t n = std::min(capacity, rope->pairs);
  std::copy(rope->frequencies, rope->frequencies + n, out);
  return n;
}

int wavepp_rope_apply(const wavepp_rope* rope, const wavepp_plan* plan, const void* q, int64_t q_stride, const void* k,
                      int64_t k_stride, void* q_out, int64_t q_out_stride, void* k_out, int64_t k_out_stride,
                      const int32_t* positions, void* workspace, size_t ws_bytes, hipStream_t stream) {
  clear_error();
  if (!rope) return set_error(WAVEPP_EINVAL, "rope is NULL");
  if (!plan) return set_error(WAVEPP_EINVAL, "plan is NULL");
  int st = check_workspace(plan, workspace, ws_bytes);
  if (st) return st;
  const int64_t D = plan->shape.head_dim_qk, T = plan->total_tokens;
  if (rope->offset > D - 2 * rope->pairs)
    return set_error(WAVEPP_EINVAL, "the turned values [%d, %d) exceed the plan's head dim %d", rope->offset,
                     rope->offset + 2 * rope->pairs, int(D));
  if (T == 0) return WAVEPP_OK;
  if (T > kRopeMaxTokens)
    return set_error(WAVEPP_EUNSUPPORTED, "the wave has %lld tokens, a call turns %lld at most: plan it in parts", (long long)T,
                     (long long)kRopeMaxTokens);
  if (!q != !q_out || !k != !k_out || (!q && !k))
    return set_error(WAVEPP_EINVAL, "q and q_out, and k and k_out, come together, and one of the pairs is needed");
  const int64_t qw = plan->shape.num_q_heads * D, kw = plan->shape.num_kv_heads * D;
  Rows rows[4];                       // inputs, then outputs
  int n = 0;
  for (const auto& r : {Rows{"q", reinterpret_cast<uintptr_t>(q), q_stride, qw}, Rows{"k", reinterpret_cast<uintptr_t>(k), k_stride, kw},
                        Rows{"q_out", reinterpret_cast<uintptr_t>(q_out), q_out_stride, qw},
                        Rows{"k_out", reinterpret_cast<uintptr_t>(k_out), k_out_stride, kw}}) {
    if (!r.at) continue;
    if (r.at % 16) return set_error(WAVEPP_EINVAL, "%s must be 16-byte aligned", r.name);
    if (r.stride < r.width || r.stride % 8 || r.stride > kMostStride)
      return set_error(WAVEPP_EINVAL, "%s has a stride of %lld elements: a multiple of 8 from %lld to 2^30 is needed", r.name,
                       (long long)r.stride, (long long)r.width);
    rows[n++] = {r.name, r.at, 2 * r.stride, 2 * r.width};
  }
  if (reinterpret_cast<uintptr_t>(positions) & 3) return set_error(WAVEPP_EINVAL, "positions must be 4-byte aligned");
  for (int o = n / 2; o < n; ++o)
    for (int i = 0; i < n; ++i) {
      if (i == o) continue;
      const bool own = i == o - n / 2;
      if (own && rows[i].at == rows[o].at && (rows[i].stride == rows[o].stride || T == 1)) continue;       // in place
      if (rows_meet(rows[i].at, rows[i].stride, rows[i].width, rows[o].at, rows[o].stride, rows[o].width, T))
        return set_error(WAVEPP_EALIAS, "%s and %s overlap", rows[o].name, rows[i].name);
    }
  if (positions && T > 0)
    for (int o = n / 2; o < n; ++o)
      if (rows_meet(reinterpret_cast<uintptr_t>(positions), 4, 4, rows[o].at, rows[o].stride, rows[o].width, T))
        return set_error(WAVEPP_EALIAS, "%s and positions overlap", rows[o].name);
  const int64_t held = int64_t(reinterpret_cast<uintptr_t>(workspace));
  for (int o = n / 2; o < n; ++o)
    if (row_meets(held, held + int64_t(plan->meta_bytes), rows[o].at, rows[o].stride, rows[o].width, T))
      return set_error(WAVEPP_EALIAS, "%s and the plan in the workspace overlap", rows[o].name);
  st = require_upload(workspace, plan->serial, "wavepp_attn_plan_upload");
  if (st) return st;
  RopeDev x{};
  x.pairs = rope->pairs;
  x.offset = rope->offset;
  x.interleaved = rope->interleaved;
  x.magnitude = rope->magnitude;
  x.positions = positions;
  x.q = q;
  x.k = k;
  x.q_out = q_out;
  x.k_out = k_out;
  x.q_stride = q_stride;
  x.k_stride = k_stride;
  x.q_out_stride = q_out_stride;
  x.k_out_stride = k_out_stride;
  const hipError_t e = launch_rope(make_dev(plan, workspace), x, rope->turns, stream);
  return e == hipSuccess ? WAVEPP_OK : set_hip_error(e, "rope launch");
}

void wavepp_rope_destroy(wavepp_rope* rope) { delete rope; }

}  // extern "C"
