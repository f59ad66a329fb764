// Layout shared by the host code (rope_host.cpp) and the kernels (rope.hip) of rotary positions.  Not part of the public
// ABI.
#pragma once

#include "internal.h"

namespace wavepp {

constexpr int kRopeMaxPairs = 128;
constexpr int64_t kRopeMaxTokens = (int64_t(1) << 24) - 1;      // a launch has less than 2^32 threads, 256 for a token

// A launch's arguments beside the DevPlan.
struct RopeDev {
  int32_t pairs, offset, interleaved;
  float magnitude;
  const int32_t* positions;          // NULL: the plan's
  const void *q, *k;                 // NULL: none
  void *q_out, *k_out;
  int64_t q_stride, k_stride, q_out_stride, k_out_stride;
};

// turns: of every pair, for one token.
hipError_t launch_rope(const DevPlan& p, const RopeDev& x, const double* turns, hipStream_t stream);

}  // namespace wavepp
