// Layout shared by the host code (lin_host.cpp) and the kernels (lin.hip) of linear attention with a decay for each head.  Not
// part of the public ABI.
#pragma once

#include "internal.h"

namespace wavepp {

constexpr uint32_t kLinMagic = 0x4C494E31u;  // "LIN1"
constexpr int kLinBlock = 64;                // tokens per block of the chunkwise form
// Chunks up to this length run token by token: 64 requests of 64 heads of 128 x 128 take 128 us so and 154 in blocks at
// eight tokens, 159 and 156 at twelve, 197 and 158 at sixteen; 4 of 32 of 128 x 64: 7.1 and 9.0, 8.9 and 9.2, 11.1 and 9.1.
constexpr int kLinStepTokens = 10;

// Heads of one workgroup of the blocks: two of 64 columns where they share q and k, whose products they then share too.
constexpr int lin_heads(int num_heads, int num_qk_heads, int head_dim_v) {
  return head_dim_v == 64 && num_heads / num_qk_heads % 2 == 0 ? 2 : 1;
}

struct alignas(16) LinHeader {
  uint32_t magic;
  uint32_t serial;
  int32_t num_steps;
  int32_t num_segments;
};

// A run of tokens of one request: a whole short chunk (token by token), or a segment of a longer one (whole blocks but
// for the request's last).  States are snapshot slots, or partial states of the workspace between segments.
struct alignas(16) LinItem {
  int32_t cu;         // first packed token
  int32_t len;        // > 0
  int32_t state_in;   // snapshot slot to start from, -1 = zero state (with part_in < 0)
  int32_t state_out;  // snapshot slot written at the end, -1 = none
  int32_t part_in;    // >= 0: start from this partial state instead
  int32_t part_out;   // >= 0: where this segment's own state goes
  int32_t pad[2];
};

// The partial states of one request's segments, in order.
struct alignas(16) LinScan {
  int32_t state_in;   // the first segment's start
  int32_t first_part;
  int32_t count;
  int32_t start_part; // >= 0: the start is copied here, for the first segment of a request whose last writes the same slot
};

struct LinDevPlan {
  const LinHeader* hdr;
  const LinItem* steps;
  const LinItem* segments;   // those with part_out >= 0 first
  const LinScan* scans;
  float* parts;              // [partial states][num_heads][head_dim_k][head_dim_v]
  float* part_decay;         // [partial states][num_heads]
  uint32_t serial;
  int32_t num_steps, num_segments, num_ahead, num_scans;
  int32_t num_heads, num_qk_heads, head_dim_k, head_dim_v, alpha_per_token;
  float scale;
};

hipError_t launch_lin(const LinDevPlan& p, const void* q, const void* k, const void* v, const float* alpha,
                      float* state_pool, void* out, hipStream_t stream);

// The metadata upload copies 16-byte words.
static_assert(sizeof(LinHeader) % 16 == 0 && sizeof(LinItem) % 16 == 0 && sizeof(LinScan) % 16 == 0,
              "metadata records are whole 16-byte words");

}  // namespace wavepp
