// Layout shared by the host code (host.cpp, q8_host.cpp) and the kernels (q8.hip) of the 8-bit paged cache.  Not part of the
// public ABI.
#pragma once

#include "internal.h"

namespace wavepp {

constexpr int kQ8Block = 16;               // tokens of one head that share a scale
constexpr int kQ8ScaleBytes = 16;          // bytes of a page's scales: page_size / 16 of them, then padding

// Keys that a new token sees: [begin, end), none where begin >= end.
struct TokenRange {
  int32_t begin, end;
};

// A block of 16 slots that receives tokens of the wave.
struct alignas(16) Q8Block {
  int32_t page;      // page of the pool
  int32_t slot;      // the block's first slot in it
  int32_t token;     // packed token of the first new slot
  int32_t span;      // new slots of the block: from the low byte to before the next byte
};

// What a work item needs to know of its request, and the first key that one of its rows sees.  (The last that it loads is the
// one before its kv_end: kv_begin is a tile's first key, which its rows need not see.)
struct alignas(16) Q8ItemReq {
  int32_t prefix, cu, bt_row;        // as in ReqMeta
  int32_t first;
};

// What the 8-bit cache's launches need beyond a DevPlan.
struct Q8Dev {
  const Q8Block* blocks;
  const Q8ItemReq* item_reqs;  // of every work item
  int32_t num_blocks;
  int32_t few_rows;            // most rows of an item that runs with few rows
  bool stream;                 // such items read pages that hardly another reads
  const TokenRange* ranges;    // of every new token; NULL: causal
  const float* slopes;         // of every query head; NULL: none
  float cap;                   // 0: none
};

// A launch has less than 2^32 threads: so many workgroups at most of the append and the read, which have four waves for four
// blocks of one head, of K or of V; of attention of few rows, of four waves; and of attention of many, of eight at most.
constexpr int64_t kQ8MostMoves = (int64_t(1) << 24) - 1, kQ8MostFew = (int64_t(1) << 24) - 1, kQ8MostMany = (int64_t(1) << 23) - 1;
inline int64_t q8_moves(int32_t num_blocks, int32_t num_kv_heads) { return (int64_t(num_blocks) + 3) / 4 * 2 * num_kv_heads; }

hipError_t launch_q8_append(const DevPlan& p, const Q8Dev& x, const void* k_new, const void* v_new, void* k_pool,
                            void* v_pool, hipStream_t stream);
hipError_t launch_q8_read(const DevPlan& p, const Q8Dev& x, const void* k_pool, const void* v_pool, void* k_out, void* v_out,
                          hipStream_t stream);
hipError_t launch_q8_attention(const DevPlan& p, const Q8Dev& x, int32_t num_few, const void* q, const void* k_pool,
                               const void* v_pool, void* out, float* lse, hipStream_t stream);

}  // namespace wavepp
