// Layout shared by the host code (host.cpp, q4_host.cpp) and the kernels (q4.hip) of the 4-bit paged cache.  Not part of the
// public ABI.
#pragma once

#include "internal.h"

namespace wavepp {

constexpr int kQ4FewRows = 32;             // 4-bit pages, few rows: query rows per work item (every wave has them all)
constexpr int kQ4FewTile = 128;            // 4-bit pages, few rows: keys per step of a workgroup, 32 a wave
constexpr int kQ4Block = 32;               // values along the head dim that share a scale

// The append and the attention of internal.h over 4-bit pages, and the way back from them to bf16 rows.
hipError_t launch_q4_append(const DevPlan& p, const void* k_new, const void* v_new, void* k_pool, void* v_pool,
                            hipStream_t stream);
hipError_t launch_q4_read(const DevPlan& p, const void* k_pool, const void* v_pool, void* k_out, void* v_out,
                          hipStream_t stream);
hipError_t launch_q4_attention(const DevPlan& p, int32_t num_few, const void* q, const void* k_pool, const void* v_pool,
                               void* out, float* lse, hipStream_t stream);   // num_few: see wavepp_plan

}  // namespace wavepp
