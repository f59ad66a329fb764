// gfx950 (CDNA4) kernels of libwavepp_attn's rotary positions.
//
// A pair (a, b) of a row becomes (a cos - b sin, a sin + b cos) of its token's position times its frequency.  Nothing is
// computed twice from the same values, so the work is to read and write every row once at the memory's rate; the angles of a
// token, in fp64 (a position of 2^20 leaves 3 of fp32's bits), are shared by all of its heads.
#include <hip/hip_runtime.h>

#include "device.h"
#include "rope.h"

#include <algorithm>

namespace wavepp {
namespace {

constexpr int kThreads = 256;

// A launch's frequencies, in turns a token: as many as the arguments need, which the host copies at every launch.
template <int MAX>
struct Turns {
  double of[MAX];
};

// The position of packed token t of its request, the last with cu <= t, which whole waves find 64 requests at a time: the search
// ends with the lane that has it.  It stays within the requests whatever it reads.
__device__ __forceinline__ int64_t position_of(const DevPlan& p, const RopeDev& x, int64_t t) {
  if (x.positions) return x.positions[t];
  const int lane = threadIdx.x & 63;
  int lo = 0, n = p.num_requests;                    // the request is one of n from lo on
  for (;;) {
    const int step = (n + 63) / 64, r = min(lo + lane * step, p.num_requests - 1);
    const int cu = p.reqs[r].cu, prefix = p.reqs[r].prefix;
    const int last = max(63 - __clzll((long long)__ballot(lane * step < n && cu <= t)), 0);      // lane 0's holds, in a plan
    if (step == 1) return int64_t(__builtin_amdgcn_readlane(prefix, last)) + (t - __builtin_amdgcn_readlane(cu, last));
    lo += last * step;
    n = min(step, n - last * step);
  }
}

// cos and sin, times the magnitude, of pair i at a position.
template <int MAX>
__device__ __forceinline__ float2 turn(const RopeDev& x, const Turns<MAX>& f, int64_t position, int i) {
  const double turns = double(position) * f.of[i];
  float s, c;
  sincospif(2.0f * float(turns - rint(turns)), &s, &c);
  return {c * x.magnitude, s * x.magnitude};
}

struct Head {
  const __bf16* in;
  __bf16* out;
};
// Head h of token t, q's first and then k's.
__device__ __forceinline__ Head head_of(const RopeDev& x, int64_t t, int h, int q_heads, int D) {
  if (h < q_heads)
    return {static_cast<const __bf16*>(x.q) + t * x.q_stride + int64_t(h) * D,
            static_cast<__bf16*>(x.q_out) + t * x.q_out_stride + int64_t(h) * D};
  h -= q_heads;
  return {static_cast<const __bf16*>(x.k) + t * x.k_stride + int64_t(h) * D,
          static_cast<__bf16*>(x.k_out) + t * x.k_out_stride + int64_t(h) * D};
}

// ---------------------------------------------------------------------------------------------
// A workgroup has one token and up to `heads` of its heads.  A thread has one unit of every head that it takes: a 16-byte
// piece of the pairs (two where they lie in halves), or a piece that stays, which is only moved where the output is another
// buffer.  All its rows are loaded before the angles are there.
// Bound by memory: 16,384 tokens of 72 heads of 128, a quarter of each turned, 113 us, 5.3 TB/s read and written, all of each 108;
// a large copy reaches 4.8.  64 tokens: 4.5 us, a launch and the search, the angles and the rows one after the other.  (Stores
// past the caches: 104 us, but the step after it, which reads these rows, loses 17.)
// ---------------------------------------------------------------------------------------------
constexpr int kUnroll = 4;

template <bool PAIRS, int MAX>
__global__ __launch_bounds__(kThreads, 8) void rope_kernel(DevPlan p, RopeDev x, Turns<MAX> f, int heads, int units, int turned) {
  __shared__ __attribute__((aligned(16))) float cs[2][MAX];
  const int64_t t = blockIdx.x;
  const int D = p.head_dim_qk, Hq = x.q ? p.num_q_heads : 0, H = Hq + (x.k ? p.num_kv_heads : 0);
  const int unit = threadIdx.x % units, step = kThreads / units;
  const int h0 = int(blockIdx.y) * heads + int(threadIdx.x) / units, h1 = min(H, int(blockIdx.y + 1) * heads);
  const bool turns = unit < turned;
  // the unit's first value, and where it has a second piece that one's
  int at, at2;
  if (turns) {
    at = x.offset + 8 * unit;
    at2 = PAIRS ? at : at + x.pairs;
  } else {
    at = 8 * (unit - turned);
    if (at >= x.offset) at += 2 * x.pairs;
    at2 = at;
  }
  u32x4 a[kUnroll], b[kUnroll];
  const bool mine = int(threadIdx.x) < step * units;
#pragma unroll
  for (int i = 0; i < kUnroll; ++i) {
    const int h = h0 + i * step;
    if (mine && h < h1) {
      const __bf16* in = head_of(x, t, h, Hq, D).in;
      a[i] = *reinterpret_cast<const u32x4*>(in + at);
      if (!PAIRS) b[i] = *reinterpret_cast<const u32x4*>(in + at2);
    }
  }
  const int64_t position = position_of(p, x, t);
  if (!meta_ok(p)) return;                       // after the loads, not before them
  for (int i = threadIdx.x; i < x.pairs; i += kThreads) {
    const float2 v = turn(x, f, position, i);
    cs[0][i] = v.x;
    cs[1][i] = v.y;
  }
  __syncthreads();
  constexpr int N = PAIRS ? 4 : 8;               // pairs of a unit
  float c[N], s[N];
  const int first = turns ? N * unit : 0;
#pragma unroll
  for (int k = 0; k < N; k += 4) {
    const f32x4 cv = *reinterpret_cast<const f32x4*>(&cs[0][first + k]), sv = *reinterpret_cast<const f32x4*>(&cs[1][first + k]);
#pragma unroll
    for (int j = 0; j < 4; ++j) c[k + j] = cv[j], s[k + j] = sv[j];
  }
#pragma unroll
  for (int i = 0; i < kUnroll; ++i) {
    const int h = h0 + i * step;
    if (!mine || h >= h1) continue;
    __bf16* out = head_of(x, t, h, Hq, D).out;
    if (!turns) {
      *reinterpret_cast<u32x4*>(out + at) = a[i];
      continue;
    }
    const bf16x8 u = __builtin_bit_cast(bf16x8, a[i]);
    if (PAIRS) {
      bf16x8 o;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float e = float(u[2 * k]), f = float(u[2 * k + 1]);
        o[2 * k] = static_cast<__bf16>(fmaf(e, c[k], -(f * s[k])));
        o[2 * k + 1] = static_cast<__bf16>(fmaf(e, s[k], f * c[k]));
      }
      *reinterpret_cast<bf16x8*>(out + at) = o;
    } else {
      const bf16x8 w = __builtin_bit_cast(bf16x8, b[i]);
      bf16x8 o, r;
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float e = float(u[k]), f = float(w[k]);
        o[k] = static_cast<__bf16>(fmaf(e, c[k], -(f * s[k])));
        r[k] = static_cast<__bf16>(fmaf(e, s[k], f * c[k]));
      }
      *reinterpret_cast<bf16x8*>(out + at) = o;
      *reinterpret_cast<bf16x8*>(out + at2) = r;
    }
  }
}

// Pairs that do not come in whole 16-byte pieces: value by value, a workgroup a token.  16,384 tokens of 72 heads of 128: 255 us
// with 126 values turned from the second on, 333 with 30, bound by the loads and stores of two bytes.
__global__ __launch_bounds__(kThreads) void rope_any_kernel(DevPlan p, RopeDev x, Turns<kRopeMaxPairs> f, int copy_q, int copy_k) {
  if (!meta_ok(p)) return;
  __shared__ float cs[2][kRopeMaxPairs];
  const int64_t t = blockIdx.x;
  const int D = p.head_dim_qk, Hq = x.q ? p.num_q_heads : 0, H = Hq + (x.k ? p.num_kv_heads : 0);
  const int64_t position = position_of(p, x, t);
  for (int i = threadIdx.x; i < x.pairs; i += kThreads) {
    const float2 v = turn(x, f, position, i);
    cs[0][i] = v.x;
    cs[1][i] = v.y;
  }
  __syncthreads();
  const int units = D - x.pairs;                 // pairs, then the values that stay
  for (int n = threadIdx.x; n < H * units; n += kThreads) {
    const int h = n / units, unit = n % units;
    const Head row = head_of(x, t, h, Hq, D);
    if (unit >= x.pairs) {
      int at = unit - x.pairs;
      if (at >= x.offset) at += 2 * x.pairs;
      if (h < Hq ? copy_q : copy_k) row.out[at] = row.in[at];
      continue;
    }
    const int a = x.offset + (x.interleaved ? 2 * unit : unit), b = a + (x.interleaved ? 1 : x.pairs);
    const float e = float(row.in[a]), f = float(row.in[b]), c = cs[0][unit], s = cs[1][unit];
    row.out[a] = static_cast<__bf16>(fmaf(e, c, -(f * s)));
    row.out[b] = static_cast<__bf16>(fmaf(e, s, f * c));
  }
}

}  // namespace

namespace {
template <int MAX>
Turns<MAX> turns_of(const double* turns, int pairs) {
  Turns<MAX> f{};
  std::copy(turns, turns + pairs, f.of);
  return f;
}
}  // namespace

hipError_t launch_rope(const DevPlan& p, const RopeDev& x, const double* turns, hipStream_t stream) {
  if (p.total_tokens > kRopeMaxTokens) return hipErrorInvalidValue;
  const int D = p.head_dim_qk, H = (x.q ? p.num_q_heads : 0) + (x.k ? p.num_kv_heads : 0);
  const int copy_q = x.q != x.q_out, copy_k = x.k != x.k_out;
  if (x.offset % 8 || (x.interleaved ? x.pairs % 4 : x.pairs % 8)) {
    hipLaunchKernelGGL(rope_any_kernel, dim3(unsigned(p.total_tokens)), dim3(kThreads), 0, stream, p, x,
                       turns_of<kRopeMaxPairs>(turns, x.pairs), copy_q, copy_k);
    return hipGetLastError();
  }
  const int turned = x.interleaved ? x.pairs / 4 : x.pairs / 8;
  const int units = turned + (copy_q || copy_k ? (D - 2 * x.pairs) / 8 : 0);
  // as few workgroups a token as the threads' kUnroll rows allow, with even shares
  const int most = kThreads / units * kUnroll, parts = (H + most - 1) / most, heads = (H + parts - 1) / parts;
  if (parts > 65535) return hipErrorInvalidValue;
  const dim3 grid(unsigned(p.total_tokens), unsigned(parts));
#define WAVEPP_ROPE(PAIRS_, MAX_)                                                                                      \
  hipLaunchKernelGGL((rope_kernel<PAIRS_, MAX_>), grid, dim3(kThreads), 0, stream, p, x, turns_of<MAX_>(turns, x.pairs), \
                     heads, units, turned)
  if (x.pairs <= 32) {
    if (x.interleaved) WAVEPP_ROPE(true, 32); else WAVEPP_ROPE(false, 32);
  } else if (x.pairs <= 64) {
    if (x.interleaved) WAVEPP_ROPE(true, 64); else WAVEPP_ROPE(false, 64);
  } else {
    if (x.interleaved) WAVEPP_ROPE(true, kRopeMaxPairs); else WAVEPP_ROPE(false, kRopeMaxPairs);
  }
#undef WAVEPP_ROPE
  return hipGetLastError();
}

}  // namespace wavepp
