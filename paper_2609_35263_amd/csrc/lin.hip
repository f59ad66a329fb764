// gfx950 (CDNA4) kernels of libwavepp_attn: linear attention with a decay for each head,
//   S_t = alpha_t S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t,
// token by token for short chunks and in blocks of 64 tokens for longer ones.
//
// Blocks.  With S0 the state before a block, lam_i = alpha_1 ... alpha_i and D[i][j] = alpha_{j+1} ... alpha_i (j <= i, 0 above
// the diagonal), its outputs and its last state are
//   O = scale (diag(lam) Q S0 + ((Q K^T) * D) V),      S = lam_64 S0 + K^T diag(D[64][.]) V.
// All factors are products of decays, never quotients, so a decay of zero (or a tiny one) needs no special case.
//
// A workgroup runs one segment of one (request, head), block after block; wave w of its d_v / 32 owns the state's
// columns 32 w .. 32 w + 31 as 32 x 32 fp32 accumulator tiles.  The accumulator layout of v_mfma_f32_32x32x16_bf16 (lane =
// column, 16 rows a lane) is that of an operand whose contraction runs over those rows in a permuted order, so
// the state feeds O^T = S0^T Q^T, and each wave's own logits feed O^T += V^T P^T, from registers; Q and K rows
// are read from LDS in that order, V and K^T by transposing LDS reads.
#include <hip/hip_runtime.h>

#include "device.h"
#include "internal.h"

#include <algorithm>

namespace wavepp {
namespace {

constexpr int kC = kLinBlock;

__device__ __forceinline__ bool lin_meta_ok(const LinDevPlan& p) {
  return p.hdr->magic == kLinMagic && p.hdr->serial == p.serial;
}

__device__ __forceinline__ bf16x8 cat(bf16x4 a, bf16x4 b) {
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// Registers 8 kk .. 8 kk + 7 of an accumulator tile in bf16: an operand whose contraction runs over those rows.
__device__ __forceinline__ bf16x8 acc_operand(const f32x16& acc, int kk) {
  bf16x8 r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = static_cast<__bf16>(acc[8 * kk + e]);
  return r;
}

// Where a segment starts: a partial state, a snapshot, or nothing.
__device__ __forceinline__ const float* start_of(const LinDevPlan& p, const LinItem& it, const float* pool, int head) {
  const int64_t size = int64_t(p.head_dim_k) * p.head_dim_v;
  if (it.part_in >= 0) return p.parts + (int64_t(it.part_in) * p.num_heads + head) * size;
  if (it.state_in >= 0) return pool + (int64_t(it.state_in) * p.num_heads + head) * size;
  return nullptr;
}

// ---------------------------------------------------------------------------------------------
// Blocks of 64 tokens.  AHEAD: only the segment's own state, from zero, and its decay.
// ---------------------------------------------------------------------------------------------
template <int DK, int DV, bool AHEAD>
__global__ __launch_bounds__(DV * 2, 2) void lin_blocks_kernel(LinDevPlan p, const __bf16* __restrict__ q,
                                                               const __bf16* __restrict__ k,
                                                               const __bf16* __restrict__ v,
                                                               const float* __restrict__ alpha, float* pool,
                                                               __bf16* __restrict__ out) {
  constexpr int NW = DV / 32, NT = NW * 64;
  constexpr int KS = DK + 8, VS = DV + 32, DS = kC + 4;
  constexpr int KL = kC * DK / 8 / NT, VL = kC * DV / 8 / NT;     // 16-byte pieces per thread and block
  constexpr int CT = DK / 32;                                     // row tiles of the state
  __shared__ __attribute__((aligned(16))) __bf16 qs[AHEAD ? 8 : kC * KS];
  __shared__ __attribute__((aligned(16))) __bf16 ks[kC * KS];
  __shared__ __attribute__((aligned(16))) __bf16 vs[kC * VS];
  __shared__ __attribute__((aligned(16))) float dm[AHEAD ? 4 : kC * DS];   // D
  __shared__ __attribute__((aligned(16))) float al[kC], lam[kC], wt[kC];   // alpha, lam, D[63]

  if (!lin_meta_ok(p)) return;
  const int H = p.num_heads, Hqk = p.num_qk_heads;
  const LinItem it = p.segments[blockIdx.x / H];
  const int head = blockIdx.x % H, qk_head = head / (H / Hqk);
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 31, hf = lane >> 5;

  f32x16 S[CT];
#pragma unroll
  for (int c = 0; c < CT; ++c) S[c] = f32x16{};
  if (!AHEAD) {
    if (const float* s0 = start_of(p, it, pool, head)) {
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int r = 0; r < 16; ++r) S[c][r] = s0[(32 * c + 8 * (r >> 2) + 4 * hf + (r & 3)) * DV + 32 * wave + col];
    }
  }

  u32x4 qreg[AHEAD ? 1 : KL], kreg[KL], vreg[VL];
  float areg = 1.0f;
  auto load = [&](int t0) {
#pragma unroll
    for (int i = 0; i < KL; ++i) {
      const int c = tid + NT * i, row = c / (DK / 8), at = c % (DK / 8) * 8;
      const bool ok = t0 + row < it.len;
      const int64_t off = (int64_t(it.cu + t0 + row) * Hqk + qk_head) * DK + at;
      if (!AHEAD) qreg[AHEAD ? 0 : i] = ok ? *reinterpret_cast<const u32x4*>(q + off) : u32x4{};
      kreg[i] = ok ? *reinterpret_cast<const u32x4*>(k + off) : u32x4{};
    }
#pragma unroll
    for (int i = 0; i < VL; ++i) {
      const int c = tid + NT * i, row = c / (DV / 8), at = c % (DV / 8) * 8;
      const bool ok = t0 + row < it.len;
      vreg[i] = ok ? *reinterpret_cast<const u32x4*>(v + (int64_t(it.cu + t0 + row) * H + head) * DV + at) : u32x4{};
    }
    areg = t0 + lane < it.len ? alpha[p.alpha_per_token ? int64_t(it.cu + t0 + lane) * H + head : int64_t(head)] : 1.0f;
  };

  float total = 1.0f;                    // AHEAD: the segment's decay so far
  load(0);
  for (int t0 = 0, n; t0 < it.len; t0 += n) {
    n = min(kC, it.len - t0);
    // A value that is not finite times a weight of zero would reach the tokens before it: such a block goes token by
    // token, in blocks of one.
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < VL; ++i)
#pragma unroll
      for (int u = 0; u < 4; ++u) top = max(top, max(vreg[i][u] & 0x7FFFu, (vreg[i][u] >> 16) & 0x7FFFu));
    if (__syncthreads_or(top >= 0x7F80u)) n = AHEAD ? n : 1;
#pragma unroll
    for (int i = 0; i < KL; ++i) {
      const int c = tid + NT * i, row = c / (DK / 8), at = c % (DK / 8) * 8;
      if (!AHEAD) *reinterpret_cast<u32x4*>(&qs[AHEAD ? 0 : row * KS + at]) = row < n ? qreg[AHEAD ? 0 : i] : u32x4{};
      *reinterpret_cast<u32x4*>(&ks[row * KS + at]) = row < n ? kreg[i] : u32x4{};
    }
#pragma unroll
    for (int i = 0; i < VL; ++i) {
      const int c = tid + NT * i, row = c / (DV / 8), at = c % (DV / 8) * 8;
      *reinterpret_cast<u32x4*>(&vs[row * VS + at]) = row < n ? vreg[i] : u32x4{};
    }
    const float a = lane < n ? areg : 1.0f;
    // D: wave w the keys 16 w .. 16 w + 15 (waves of a narrower head two such groups), lane i the query
    float g = a;                         // products of the decays up to this lane's
#pragma unroll
    for (int s = 1; s < 64; s *= 2) {
      const float o = __shfl_up(g, s);
      if (lane >= s) g *= o;
    }
    if (wave == 0) {
      lam[lane] = g;
      al[lane] = a;
    }
    total *= __shfl(g, 63);
    if (AHEAD) {
      if (wave == 0) {
        float b = __shfl_down(a, 1);     // products of the decays after this lane's
        if (lane == 63) b = 1.0f;
#pragma unroll
        for (int s = 1; s < 64; s *= 2) {
          const float o = __shfl_down(b, s);
          if (lane + s < 64) b *= o;
        }
        wt[lane] = b;
      }
    } else {
#pragma unroll
      for (int j0 = 16 * wave; j0 < 64; j0 += 16 * NW) {
        float x = lane >= j0 + 16 ? a : 1.0f;              // products from key j0 + 16 up to this lane's
#pragma unroll
        for (int s = 1; s < 64; s *= 2) {
          const float o = __shfl_up(x, s);
          if (lane >= s) x *= o;
        }
        if (lane < j0 + 15) x = 0.0f;
        float d[16];
#pragma unroll
        for (int j = 15; j >= 0; --j) {
          if (j < 15) x *= __shfl(a, j0 + j + 1);
          if (lane == j0 + j) x = 1.0f;
          d[j] = lane < j0 + j ? 0.0f : x;
        }
#pragma unroll
        for (int j = 0; j < 16; j += 4)
          *reinterpret_cast<f32x4*>(&dm[AHEAD ? 0 : lane * DS + j0 + j]) = f32x4{d[j], d[j + 1], d[j + 2], d[j + 3]};
      }
    }
    __syncthreads();
    if (t0 + n < it.len) load(t0 + n);

    const __bf16* vl = &vs[(4 * hf + (lane & 15) / 4) * VS + 32 * wave + 16 * ((lane >> 4) & 1) + 4 * (lane & 3)];
    bf16x8 vf[4];                        // V^T of this wave's columns: tokens 16 t + 8 (e / 4) + 4 hf + e % 4
#pragma unroll
    for (int t = 0; t < 4; ++t) vf[t] = cat(lds_read_tr(vl + 16 * t * VS), lds_read_tr(vl + (16 * t + 8) * VS));

    if constexpr (!AHEAD) {
      f32x16 o[2] = {f32x16{}, f32x16{}};                  // O^T: tokens 0-31 and 32-63
      f32x16 s00 = f32x16{}, s01 = f32x16{}, s11 = f32x16{};   // K Q^T: key half, query half
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
          const int at = 32 * c + 16 * kk + 4 * hf;
          auto row = [&](const __bf16* m, int r) {
            const __bf16* x = m + r * KS + at;
            return cat(*reinterpret_cast<const bf16x4*>(x), *reinterpret_cast<const bf16x4*>(x + 8));
          };
          const bf16x8 q0 = row(qs, col), q1 = row(qs, 32 + col), k0 = row(ks, col), k1 = row(ks, 32 + col);
          const bf16x8 st = acc_operand(S[c], kk);
          o[0] = mfma(st, q0, o[0]);
          o[1] = mfma(st, q1, o[1]);
          s00 = mfma(k0, q0, s00);
          s01 = mfma(k0, q1, s01);
          s11 = mfma(k1, q1, s11);
        }
      const float l0 = lam[col], l1 = lam[32 + col];
#pragma unroll
      for (int r = 0; r < 16; ++r) o[0][r] *= l0, o[1][r] *= l1;
      // the weights of the keys for this lane's two queries; above the diagonal nothing, whatever the product was
      auto weigh = [&](f32x16& s, int i0, int j0) {
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const f32x4 d = *reinterpret_cast<const f32x4*>(&dm[(i0 + col) * DS + j0 + 8 * u + 4 * hf]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float x = s[4 * u + e] * d[e];
            s[4 * u + e] = i0 != j0 || 8 * u + 4 * hf + e <= col ? x : 0.0f;
          }
        }
      };
      weigh(s00, 0, 0);
      weigh(s01, 32, 0);
      weigh(s11, 32, 32);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        o[0] = mfma(vf[t], acc_operand(s00, t), o[0]);
        o[1] = mfma(vf[t], acc_operand(s01, t), o[1]);
        o[1] = mfma(vf[2 + t], acc_operand(s11, t), o[1]);
      }
      // O^T through this wave's columns of V in LDS (its reads of them are done) to rows of 64 bytes
      __bf16* mine = &vs[32 * wave];
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          bf16x4 x;
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = static_cast<__bf16>(o[i][4 * u + e] * p.scale);
          *reinterpret_cast<bf16x4*>(mine + (32 * i + col) * VS + 8 * u + 4 * hf) = x;
        }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int row = 16 * i + lane / 4, at = 8 * (lane & 3);
        const u32x4 x = *reinterpret_cast<const u32x4*>(mine + row * VS + at);
        if (row < n)
          *reinterpret_cast<u32x4*>(out + (int64_t(it.cu + t0 + row) * H + head) * DV + 32 * wave + at) = x;
      }
    }

    // S = lam_64 S + K^T (w V): the weighted values as two bf16 parts, which leave the state right to 2^-16
    const float gamma = lam[63];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) S[c][r] *= gamma;
    const __bf16* kl = &ks[(4 * hf + (lane & 15) / 4) * KS + 16 * ((lane >> 4) & 1) + 4 * (lane & 3)];
    const float* last = AHEAD ? wt : &dm[AHEAD ? 0 : 63 * DS];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      const f32x4 w0 = *reinterpret_cast<const f32x4*>(last + 16 * t + 4 * hf), w1 = *reinterpret_cast<const f32x4*>(last + 16 * t + 8 + 4 * hf);
      bf16x8 hi, lo;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = float(vf[t][e]) * (e < 4 ? w0[e & 3] : w1[e & 3]);
        hi[e] = static_cast<__bf16>(x);
        lo[e] = static_cast<__bf16>(x - float(hi[e]));
      }
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const bf16x8 kt = cat(lds_read_tr(kl + 16 * t * KS + 32 * c), lds_read_tr(kl + (16 * t + 8) * KS + 32 * c));
        S[c] = mfma(kt, hi, S[c]);
        S[c] = mfma(kt, lo, S[c]);
      }
    }
  }

  const int64_t size = int64_t(DK) * DV;
  float* to = AHEAD ? p.parts + (int64_t(it.part_out) * H + head) * size
                    : it.state_out >= 0 ? pool + (int64_t(it.state_out) * H + head) * size : nullptr;
  if (to) {
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int r = 0; r < 16; ++r) to[(32 * c + 8 * (r >> 2) + 4 * hf + (r & 3)) * DV + 32 * wave + col] = S[c][r];
  }
  if (AHEAD && tid == 0) p.part_decay[int64_t(it.part_out) * H + head] = total;
}

// ---------------------------------------------------------------------------------------------
// The states between the segments of a request, in place of the segments' own states: one thread four values.
// ---------------------------------------------------------------------------------------------
__global__ __launch_bounds__(256) void lin_scan_kernel(LinDevPlan p, const float* __restrict__ pool) {
  if (!lin_meta_ok(p)) return;
  const int H = p.num_heads;
  const LinScan sc = p.scans[blockIdx.x / H];
  const int head = blockIdx.x % H;
  const int64_t size = int64_t(p.head_dim_k) * p.head_dim_v, at = 4 * (int64_t(blockIdx.y) * 256 + threadIdx.x);
  f32x4 s = f32x4{};
  if (sc.state_in >= 0) s = *reinterpret_cast<const f32x4*>(pool + (int64_t(sc.state_in) * H + head) * size + at);
  if (sc.start_part >= 0) *reinterpret_cast<f32x4*>(p.parts + (int64_t(sc.start_part) * H + head) * size + at) = s;
  for (int i = 0; i < sc.count; ++i) {
    const int64_t part = int64_t(sc.first_part + i) * H + head;
    const float g = p.part_decay[part];
    f32x4* own = reinterpret_cast<f32x4*>(p.parts + part * size + at);
    s = g * s + *own;
    *own = s;
  }
}

// ---------------------------------------------------------------------------------------------
// Token by token, in fp32.  A workgroup has 32 columns of one (request, head)'s state in registers: thread (row group,
// column quad).  The outputs' sums over the rows are joined in LDS.
// ---------------------------------------------------------------------------------------------
template <int DK, int DV>
__global__ __launch_bounds__(256) void lin_step_kernel(LinDevPlan p, const __bf16* __restrict__ q,
                                                       const __bf16* __restrict__ k, const __bf16* __restrict__ v,
                                                       const float* __restrict__ alpha, float* pool,
                                                       __bf16* __restrict__ out) {
  constexpr int W = 32, RG = 256 / (W / 4), RPT = DK / RG;     // columns, row groups, rows per thread
  __shared__ __attribute__((aligned(16))) f32x4 sum[RG][W / 4];
  if (!lin_meta_ok(p)) return;
  const int H = p.num_heads, Hqk = p.num_qk_heads;
  const LinItem it = p.steps[blockIdx.x / (DV / W) / H];
  const int head = blockIdx.x / (DV / W) % H, c0 = blockIdx.x % (DV / W) * W, qk_head = head / (H / Hqk);
  const int tid = threadIdx.x, cq = tid % (W / 4), rg = tid / (W / 4), at = c0 + 4 * cq;
  const int64_t size = int64_t(DK) * DV;
  f32x4 S[RPT];
  if (const float* s0 = start_of(p, it, pool, head)) {
#pragma unroll
    for (int i = 0; i < RPT; ++i) S[i] = *reinterpret_cast<const f32x4*>(s0 + (rg + RG * i) * DV + at);
  } else {
#pragma unroll
    for (int i = 0; i < RPT; ++i) S[i] = f32x4{};
  }
  for (int t = 0; t < it.len; ++t) {
    const int64_t tok = it.cu + t;
    const float a = alpha[p.alpha_per_token ? tok * H + head : int64_t(head)];
    const bf16x4 vb = *reinterpret_cast<const bf16x4*>(v + (tok * H + head) * DV + at);
    f32x4 x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = float(vb[e]);
    f32x4 o = f32x4{};
#pragma unroll
    for (int i = 0; i < RPT; ++i) {
      const int64_t row = (tok * Hqk + qk_head) * DK + rg + RG * i;
      const float kr = float(k[row]), qr = float(q[row]);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        S[i][e] = fmaf(kr, x[e], a * S[i][e]);
        o[e] = fmaf(qr, S[i][e], o[e]);
      }
    }
    if (t) __syncthreads();                // the sums of the token before are read
    sum[rg][cq] = o;
    __syncthreads();
    if (tid < W) {
      float y = 0.0f;
#pragma unroll
      for (int g = 0; g < RG; ++g) y += sum[g][tid / 4][tid % 4];
      out[(tok * H + head) * DV + c0 + tid] = static_cast<__bf16>(y * p.scale);
    }
  }
  float* to = pool + (int64_t(it.state_out) * H + head) * size;
#pragma unroll
  for (int i = 0; i < RPT; ++i) *reinterpret_cast<f32x4*>(to + (rg + RG * i) * DV + at) = S[i];
}

template <int DK, int DV>
hipError_t launch_dims(const LinDevPlan& p, const __bf16* q, const __bf16* k, const __bf16* v, const float* alpha,
                       float* pool, __bf16* out, hipStream_t stream) {
  const int H = p.num_heads;
  if (p.num_steps)
    hipLaunchKernelGGL((lin_step_kernel<DK, DV>), dim3(p.num_steps * H * (DV / 32)), dim3(256), 0, stream, p, q, k, v, alpha,
                       pool, out);
  if (p.num_ahead)
    hipLaunchKernelGGL((lin_blocks_kernel<DK, DV, true>), dim3(p.num_ahead * H), dim3(2 * DV), 0, stream, p, q, k, v, alpha,
                       pool, out);
  if (p.num_scans)
    hipLaunchKernelGGL(lin_scan_kernel, dim3(p.num_scans * H, DK * DV / 1024), dim3(256), 0, stream, p, pool);
  if (p.num_segments)
    hipLaunchKernelGGL((lin_blocks_kernel<DK, DV, false>), dim3(p.num_segments * H), dim3(2 * DV), 0, stream, p, q, k, v,
                       alpha, pool, out);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_lin(const LinDevPlan& p, const void* q, const void* k, const void* v, const float* alpha,
                      float* state_pool, void* out, hipStream_t stream) {
  auto qq = static_cast<const __bf16*>(q);
  auto kk = static_cast<const __bf16*>(k);
  auto vv = static_cast<const __bf16*>(v);
  auto oo = static_cast<__bf16*>(out);
  if (p.head_dim_k == 128 && p.head_dim_v == 128) return launch_dims<128, 128>(p, qq, kk, vv, alpha, state_pool, oo, stream);
  if (p.head_dim_k == 128 && p.head_dim_v == 64) return launch_dims<128, 64>(p, qq, kk, vv, alpha, state_pool, oo, stream);
  if (p.head_dim_k == 64 && p.head_dim_v == 128) return launch_dims<64, 128>(p, qq, kk, vv, alpha, state_pool, oo, stream);
  if (p.head_dim_k == 64 && p.head_dim_v == 64) return launch_dims<64, 64>(p, qq, kk, vv, alpha, state_pool, oo, stream);
  return hipErrorInvalidValue;
}

}  // namespace wavepp
