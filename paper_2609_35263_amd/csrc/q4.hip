// gfx950 (CDNA4) kernels of libwavepp_attn's 4-bit paged cache: the append that quantises, the way back to bf16
// rows, and grouped-query attention over 4-bit pages.
//
// A value is an e2m1 code times the power of two 2^(e - 127) of its block of 32 along the head dim, so it is exactly
// a bf16 number and the attention multiplies bf16 operands that equal the cached values: nothing is lost after the
// append.  gfx950 turns eight codes of a 32-bit word into eight scaled bf16 with four instructions
// (v_cvt_scalef32_pk_bf16_fp4), which leaves them in the order of a matrix instruction's operand.
#include <hip/hip_runtime.h>

#include "device.h"
#include "q4.h"

#include <algorithm>

namespace wavepp {
namespace {

// One page of one head: codes of all rows, then their scale bytes.
template <int D, int PAGE>
struct Q4Page {
  static constexpr int ROW = D / 2;                  // code bytes of a row
  static constexpr int NB = D / kQ4Block;            // blocks, so scale bytes, of a row
  static constexpr int CODES = PAGE * ROW;
  static constexpr int BYTES = CODES + PAGE * NB;
};

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// The eight values of a word of codes, lowest nibble first.
__device__ __forceinline__ bf16x8 q4_values(uint32_t codes, float scale) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// Where the 8-value piece c of a V row lies in its LDS row (stride 16 banks past a multiple of 64): the four pieces of a
// block of 32 exchange places by the block's number.  A thread writes one block piece by piece; in order, all threads'
// pieces of one turn would fall on a quarter of the banks (192 of 290 LDS cycles a block of 32 keys were such conflicts).
__device__ __forceinline__ int v_place(int c) { return 8 * (c ^ ((c >> 2) & 3)); }

// ---------------------------------------------------------------------------------------------
// Append and read.  One thread moves eight values of a row (16 bytes of bf16, 4 of codes); the four
// threads of a block of 32 find its largest magnitude between them.  A workgroup takes TOK consecutive tokens.
// ---------------------------------------------------------------------------------------------

// The value of another lane of the same four, by a quad permutation.
template <int CTRL>
__device__ __forceinline__ uint32_t quad_other(uint32_t x) {
  return uint32_t(__builtin_amdgcn_update_dpp(0, int(x), CTRL, 0xF, 0xF, true));
}

// The request that holds packed token t: the last with cu <= t (requests without a chunk share cu with the next).
__device__ __forceinline__ int request_of(const DevPlan& p, int64_t t) {
  int lo = 0, hi = p.num_requests - 1;
  while (hi > lo) {
    const int mid = (lo + hi + 1) >> 1;
    if (const_load(&p.reqs[mid].cu) <= t) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// The first of the workgroup's TOK tokens.  Each L2 domain (workgroups go to them round-robin) has a run of the wave's
// tokens, so that the rows and scales that share a line of a page meet in one L2.
template <int TOK>
__device__ __forceinline__ int64_t first_token(const DevPlan& p) {
  const int64_t per = gridDim.x / kNumXcd;
  return (int64_t(blockIdx.x) % kNumXcd * per + blockIdx.x / kNumXcd) * TOK;
}

// The workgroup's tokens: page of the pool and slot in it of each; the number of tokens.
template <int TOK>
__device__ __forceinline__ int token_places(const DevPlan& p, int64_t t0, int64_t (&page)[TOK], int (&slot)[TOK]) {
  int r = request_of(p, t0);
  const int n = int(min(int64_t(TOK), p.total_tokens - t0));
#pragma unroll
  for (int i = 0; i < TOK; ++i) {
    const int64_t t = t0 + min(i, n - 1);
    while (r + 1 < p.num_requests && const_load(&p.reqs[r + 1].cu) <= t) ++r;
    const ReqMeta* rq = &p.reqs[r];
    const int pos = const_load(&rq->prefix) + int(t - const_load(&rq->cu));
    page[i] = const_load(&p.bt[const_load(&rq->bt_row) + pos / p.page_size]);
    slot[i] = pos % p.page_size;
  }
  return n;
}

template <int D, int TOK>
__global__ __launch_bounds__(256) void q4_append_kernel(DevPlan p, const u32x4* __restrict__ k_new,
                                                        const u32x4* __restrict__ v_new, uint8_t* __restrict__ k_pool,
                                                        uint8_t* __restrict__ v_pool) {
  if (!meta_ok(p)) return;
  constexpr int CH = D / 8, NB = D / kQ4Block;
  const int Hkv = p.num_kv_heads, B = p.page_size;
  const int64_t page_bytes = int64_t(B) * (D / 2 + NB), t0 = first_token<TOK>(p);
  if (t0 >= p.total_tokens) return;
  int64_t page[TOK];
  int slot[TOK];
  const int n = token_places(p, t0, page, slot);
  for (int u = threadIdx.x; u < Hkv * 2 * CH; u += blockDim.x) {
    const int h = u / (2 * CH), c = u % CH;
    const bool is_v = u % (2 * CH) >= CH;
    const u32x4* rows = (is_v ? v_new : k_new) + (t0 * Hkv + h) * CH + c;
    u32x4 x[TOK];
#pragma unroll
    for (int i = 0; i < TOK; ++i) x[i] = rows[int64_t(min(i, n - 1)) * Hkv * CH];
#pragma unroll
    for (int i = 0; i < TOK; ++i) {
      if (i >= n) break;
      // magnitudes of bf16 order like integers; NaN and infinities become the largest finite one
      uint32_t y[4], top = 0;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const uint32_t lo = min(x[i][w] & 0x7FFFu, 0x7F7Fu), hi = min((x[i][w] >> 16) & 0x7FFFu, 0x7F7Fu);
        y[w] = (x[i][w] & 0x80008000u) | lo | (hi << 16);
        top = max(top, max(lo, hi));
      }
      top = max(top, quad_other<0xB1>(top));               // lanes 1, 0, 3, 2
      top = max(top, quad_other<0x4E>(top));               // lanes 2, 3, 0, 1
      // top = 1.m * 2^(E - 127): the smallest s with top <= 7 s is 2^(E - 127 - 2), twice that where 1.m > 1.75
      const int e = min(max(int(top >> 7) - 2 + int((top & 0x7Fu) > 0x60u), 8), 252);
      const float s = scale_of(uint32_t(e));
      uint32_t codes = 0;
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, y[0]), s, 0);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, y[1]), s, 1);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, y[2]), s, 2);
      codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(codes, __builtin_bit_cast(bf16x2, y[3]), s, 3);
      uint8_t* run = (is_v ? v_pool : k_pool) + (page[i] * Hkv + h) * page_bytes;
      *reinterpret_cast<uint32_t*>(run + slot[i] * (D / 2) + 4 * c) = codes;
      if (c % 4 == 0) run[B * (D / 2) + slot[i] * NB + c / 4] = uint8_t(e);
    }
  }
}

template <int D, int TOK>
__global__ __launch_bounds__(256) void q4_read_kernel(DevPlan p, const uint8_t* __restrict__ k_pool,
                                                      const uint8_t* __restrict__ v_pool, bf16x8* __restrict__ k_out,
                                                      bf16x8* __restrict__ v_out) {
  if (!meta_ok(p)) return;
  constexpr int CH = D / 8, NB = D / kQ4Block;
  const int Hkv = p.num_kv_heads, B = p.page_size;
  const int64_t page_bytes = int64_t(B) * (D / 2 + NB), t0 = first_token<TOK>(p);
  if (t0 >= p.total_tokens) return;
  int64_t page[TOK];
  int slot[TOK];
  const int n = token_places(p, t0, page, slot);
  for (int u = threadIdx.x; u < Hkv * 2 * CH; u += blockDim.x) {
    const int h = u / (2 * CH), c = u % CH;
    const bool is_v = u % (2 * CH) >= CH;
    const uint8_t* pool = (is_v ? v_pool : k_pool) + h * page_bytes;
    uint32_t codes[TOK], scale[TOK];
#pragma unroll
    for (int i = 0; i < TOK; ++i) {
      const uint8_t* run = pool + page[i] * Hkv * page_bytes;
      codes[i] = *reinterpret_cast<const uint32_t*>(run + slot[i] * (D / 2) + 4 * c);
      scale[i] = run[B * (D / 2) + slot[i] * NB + c / 4];
    }
    bf16x8* rows = (is_v ? v_out : k_out) + (t0 * Hkv + h) * CH + c;
#pragma unroll
    for (int i = 0; i < TOK; ++i)
      if (i < n) rows[int64_t(i) * Hkv * CH] = q4_values(codes[i], scale_of(scale[i]));
  }
}

// A weight is 2 to the power of its logit (times log2 e) less a reference m, which lies at most 8 under the largest.  The key that
// set m has a weight of 2^d, d being what m lost when it was rounded: nothing that matters up to 2^28, where d is 16 at
// most and the row's sum takes it out again; beyond, that weight could be anything, 0 and infinity among it.  So logits
// under -2^28 weigh nothing, like masked ones (a split may hold no others), and a reference over 2^28 gives a row of NaN.
constexpr float kFarLogit = 0x1p28f;
__device__ __forceinline__ float reference(float m) { return m < -kFarLogit ? 0.0f : m; }
// The sum that a row's outputs are divided by: 0 for a row of no weight, NaN for one that has no sum.
__device__ __forceinline__ float row_sum(float m, float l) { return m <= kFarLogit ? l : NAN; }

// ---------------------------------------------------------------------------------------------
// Attention of many rows.  The layout is that of the kernel over bf16 pages (kernels.hip): a workgroup of NW waves
// takes 32 NW query rows of one (request, KV head) and walks tiles of keys that all its rows share; logits S^T = K Q^T
// and O^T += V^T P^T on 32x32x16 matrix instructions, K from LDS rows, V by transposing LDS reads, the probabilities
// straight from the accumulators.  A tile's codes are loaded (a quarter of the bytes, 8 registers a thread) before
// the MFMAs of the tile before it and turned into bf16 rows in the other LDS buffer after them: once for all NW waves.
// It is bound by the matrix instructions and the softmax's VALU work beside them, as over bf16 pages: 1,024 tokens behind 65,536
// (64/8 heads of 128) 1,834 us, 1.21 PFLOP/s where a large library product reaches 1.35 (1,885 us with V's pieces in order,
// see v_place).  8 x 16 tokens behind 16-32 K: 136 us, four waves, twice the dequantisation for a row; the memory would
// take 48.
// ---------------------------------------------------------------------------------------------
template <int D, int PAGE, int NW>
__global__ __launch_bounds__(NW * 64, NW == 4 ? 2 : 1) void attn_q4_kernel(DevPlan p, const __bf16* __restrict__ q,
                                                                           const uint8_t* __restrict__ kpool,
                                                                           const uint8_t* __restrict__ vpool,
                                                                           __bf16* __restrict__ out,
                                                                           float* __restrict__ lse_out) {
  typedef Q4Page<D, PAGE> Page;
  constexpr int KT = NW == 4 ? kKvTile / 2 : kKvTile;   // keys per tile
  constexpr int NKB = KT / 32;
  constexpr int KSTR = D + 8;          // K rows in LDS: 16-byte reads of 8 rows land on distinct banks
  constexpr int VSTR = D + 32;         // V rows: transposed reads of 4 rows x 2 groups x 32 bytes on distinct banks
  constexpr int W = D / 32;            // words of codes per thread and tile, for K and for V: a quarter of a row
  static_assert(KT * 4 == NW * 64, "four threads a key");
  __shared__ __attribute__((aligned(16))) __bf16 ks[2][KT * KSTR];
  __shared__ __attribute__((aligned(16))) __bf16 vs[2][KT * VSTR];

  if (!meta_ok(p)) return;
  const WorkItem it = p.items[blockIdx.x];
  if (it.rows <= 0) return;
  const ReqMeta rm = p.reqs[it.req];
  const int Hq = p.num_q_heads, Hkv = p.num_kv_heads;
  const int G = Hq / Hkv;
  const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, col = lane & 31, hf = lane >> 5;
  const int n_valid = rm.prefix + rm.chunk;
  const int32_t* __restrict__ bt = p.bt + rm.bt_row;
  const int64_t page_stride = int64_t(Hkv) * Page::BYTES;
  const uint8_t* __restrict__ kpool_h = kpool + int64_t(it.kv_head) * Page::BYTES;
  const uint8_t* __restrict__ vpool_h = vpool + int64_t(it.kv_head) * Page::BYTES;

  // ---- this lane's query row -----------------------------------------------------------------
  const int lrow = wave * 32 + col;
  const bool row_ok = lrow < it.rows;
  const int prow = it.row0 + (row_ok ? lrow : 0);
  const int tok = prow / G;
  const int head = it.kv_head * G + (prow - tok * G);
  const int limit = rm.prefix + tok;                             // last key this row may see
  bf16x8 qf[D / 16];
  {
    const __bf16* qrow = q + (int64_t(rm.cu + tok) * Hq + head) * D + 8 * hf;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) qf[s] = row_ok ? *reinterpret_cast<const bf16x8*>(qrow + 16 * s) : bf16x8{};
  }
  const int wrow0 = wave * 32;
  const bool wave_active = wrow0 < it.rows;
  const int wrow_last = min(it.rows, wrow0 + 32) - 1;
  const int wave_min_lim = rm.prefix + (it.row0 + wrow0) / G;
  const int wave_max_lim = rm.prefix + (it.row0 + max(wrow_last, wrow0)) / G;

  f32x16 oacc[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db) oacc[db] = f32x16{};
  float m_run = -INFINITY, l_run = 0.0f;
  const float sl2 = p.softmax_scale * kLog2e;

  // ---- K/V tile staging -----------------------------------------------------------------------
  // Thread tid has a quarter of key tid / 4's row.  Positions past the request's last valid one are clamped to that
  // one: finite copies that the mask gives zero weight, so stale slots are never read.
  const int key = tid >> 2, part = tid & 3;
  uint32_t kreg[W], vreg[W], kscale = 0, vscale = 0;
  // The page of this thread's key is looked up one tile ahead.
  auto page_of = [&](int tile) { return bt[min(tile * KT + key, n_valid - 1) / PAGE]; };
  auto load_tile = [&](int tile, int page) {
    const int j = min(tile * KT + key, n_valid - 1);
    const int64_t at = int64_t(page) * page_stride;
    const uint32_t off = uint32_t(j % PAGE) * Page::ROW + part * (W * 4);
    const uint32_t soff = Page::CODES + uint32_t(j % PAGE) * Page::NB + part * Page::NB / 4;
    if constexpr (W == 4) {
      const u32x4 a = *reinterpret_cast<const u32x4*>(kpool_h + at + off);
      const u32x4 b = *reinterpret_cast<const u32x4*>(vpool_h + at + off);
#pragma unroll
      for (int i = 0; i < W; ++i) kreg[i] = a[i], vreg[i] = b[i];
    } else {
      const u32x2 a = *reinterpret_cast<const u32x2*>(kpool_h + at + off);
      const u32x2 b = *reinterpret_cast<const u32x2*>(vpool_h + at + off);
#pragma unroll
      for (int i = 0; i < W; ++i) kreg[i] = a[i], vreg[i] = b[i];
    }
    kscale = kpool_h[at + soff];
    vscale = vpool_h[at + soff];
  };
  auto store_tile = [&](int buf) {
    __bf16* kd = &ks[buf][key * KSTR + part * (W * 8)];
    const float a = scale_of(kscale), b = scale_of(vscale);
#pragma unroll
    for (int i = 0; i < W; ++i) {
      *reinterpret_cast<bf16x8*>(kd + 8 * i) = q4_values(kreg[i], a);
      *reinterpret_cast<bf16x8*>(&vs[buf][key * VSTR + v_place(part * W + i)]) = q4_values(vreg[i], b);
    }
  };

  // per-lane LDS read bases.  K (A operand of S^T = K Q^T): row col, elements 8*hf.. of each
  // 16-wide step.  V (A operand of O^T = V^T P^T, read transposed): within its 16-lane group, lane
  // j = lane % 16 addresses key 4*hf + j/4 and d = 16*((lane/16) % 2) + 4*(j%4) of a 16-key step.
  const int k_lane = col * KSTR + 8 * hf;
  int v_lane[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
    v_lane[db] = (4 * hf + (lane & 15) / 4) * VSTR + v_place(4 * db + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) +
                 4 * (lane & 1);

  const int t_begin = it.kv_begin / KT;
  const int t_end = (it.kv_end + KT - 1) / KT;
  load_tile(t_begin, page_of(t_begin));
  store_tile(0);
  int pg_nxt = page_of(t_begin + 1);
  __syncthreads();

  for (int tile = t_begin; tile < t_end; ++tile) {
    const int buf = (tile - t_begin) & 1;
    const bool has_next = tile + 1 < t_end;
    if (has_next) {
      load_tile(tile + 1, pg_nxt);
      pg_nxt = page_of(tile + 2);
    }
    const int kbase = tile * KT;
    if (wave_active && kbase <= wave_max_lim) {
      // S^T[key][row] for the KT keys of the tile, as NKB 32-key blocks
      f32x16 sacc[NKB];
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb) sacc[kb] = f32x16{};
      const __bf16* kl = &ks[buf][k_lane];
#pragma unroll
      for (int s = 0; s < D / 16; ++s)
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb) {
          const bf16x8 kf = *reinterpret_cast<const bf16x8*>(kl + 32 * kb * KSTR + 16 * s);
          sacc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[s], sacc[kb], 0, 0, 0);
        }
      // keep four K fragment reads in flight ahead of the MFMAs that consume them
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
      for (int i = 0; i < (D / 16) * NKB - 4; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
      // accumulator element r of block kb holds key 32*kb + 8*(r/4) + 4*hf + (r%4)
      const bool need_mask = (kbase + KT - 1 > wave_min_lim) || (kbase + KT > it.kv_end);
      if (need_mask) {
        const int bound = min(limit, it.kv_end - 1) - kbase - 4 * hf;
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (32 * kb + 8 * (r >> 2) + (r & 3) > bound) sacc[kb][r] = -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sacc[kb][r]);
      mx = halves_max(mx) * sl2;
      // The reference max only moves when the tile's max exceeds it by more than 2^8, so most tiles
      // skip rescaling the accumulators; probabilities stay below 256, which bf16/fp32 represent as
      // well as values below 1.  The final normalization uses the same reference.
      const bool bump = mx > m_run + 8.0f;
      const float m_new = bump ? mx : m_run;
      const float m_use = reference(m_new);
      float rs = 0.0f;
      bf16x8 pb[2 * NKB];
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float e = fast_exp2(fmaf(sacc[kb][r], sl2, -m_use));
          rs += e;
          pb[2 * kb + (r >> 3)][r & 7] = static_cast<__bf16>(e);
        }
      rs = halves_sum(rs);
      if (__any(bump)) {
        const float alpha = fast_exp2(m_run - m_use);
        l_run *= alpha;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) oacc[db][r] *= alpha;
      }
      l_run += rs;
      m_run = m_new;
      // O^T[d][row] += V^T[d][key] P^T[key][row]; step t covers keys 16t + 8*(e/4) + 4*hf + (e%4),
      // the order in which the S^T accumulator holds them
      const __bf16* vl = &vs[buf][0];
#pragma unroll
      for (int t = 0; t < 2 * NKB; ++t)
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
          const bf16x4 lo = lds_read_tr(vl + v_lane[db] + 16 * t * VSTR);
          const bf16x4 hi = lds_read_tr(vl + v_lane[db] + (16 * t + 8) * VSTR);
          const bf16x8 a = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
          oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[t], oacc[db], 0, 0, 0);
        }
      // keep two MFMAs' worth of transposed V reads in flight
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 1);
#pragma unroll
      for (int i = 0; i < (D / 32) * 2 * NKB - 2; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 1);
        __builtin_amdgcn_sched_group_barrier(0x100, 2, 1);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, 2, 1);
    }
    if (has_next) store_tile(buf ^ 1);
    __syncthreads();
  }

  // ---- epilogue: O = O^T / l, lse = ln(l) + m (natural log) ------------------------------------
  if (!row_ok) return;
  const float sum = row_sum(m_run, l_run);
  const float inv_l = sum == 0.0f ? 0.0f : 1.0f / sum;
  const float lse_v = sum == 0.0f ? -INFINITY : (m_run + __log2f(sum)) * kLn2;
  if (it.part < 0) {
    __bf16* orow = out + (int64_t(rm.cu + tok) * Hq + head) * D;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        bf16x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = static_cast<__bf16>(oacc[db][4 * u + k] * inv_l);
        *reinterpret_cast<bf16x4*>(orow + 32 * db + 8 * u + 4 * hf) = v;
      }
    if (lse_out && hf == 0) lse_out[int64_t(rm.cu + tok) * Hq + head] = lse_v;
  } else {
    float* orow = p.opart + int64_t(it.part + lrow) * D;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        f32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = oacc[db][4 * u + k] * inv_l;
        *reinterpret_cast<f32x4*>(orow + 32 * db + 8 * u + 4 * hf) = v;
      }
    if (hf == 0) p.lpart[it.part + lrow] = lse_v;
  }
}

// ---------------------------------------------------------------------------------------------
// Attention of few rows: up to 32 query rows for each (request, KV head), so one token of up to 32 heads a group or a
// few tokens.  The cache is read once and hardly computed with, so the work is to keep loads in flight: the
// four waves of a workgroup each take every fourth block of 32 keys with all the rows, straight from memory into
// registers, and join their sums at the end.
//   * K needs no LDS: a lane has 16-byte pieces (one scale block each) of the row it feeds to the matrix instruction.
//     Any order of the contraction over the head dim will do, so step 4 i + u takes word u of piece i: the values
//     32 (2 i + hf) + 8 u .. + 7 of the row, and Q's rows are loaded in that order.
//   * V needs transposing: its bf16 values go through rows in LDS that belong to the wave alone, without barriers.
// Bound by memory: a token each behind 64 x 1-32 K cached (64/8 heads of 128, pages of 64) 226 us, 5.1 TB/s of codes and
// scales, above a large copy's rate (321 us with branches around the loads and whole items, see few_rows_split for the cut).
// With pages of 16 the same wave takes 280 us: at head dim 128 that form has 10 registers too many, and what it reads back
// from scratch waits for both blocks in flight (28 bytes a lane; the form with pages of 64 has 254 registers and none).
// ---------------------------------------------------------------------------------------------
template <int D, int PAGE>
__global__ __launch_bounds__(256, 2) void attn_q4_few_kernel(DevPlan p, const __bf16* __restrict__ q,
                                                             const uint8_t* __restrict__ kpool,
                                                             const uint8_t* __restrict__ vpool,
                                                             __bf16* __restrict__ out, float* __restrict__ lse_out) {
  typedef Q4Page<D, PAGE> Page;
  constexpr int NB = Page::NB, NL = D / 64;      // 16-byte pieces per lane of 32 rows
  constexpr int VSTR = D + 32;                   // transposed reads of 4 rows x 2 groups x 32 bytes on distinct banks
  constexpr int OSTR = 64 + 4;                   // floats per row while the waves' sums are joined
  constexpr int VBYTES = 32 * VSTR * 2, JOIN = 4 * 32 * OSTR * 4;
  __shared__ __attribute__((aligned(16))) unsigned char smem[4 * VBYTES > JOIN ? 4 * VBYTES : JOIN];
  __shared__ float wave_m[4][32], wave_l[4][32];

  if (!meta_ok(p)) return;
  const WorkItem it = p.items[blockIdx.x];
  if (it.rows <= 0) return;
  const ReqMeta rm = p.reqs[it.req];
  const int Hq = p.num_q_heads, Hkv = p.num_kv_heads;
  const int G = Hq / Hkv;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int last = rm.prefix + rm.chunk - 1;     // the request's last valid position
  const int32_t* __restrict__ bt = p.bt + rm.bt_row;
  const int64_t page_stride = int64_t(Hkv) * Page::BYTES;
  const uint8_t* __restrict__ kpool_h = kpool + int64_t(it.kv_head) * Page::BYTES;
  const uint8_t* __restrict__ vpool_h = vpool + int64_t(it.kv_head) * Page::BYTES;

  const bool row_ok = col < it.rows;
  const int prow = it.row0 + (row_ok ? col : 0);
  const int tok = prow / G;
  const int limit = rm.prefix + tok;             // last key this row may see
  bf16x8 qf[D / 16];
  {
    const __bf16* qrow = q + (int64_t(rm.cu + tok) * Hq + it.kv_head * G + (prow - tok * G)) * D;
#pragma unroll
    for (int s = 0; s < D / 16; ++s)
      qf[s] = row_ok ? *reinterpret_cast<const bf16x8*>(qrow + 64 * (s / 4) + 32 * hf + 8 * (s % 4)) : bf16x8{};
  }
  const int min_lim = rm.prefix + it.row0 / G;
  const float sl2 = p.softmax_scale * kLog2e;

  struct Block {                                 // 32 keys
    u32x4 k[NL], v[NL];
    uint32_t kscale, vscale[NL];
  };
  // Positions past the last valid one are clamped to it, so stale slots are never read.
  auto load = [&](Block& b, int block) {
    const int kbase = 32 * block;
    const int pg0 = bt[kbase / PAGE], pg1 = PAGE == 16 ? bt[min(kbase + 16, last) / PAGE] : pg0;
    auto run = [&](const uint8_t* pool, int j) {
      const int page = PAGE == 16 && j - kbase >= 16 ? pg1 : pg0;
      return pool + int64_t(page) * page_stride;
    };
    {
      const int j = min(kbase + col, last), slot = j % PAGE;
      const uint8_t* r = run(kpool_h, j);
#pragma unroll
      for (int i = 0; i < NL; ++i) b.k[i] = *reinterpret_cast<const u32x4*>(r + slot * Page::ROW + 16 * (2 * i + hf));
      b.kscale = NB == 4 ? *reinterpret_cast<const uint32_t*>(r + Page::CODES + slot * NB)
                         : *reinterpret_cast<const uint16_t*>(r + Page::CODES + slot * NB);
    }
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int piece = lane + 64 * i;
      const int j = min(kbase + piece / NB, last), slot = j % PAGE;
      const uint8_t* r = run(vpool_h, j);
      b.v[i] = *reinterpret_cast<const u32x4*>(r + slot * Page::ROW + 16 * (piece % NB));
      b.vscale[i] = r[Page::CODES + slot * NB + piece % NB];
    }
  };

  __bf16* const vs = reinterpret_cast<__bf16*>(smem + wave * VBYTES);
  const __bf16* vl[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
    vl[db] = vs + (4 * hf + (lane & 15) / 4) * VSTR + v_place(4 * db + 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1)) +
             4 * (lane & 1);
  f32x16 oacc[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db) oacc[db] = f32x16{};
  float m_run = -INFINITY, l_run = 0.0f;

  auto attend = [&](const Block& b, int block) {
    const int kbase = 32 * block;
    f32x16 s = f32x16{};
    const uint32_t scales = b.kscale >> (8 * hf);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const float a = scale_of((scales >> (16 * i)) & 255u);
#pragma unroll
      for (int u = 0; u < 4; ++u)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q4_values(b.k[i][u], a), qf[4 * i + u], s, 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int piece = lane + 64 * i;
      const float a = scale_of(b.vscale[i]);
      __bf16* row = vs + piece / NB * VSTR;
#pragma unroll
      for (int u = 0; u < 4; ++u) *reinterpret_cast<bf16x8*>(row + v_place(4 * (piece % NB) + u)) = q4_values(b.v[i][u], a);
    }
    // accumulator element r holds key 8*(r/4) + 4*hf + (r%4)
    if (kbase + 31 > min_lim || kbase + 32 > it.kv_end) {
      const int bound = min(limit, it.kv_end - 1) - kbase - 4 * hf;
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (8 * (r >> 2) + (r & 3) > bound) s[r] = -INFINITY;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[r]);
    mx = halves_max(mx) * sl2;
    const bool bump = mx > m_run + 8.0f;         // as in the kernel above
    const float m_new = bump ? mx : m_run;
    const float m_use = reference(m_new);
    float rs = 0.0f;
    bf16x8 pb[2];
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float e = fast_exp2(fmaf(s[r], sl2, -m_use));
      rs += e;
      pb[r >> 3][r & 7] = static_cast<__bf16>(e);
    }
    rs = halves_sum(rs);
    if (__any(bump)) {
      const float alpha = fast_exp2(m_run - m_use);
      l_run *= alpha;
#pragma unroll
      for (int db = 0; db < D / 32; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[db][r] *= alpha;
    }
    l_run += rs;
    m_run = m_new;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int db = 0; db < D / 32; ++db) {
        const bf16x4 lo = lds_read_tr(vl[db] + 16 * t * VSTR);
        const bf16x4 hi = lds_read_tr(vl[db] + (16 * t + 8) * VSTR);
        const bf16x8 a = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[t], oacc[db], 0, 0, 0);
      }
  };

  // Two blocks are in flight.  Loads are not branched around (a last block is loaded again instead), so the compiler
  // knows their number and waits for the older block alone (but for the form that spills, see above).
  const int end = (it.kv_end + 31) / 32;
  int block = it.kv_begin / 32 + wave;
  if (block < end) {
    Block b0, b1;
    load(b0, block);
    __builtin_amdgcn_sched_barrier(0);
    load(b1, min(block + 4, end - 1));
    for (;;) {
      attend(b0, block);
      load(b0, min(block + 8, end - 1));
      if (block + 4 >= end) break;
      attend(b1, block + 4);
      load(b1, min(block + 12, end - 1));
      block += 8;
      if (block >= end) break;
    }
  }

  // ---- the waves' sums joined -------------------------------------------------------------------
  if (hf == 0) {
    wave_m[wave][col] = m_run;
    wave_l[wave][col] = l_run;
  }
  __syncthreads();
  float m = -INFINITY;
#pragma unroll
  for (int w = 0; w < 4; ++w) m = fmaxf(m, wave_m[w][col]);
  const float mine = m_run == -INFINITY ? 0.0f : fast_exp2(m_run - m);
  float* const join = reinterpret_cast<float*>(smem);
  const int row = tid >> 3, c8 = 8 * (tid & 7);
  float rm_ = -INFINITY, l = 0.0f;
#pragma unroll
  for (int w = 0; w < 4; ++w) rm_ = fmaxf(rm_, wave_m[w][row]);
#pragma unroll
  for (int w = 0; w < 4; ++w) l += wave_l[w][row] == 0.0f ? 0.0f : wave_l[w][row] * fast_exp2(wave_m[w][row] - rm_);
  l = row_sum(rm_, l);
  const float inv_l = l == 0.0f ? 0.0f : 1.0f / l;
  const float lse_v = l == 0.0f ? -INFINITY : (rm_ + __log2f(l)) * kLn2;
  const int orow_t = it.row0 + row, otok = orow_t / G;
  const int64_t orow = int64_t(rm.cu + otok) * Hq + it.kv_head * G + (orow_t - otok * G);
#pragma unroll
  for (int half = 0; half < D / 64; ++half) {
    if (half) __syncthreads();                   // the sums before are read
#pragma unroll
    for (int db = 0; db < 2; ++db)
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        f32x4 v;
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = oacc[2 * half + db][4 * u + k] * mine;
        *reinterpret_cast<f32x4*>(join + (wave * 32 + col) * OSTR + 32 * db + 8 * u + 4 * hf) = v;
      }
    __syncthreads();
    if (row < it.rows) {
      f32x4 a = f32x4{}, b = f32x4{};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        a += *reinterpret_cast<const f32x4*>(join + (w * 32 + row) * OSTR + c8);
        b += *reinterpret_cast<const f32x4*>(join + (w * 32 + row) * OSTR + c8 + 4);
      }
      a *= inv_l;
      b *= inv_l;
      if (it.part < 0) {
        bf16x8 o;
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = static_cast<__bf16>(a[k]), o[4 + k] = static_cast<__bf16>(b[k]);
        *reinterpret_cast<bf16x8*>(out + orow * D + 64 * half + c8) = o;
      } else {
        float* to = p.opart + int64_t(it.part + row) * D + 64 * half + c8;
        *reinterpret_cast<f32x4*>(to) = a;
        *reinterpret_cast<f32x4*>(to + 4) = b;
      }
    }
  }
  if (row < it.rows && c8 == 0) {
    if (it.part >= 0) p.lpart[it.part + row] = lse_v;
    else if (lse_out) lse_out[orow] = lse_v;
  }
}

// Launch shape of the append and the read: a token per workgroup in waves that do not fill the chip, four beyond, whose
// rows are all loaded first (16,384 tokens of 8 heads of 128, stored and read back from cold memory: 49 us one by one, 44 with
// two, 43 with four, 47 with eight).
struct Moves {
  bool few;
  int64_t blocks;
  int threads;
  explicit Moves(const DevPlan& p)
      : few(p.total_tokens <= 2048),
        blocks(((few ? p.total_tokens : (p.total_tokens + 3) / 4) + kNumXcd - 1) / kNumXcd * kNumXcd),
        threads(std::min(256, (p.num_kv_heads * p.head_dim_qk / 4 + 63) / 64 * 64)) {}
};

}  // namespace

// ---------------------------------------------------------------------------------------------
// Launchers
// ---------------------------------------------------------------------------------------------
hipError_t launch_q4_append(const DevPlan& p, const void* k_new, const void* v_new, void* k_pool, void* v_pool,
                            hipStream_t stream) {
  const Moves g(p);
  if (g.blocks >= 1 << 24) return hipErrorInvalidValue;
  auto kn = static_cast<const u32x4*>(k_new);
  auto vn = static_cast<const u32x4*>(v_new);
  auto kp = static_cast<uint8_t*>(k_pool);
  auto vp = static_cast<uint8_t*>(v_pool);
#define WAVEPP_Q4_MOVE(D_)                                                                                            \
  if (g.few) hipLaunchKernelGGL((q4_append_kernel<D_, 1>), dim3(g.blocks), dim3(g.threads), 0, stream, p, kn, vn, kp, vp);  \
  else hipLaunchKernelGGL((q4_append_kernel<D_, 4>), dim3(g.blocks), dim3(g.threads), 0, stream, p, kn, vn, kp, vp);
  if (p.head_dim_qk == 128) {
    WAVEPP_Q4_MOVE(128)
  } else if (p.head_dim_qk == 64) {
    WAVEPP_Q4_MOVE(64)
  } else {
    return hipErrorInvalidValue;
  }
#undef WAVEPP_Q4_MOVE
  return hipGetLastError();
}

hipError_t launch_q4_read(const DevPlan& p, const void* k_pool, const void* v_pool, void* k_out, void* v_out,
                          hipStream_t stream) {
  const Moves g(p);
  if (g.blocks >= 1 << 24) return hipErrorInvalidValue;
  auto kp = static_cast<const uint8_t*>(k_pool);
  auto vp = static_cast<const uint8_t*>(v_pool);
  auto ko = static_cast<bf16x8*>(k_out);
  auto vo = static_cast<bf16x8*>(v_out);
#define WAVEPP_Q4_MOVE(D_)                                                                                          \
  if (g.few) hipLaunchKernelGGL((q4_read_kernel<D_, 1>), dim3(g.blocks), dim3(g.threads), 0, stream, p, kp, vp, ko, vo);  \
  else hipLaunchKernelGGL((q4_read_kernel<D_, 4>), dim3(g.blocks), dim3(g.threads), 0, stream, p, kp, vp, ko, vo);
  if (p.head_dim_qk == 128) {
    WAVEPP_Q4_MOVE(128)
  } else if (p.head_dim_qk == 64) {
    WAVEPP_Q4_MOVE(64)
  } else {
    return hipErrorInvalidValue;
  }
#undef WAVEPP_Q4_MOVE
  return hipGetLastError();
}

hipError_t launch_q4_attention(const DevPlan& p, int32_t num_few, const void* q, const void* k_pool, const void* v_pool,
                               void* out, float* lse, hipStream_t stream) {
  if (p.num_items == 0) return hipSuccess;
  auto qq = static_cast<const __bf16*>(q);
  auto kp = static_cast<const uint8_t*>(k_pool);
  auto vp = static_cast<const uint8_t*>(v_pool);
  auto oo = static_cast<__bf16*>(out);
  const int32_t num_many = p.num_items - num_few;
  const bool w8 = p.rows_per_item == kGqaRowsPerItem;
  if (num_many && !w8 && p.rows_per_item != kGqaRowsPerItem / 2) return hipErrorInvalidValue;
  DevPlan few = p;
  few.items += num_many;
#define WAVEPP_Q4(D_, P_)                                                                                             \
  if (num_many && w8)                                                                                                 \
    hipLaunchKernelGGL((attn_q4_kernel<D_, P_, 8>), dim3(num_many), dim3(512), 0, stream, p, qq, kp, vp, oo, lse);     \
  else if (num_many)                                                                                                  \
    hipLaunchKernelGGL((attn_q4_kernel<D_, P_, 4>), dim3(num_many), dim3(256), 0, stream, p, qq, kp, vp, oo, lse);     \
  if (num_few)                                                                                                        \
    hipLaunchKernelGGL((attn_q4_few_kernel<D_, P_>), dim3(num_few), dim3(256), 0, stream, few, qq, kp, vp, oo, lse);
  if (p.head_dim_qk == 128 && p.page_size == 64) {
    WAVEPP_Q4(128, 64)
  } else if (p.head_dim_qk == 128 && p.page_size == 16) {
    WAVEPP_Q4(128, 16)
  } else if (p.head_dim_qk == 64 && p.page_size == 64) {
    WAVEPP_Q4(64, 64)
  } else if (p.head_dim_qk == 64 && p.page_size == 16) {
    WAVEPP_Q4(64, 16)
  } else {
    return hipErrorInvalidValue;
  }
#undef WAVEPP_Q4
  return hipGetLastError();
}

}  // namespace wavepp
