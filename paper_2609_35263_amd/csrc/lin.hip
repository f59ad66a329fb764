// gfx950 (CDNA4) kernels of libwavepp_attn: linear attention with a decay for each head,
//   S_t = alpha_t S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t,
// token by token for short chunks and in blocks of 64 tokens for longer ones.
//
// Blocks.  With S0 the state before a block, lam_i = alpha_1 ... alpha_i and D[i][j] = alpha_{j+1} ... alpha_i (j <= i, 0 above
// the diagonal), its outputs and its last state are
//   O = scale (diag(lam) Q S0 + ((Q K^T) * D) V),      S = lam_64 S0 + K^T diag(D[64][.]) V.
// All factors are products of decays, never quotients, so a decay of zero (or a tiny one) needs no special case.
//
// A workgroup runs one segment of one (request, head), or of two heads, block after block; wave w of a head owns its state's
// columns 16 w .. 16 w + 15 as 16 x 16 fp32 accumulator tiles.  The accumulator layout of v_mfma_f32_16x16x32_bf16 (lane =
// column, four rows a lane) is that of an operand whose contraction runs over the rows of two tiles in a permuted
// order, so the state feeds O^T = S0^T Q^T from registers, Q rows being read from LDS in that order; V and K^T
// are read by transposing LDS reads.  The ten 16 x 16 tiles of (Q K^T) * D on and under the diagonal are shared out over
// the waves and go through LDS.  The next block's rows are loaded while a block is worked on.
//
// What bounds it.  A block of 128 + 128 columns is 64 KiB of memory traffic, 3.4 us of a CU's share of a copy's rate; a
// block's work is a chain of LDS reads, products and a barrier of about 3.1 us.  4 x 4,096 tokens, 64 heads of 128 x 128, one
// workgroup on each of 256 CUs: 271 us, 4.1 TB/s where a large copy reaches 4.75 (232 us); 244 us without the products, 200
// without the memory.  Measured on the way there (same wave): four waves of 32 columns that keep the logits in registers
// 1,092 us (spills); eight of 16 with P in LDS 355; one barrier a block in place of three 325; Q and P in operand order, K's
// pieces swapped 289 (the first bank conflicts took half the LDS's cycles); loads without branches 278; P before the rest
// 269.  Not kept: two blocks of rows on their way (297: the registers spill), two workgroups of 64 columns a CU (352
// against 289 then), the move of the next block to LDS first in a block (298), stores past the caches (361).
#include <hip/hip_runtime.h>

#include "device.h"
#include "lin.h"

#include <algorithm>

namespace wavepp {
namespace {

typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

constexpr int kC = kLinBlock;

__device__ __forceinline__ bool lin_meta_ok(const LinDevPlan& p) {
  return p.hdr->magic == kLinMagic && p.hdr->serial == p.serial;
}

__device__ __forceinline__ bf16x8 cat(bf16x4 a, bf16x4 b) {
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

__device__ __forceinline__ f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Two accumulator tiles in bf16: an operand whose contraction runs over their 32 rows, slot e of lane group g being
// row 4 g + e of the first and 4 g + e - 4 of the second.
__device__ __forceinline__ bf16x8 acc_operand(const f32x4& a, const f32x4& b) {
  bf16x8 r;
#pragma unroll
  for (int e = 0; e < 4; ++e) r[e] = static_cast<__bf16>(a[e]), r[4 + e] = static_cast<__bf16>(b[e]);
  return r;
}

// Two fp32 values as three bf16 each, 8 bits of the value a part: word u of the parts' operands.  Cutting off instead of
// rounding costs an instruction less a value and leaves the last part exact.
__device__ __forceinline__ void split_pair(float x0, float x1, int u, u32x4& hi, u32x4& mid, u32x4& lo) {
  auto upper = [](float a, float b) { return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302); };
  auto rest = [](float a) { return a - __uint_as_float(__float_as_uint(a) & 0xFFFF0000u); };
  const float y0 = rest(x0), y1 = rest(x1);
  hi[u] = upper(x0, x1);
  mid[u] = upper(y0, y1);
  lo[u] = upper(rest(y0), rest(y1));
}

// The value of another lane of the same 16; where there is none, 1.
template <int CTRL>
__device__ __forceinline__ float row_or_one(float x) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0x3F800000, __float_as_uint(x), CTRL, 0xF, 0xF, false));
}
constexpr int kRowShl = 0x100, kRowShr = 0x110, kRowBcast = 0x150;   // + distance, or the lane broadcast

// Products of x over this lane and those before it in its 16 lanes.
__device__ __forceinline__ float row_products(float x) {
  x *= row_or_one<kRowShr + 1>(x);
  x *= row_or_one<kRowShr + 2>(x);
  x *= row_or_one<kRowShr + 4>(x);
  x *= row_or_one<kRowShr + 8>(x);
  return x;
}
// The same over the lanes after it.
__device__ __forceinline__ float row_products_after(float x) {
  x = row_or_one<kRowShl + 1>(x);
  x *= row_or_one<kRowShl + 1>(x);
  x *= row_or_one<kRowShl + 2>(x);
  x *= row_or_one<kRowShl + 4>(x);
  x *= row_or_one<kRowShl + 8>(x);
  return x;
}

// Row l of a lower-triangular 16 x 16 table in lane l of each 16: d[j] = a[j + 1] ... a[l], 1 at j = l, 0 above.
template <int J = 15>
__device__ __forceinline__ void row_table(float a, int l, float x, float (&d)[16]) {
  if constexpr (J < 15) x *= row_or_one<kRowBcast + J + 1>(a);
  if (l == J) x = 1.0f;
  d[J] = l < J ? 0.0f : x;
  if constexpr (J > 0) row_table<J - 1>(a, l, x, d);
}

// A buffer descriptor of `bytes` from a uniform address: loads behind them give zero, stores behind them do nothing.
template <typename T>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t block_rows(const T* base, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(base), 0, bytes, 0x00027000);
}

// An item by scalar loads (the kernels never write the metadata), so that the compiler knows it is uniform.
__device__ __forceinline__ LinItem item_at(const LinItem* at) {
  const u32x4* words = reinterpret_cast<const u32x4*>(at);
  struct Halves { u32x4 a, b; } x = {const_load(words), const_load(words + 1)};
  return __builtin_bit_cast(LinItem, x);
}

// Where a segment starts: a partial state, a snapshot, or nothing.
__device__ __forceinline__ const float* start_of(const LinDevPlan& p, const LinItem& it, const float* pool, int head) {
  const int64_t size = int64_t(p.head_dim_k) * p.head_dim_v;
  if (it.part_in >= 0) return p.parts + (int64_t(it.part_in) * p.num_heads + head) * size;
  if (it.state_in >= 0) return pool + (int64_t(it.state_in) * p.num_heads + head) * size;
  return nullptr;
}

// ---------------------------------------------------------------------------------------------
// Blocks of 64 tokens.  AHEAD: only the segment's own state, from zero, and its decay.  A workgroup has 128 columns: a head's,
// or those of two heads of 64 that share q and k (HP = 2), whose rows of v and out lie side by side and whose Q K^T is one
// product with two tables of decays (three ragged prompts, 32/8 heads of 128 x 64: 132 -> 124 us, 119 -> 118 with the inputs
// in a cache).  Two blocks lie in LDS then, one workgroup of eight waves a CU; heads of 64 by themselves have one block and two
// workgroups of four waves (207 -> 170 us on those prompts when it came in).
// ---------------------------------------------------------------------------------------------
template <int DK, int DV, int HP, bool AHEAD>
__global__ __launch_bounds__(DV * HP * 4, AHEAD && DV * HP == 128 ? 4 : 2) void lin_blocks_kernel(
    LinDevPlan p, const __bf16* __restrict__ q, const __bf16* __restrict__ k, const __bf16* __restrict__ v,
    const float* __restrict__ alpha, float* pool, __bf16* __restrict__ out) {
  constexpr int COLS = DV * HP, NW = COLS / 16, NT = NW * 64;    // columns of the workgroup's heads, side by side
  // LDS layouts, for its 64 banks.  Q's and P's rows keep each 32 of their columns in the order of an operand's slots
  // (4-column group u of eight at place 2 (u % 4) + u / 4), so one 16-byte read gives an operand, eight rows on distinct
  // banks.  K, V: transposed reads of 8 rows x 32 bytes on distinct banks.  K's rows with bit 3 set have neighbouring
  // 16-byte pieces swapped, which puts the 8-byte reads of 16 rows on distinct banks too.
  constexpr int QS = DK + 8, KS = DK + 16, VS = COLS + 16, PS = kC + 8;
  constexpr int KL = kC * DK / 8 / NT, VL = kC * COLS / 8 / NT;   // 16-byte pieces per thread and block
  constexpr int CT = DK / 16;                                     // row tiles of the state
  constexpr int BUF = COLS == 128 ? 2 : 1;                        // blocks in LDS
  constexpr int DT = 160;                                         // a tile of D on the diagonal
  struct alignas(16) Decays {
    float run[3][kC];                  // [u][i]: alpha_{16 (u + 1)} ... alpha_i
    float lam[kC];                     // scale alpha_0 ... alpha_i
    float rest[kC], wt[kC];            // alpha after j: in its 16 times scale, in the block
    float diag[AHEAD ? 4 : 4 * DT];    // D's 16 x 16 tiles on the diagonal, times scale, see diag_at
  };
  struct alignas(16) Block {
    __bf16 q[AHEAD ? 8 : kC * QS];
    __bf16 k[kC * KS];
    __bf16 v[kC * VS];
    Decays d[HP];
    float gamma[HP];                   // the block's decay
    int bad[NW];                       // per wave, bit h: a value of V of head h is not finite
  };
  __shared__ __attribute__((aligned(16))) Block blk[BUF];
  __shared__ __attribute__((aligned(16))) __bf16 pm[2][HP][AHEAD ? 8 : kC * PS];   // scale (Q K^T) * D
  // Where four columns of row l of a diagonal tile lie: only the quads that reach the diagonal are kept.
  auto diag_at = [](int l, int quad) { return 4 * (2 * (l / 4) * (l / 4 + 1) + l % 4 * (l / 4 + 1) + quad); };

  if (!lin_meta_ok(p)) return;
  const int H = p.num_heads, Hqk = p.num_qk_heads;
  // Workgroups go round-robin to the kNumXcd L2 domains: the heads that share a q/k head read its rows through one.
  const int G = H / Hqk / HP, unit = blockIdx.x / (kNumXcd * G) * kNumXcd + blockIdx.x % kNumXcd;
  if (unit >= (AHEAD ? p.num_ahead : p.num_segments) * Hqk) return;
  const LinItem it = item_at(p.segments + unit / Hqk);
  const int qk_head = unit % Hqk, first = (qk_head * G + blockIdx.x / kNumXcd % G) * HP;
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int mine = HP == 1 ? 0 : wave / (DV / 16), part = HP == 1 ? wave : wave % (DV / 16);   // of the heads; of the head
  const int head = first + mine, col = 16 * part + l16;

  f32x4 S[CT];                           // tile c, lane: rows 16 c + 4 g .. + 3 of column col
#pragma unroll
  for (int c = 0; c < CT; ++c) S[c] = f32x4{};
  if (!AHEAD) {
    if (const float* s0 = start_of(p, it, pool, head)) {
#pragma unroll
      for (int c = 0; c < CT; ++c)
#pragma unroll
        for (int r = 0; r < 4; ++r) S[c][r] = s0[(16 * c + 4 * g + r) * DV + col];
    }
    // the tiles above the diagonal that the products with V run over
    for (int i = tid; i < 2 * HP * 32 * 16; i += NT) {
      const int u = i % 512;
      const int at = (u / 256 * 32 + u / 16 % 16) * PS + u / 256 * 32 + u / 4 % 4 * 8 + 4 + u % 4;
      pm[i / 512 % 2][i / 1024][AHEAD ? 0 : at] = __bf16(0.0f);
    }
  }

  struct Rows {                          // a block on its way from memory
    u32x4 q[AHEAD ? 1 : KL], k[KL], v[VL];
    float a;
  };
  // Byte offsets of this thread's pieces in a block.  Loads and stores go through buffer descriptors that end with the
  // segment's last token: what lies behind reads as zero and is not written, and there is no branch around them, so the
  // compiler knows how many are in flight and waits for the oldest block alone.
  uint32_t qk_off[KL], v_off[VL];
#pragma unroll
  for (int i = 0; i < KL; ++i) {
    const int c = tid + NT * i;
    qk_off[i] = uint32_t(c / (DK / 8) * Hqk * DK + c % (DK / 8) * 8) * 2;
  }
#pragma unroll
  for (int i = 0; i < VL; ++i) {
    const int c = tid + NT * i;
    v_off[i] = uint32_t(c / (COLS / 8) * H * DV + c % (COLS / 8) * 8) * 2;
  }
  const uint32_t a_row = p.alpha_per_token ? uint32_t(H) * 4 : 0;
  auto load = [&](Rows& x, int t0) {
    const int rows = __builtin_amdgcn_readfirstlane(max(0, min(kC, it.len - t0)));
    const int64_t tok = it.cu + min(t0, it.len);
    const auto qb = block_rows(q + (tok * Hqk + qk_head) * DK, rows * uint32_t(Hqk * DK * 2));
    const auto kb = block_rows(k + (tok * Hqk + qk_head) * DK, rows * uint32_t(Hqk * DK * 2));
    const auto vb = block_rows(v + (tok * H + first) * DV, rows * uint32_t(H * DV * 2));
    const auto ab = block_rows(alpha + (p.alpha_per_token ? tok * H + head : head), p.alpha_per_token ? rows * a_row : 4);
#pragma unroll
    for (int i = 0; i < KL; ++i) {
      if (!AHEAD) x.q[AHEAD ? 0 : i] = __builtin_amdgcn_raw_buffer_load_b128(qb, qk_off[i], 0, 0);
      x.k[i] = __builtin_amdgcn_raw_buffer_load_b128(kb, qk_off[i], 0, 0);
    }
#pragma unroll
    for (int i = 0; i < VL; ++i) x.v[i] = __builtin_amdgcn_raw_buffer_load_b128(vb, v_off[i], 0, 0);
    x.a = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(ab, lane * a_row, 0, 0));
  };
  float total = 1.0f;                    // AHEAD: the segment's decay so far
  // The loaded rows to LDS, and the products of their decays: every wave has the 64 in its lanes, four make a part each.
  auto store = [&](Block& b, const Rows& rows, int t0) {
    u16x2 top = u16x2{0, 0};
#pragma unroll
    for (int i = 0; i < KL; ++i) {
      const int c = tid + NT * i, row = c / (DK / 8), at = c % (DK / 8) * 8;
      if (!AHEAD) {
        const int u = at / 8 % 4;                          // 4-column groups 2 u and 2 u + 1 of their 32 columns
        __bf16* to = &b.q[AHEAD ? 0 : row * QS + at / 32 * 32 + u % 2 * 16 + u / 2 * 4];
        const u32x4 x = rows.q[AHEAD ? 0 : i];
        *reinterpret_cast<u32x2*>(to) = u32x2{x[0], x[1]};
        *reinterpret_cast<u32x2*>(to + 8) = u32x2{x[2], x[3]};
      }
      *reinterpret_cast<u32x4*>(&b.k[row * KS + (at ^ (row & 8))]) = rows.k[i];
    }
#pragma unroll
    for (int i = 0; i < VL; ++i) {
      const int c = tid + NT * i, row = c / (COLS / 8), at = c % (COLS / 8) * 8;
      *reinterpret_cast<u32x4*>(&b.v[row * VS + at]) = rows.v[i];
#pragma unroll
      for (int u = 0; u < 4; ++u) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, rows.v[i][u] & 0x7FFF7FFFu));
    }
    if (!AHEAD) {
      const uint64_t bad = __ballot(max(top[0], top[1]) >= 0x7F80);      // of two heads, each second eight lanes have one
      const uint64_t one = HP == 1 ? ~uint64_t(0) : 0x00FF00FF00FF00FFull;
      if (lane == 0) b.bad[wave] = int((bad & one) != 0) | int((bad & ~one) != 0) << 1;
    }
    const float a = t0 + lane < it.len ? rows.a : 1.0f;    // no decay behind the last token
    if (part < 4) {
      Decays& d = b.d[mine];
      const float x = row_products(a);
      const float x0 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), 15));
      const float x1 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), 31));
      const float x2 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), 47));
      const float x3 = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), 63));
      float before = 1.0f;
      if (g > 0 && part <= 0) before *= x0;
      if (g > 1 && part <= 1) before *= x1;
      if (g > 2 && part <= 2) before *= x2;
      if (part > 0) d.run[part - 1][lane] = before * x;
      else d.lam[lane] = before * x * p.scale;
      const float all = x0 * x1 * x2 * x3;
      total *= all;
      if (part == 0 && lane == 0) b.gamma[mine] = all;
      if (part == 1) {
        const float y = row_products_after(a);
        d.rest[lane] = y * p.scale;
        float after = 1.0f;
        if (g < 3) after *= x3;
        if (g < 2) after *= x2;
        if (g < 1) after *= x1;
        d.wt[lane] = y * after;
      }
      if (!AHEAD && part == 2) {
        float row[16];
        row_table(a, l16, 0.0f, row);
#pragma unroll
        for (int u = 0; u < 4; ++u)
          if (4 * u <= l16)
            *reinterpret_cast<f32x4*>(&d.diag[AHEAD ? 0 : DT * g + diag_at(l16, u)]) =
                f32x4{row[4 * u], row[4 * u + 1], row[4 * u + 2], row[4 * u + 3]} * p.scale;
      }
    }
  };
  auto operand = [&](const __bf16* m, int at) { return *reinterpret_cast<const bf16x8*>(m + at); };

  // What a block leaves for the step after it: its part of O, and V^T of this wave's columns (slot e of lane group g is
  // token 32 t + 4 g + e, or 16 + 4 g + e - 4 from the fifth on).
  f32x4 o[4];                            // O^T: columns' rows 4 g .. + 3 of tokens 16 i + l16
  bf16x8 vf[2];
  const uint32_t o_off = uint32_t(l16 * H * DV + 16 * wave + 4 * g) * 2;
  auto put = [&](int t0) {
    const int rows = __builtin_amdgcn_readfirstlane(min(kC, it.len - t0));
    const auto ob = block_rows(out + (int64_t(it.cu + t0) * H + first) * DV, rows * uint32_t(H * DV * 2));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      bf16x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = static_cast<__bf16>(o[i][e]);
      __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(u32x2, x), ob, o_off + 16 * i * uint32_t(H * DV * 2), 0, 0);
    }
  };
  auto finish = [&](const __bf16* pb, int t0) {            // O += P V, and out
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t <= i / 2; ++t) o[i] = mfma(vf[t], operand(pb, (16 * i + l16) * PS + 32 * t + 8 * g), o[i]);
    put(t0);
  };

  // Between two barriers a wave finishes the block before (whose P is whole by then), works on the present one, moves the
  // next one from its registers to LDS and asks for the one after.  With two buffers that is one barrier a block; one
  // buffer takes another before the move, and leaves room for a second workgroup.
  Rows rows;
  load(rows, 0);
  store(blk[0], rows, 0);
  load(rows, kC);
  __syncthreads();
  bool pending = false;
  for (int t0 = 0, half = 0; t0 < it.len; t0 += kC, half ^= 1) {
    const Block& b = blk[half % BUF];
    if constexpr (!AHEAD) {
      for (int tile = wave; tile < 10; tile += NW) {       // (queries ti, keys tj), ti >= tj
        const int ti = tile < 1 ? 0 : tile < 3 ? 1 : tile < 6 ? 2 : 3, tj = tile - ti * (ti + 1) / 2;
        f32x4 x = f32x4{};                                 // K Q^T: keys 4 g .. + 3 of query l16
#pragma unroll
        for (int s = 0; s < CT / 2; ++s) {
          const __bf16* kr = &b.k[(16 * tj + l16) * KS + 32 * s + ((4 * g) ^ (l16 & 8))];
          x = mfma(cat(*reinterpret_cast<const bf16x4*>(kr), *reinterpret_cast<const bf16x4*>(kr + 16)),
                   operand(b.q, (16 * ti + l16) * QS + 32 * s + 8 * g), x);
        }
#pragma unroll
        for (int h = 0; h < HP; ++h) {
          bf16x4 y;
          if (ti == tj) {                                  // above the diagonal nothing, whatever the product was
            const f32x4 d = *reinterpret_cast<const f32x4*>(&b.d[h].diag[DT * ti + diag_at(l16, min(g, l16 / 4))]);
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = static_cast<__bf16>(4 * g + e <= l16 ? x[e] * d[e] : 0.0f);
          } else {
            const f32x4 d = *reinterpret_cast<const f32x4*>(&b.d[h].rest[16 * tj + 4 * g]);
            const float w = b.d[h].run[tj][16 * ti + l16];
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = static_cast<__bf16>(x[e] * (d[e] * w));
          }
          *reinterpret_cast<bf16x4*>(&pm[half][h][(16 * ti + l16) * PS + tj / 2 * 32 + 8 * g + tj % 2 * 4]) = y;
        }
      }
    }
    if (pending) finish(pm[half ^ 1][mine], t0 - kC);
    if constexpr (!AHEAD) {
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = f32x4{};
#pragma unroll
      for (int s = 0; s < CT / 2; ++s) {
        const bf16x8 st = acc_operand(S[2 * s], S[2 * s + 1]);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = mfma(st, operand(b.q, (16 * i + l16) * QS + 32 * s + 8 * g), o[i]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float l = b.d[mine].lam[16 * i + l16];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][e] *= l;
      }
    }

    const __bf16* vl = &b.v[(4 * g + (l16 >> 2)) * VS + 16 * wave + 4 * (l16 & 3)];
#pragma unroll
    for (int t = 0; t < 2; ++t) vf[t] = cat(lds_read_tr(vl + 32 * t * VS), lds_read_tr(vl + (32 * t + 16) * VS));
    // S = lam_64 S + K^T (w V): the weighted values as three bf16 parts, 24 bits, so that the state is as exact as in fp32
    const float gamma = b.gamma[mine];
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int r = 0; r < 4; ++r) S[c][r] *= gamma;
    const __bf16* kl = &b.k[(4 * g + (l16 >> 2)) * KS + ((4 * (l16 & 3)) ^ (4 * g & 8))];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const f32x4 w0 = *reinterpret_cast<const f32x4*>(&b.d[mine].wt[32 * t + 4 * g]);
      const f32x4 w1 = *reinterpret_cast<const f32x4*>(&b.d[mine].wt[32 * t + 16 + 4 * g]);
      u32x4 hi, mid, lo;
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const f32x4 w = u < 2 ? w0 : w1;
        split_pair(float(vf[t][2 * u]) * w[2 * u & 3], float(vf[t][2 * u + 1]) * w[(2 * u + 1) & 3], u, hi, mid, lo);
      }
      // part by part: no product waits for the sum of the one before it
      bf16x8 kt[CT];
#pragma unroll
      for (int c = 0; c < CT; ++c)
        kt[c] = cat(lds_read_tr(kl + 32 * t * KS + 16 * c), lds_read_tr(kl + (32 * t + 16) * KS + 16 * c));
#pragma unroll
      for (int c = 0; c < CT; ++c) S[c] = mfma(kt[c], __builtin_bit_cast(bf16x8, hi), S[c]);
#pragma unroll
      for (int c = 0; c < CT; ++c) S[c] = mfma(kt[c], __builtin_bit_cast(bf16x8, mid), S[c]);
#pragma unroll
      for (int c = 0; c < CT; ++c) S[c] = mfma(kt[c], __builtin_bit_cast(bf16x8, lo), S[c]);
    }
    pending = !AHEAD;
    if constexpr (!AHEAD) {
      int any = 0;
#pragma unroll
      for (int w = 0; w < NW; ++w) any |= b.bad[w];
      // A value of V that is not finite, times the zeros above the diagonal, would reach the tokens before it: such a
      // block's weights and values are summed pair by pair.
      any = __builtin_amdgcn_readfirstlane(any);
      if (any) __syncthreads();          // P is whole
      if (any >> mine & 1) {
        for (int j = 0; j < kC; ++j) {
          const bf16x4 x = *reinterpret_cast<const bf16x4*>(&b.v[j * VS + 16 * wave + 4 * g]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float w = float(pm[half][mine][(16 * i + l16) * PS + j / 32 * 32 + j / 4 % 4 * 8 + j / 16 % 2 * 4 + j % 4]);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][e] = j <= 16 * i + l16 ? fmaf(w, float(x[e]), o[i][e]) : o[i][e];
          }
        }
        put(t0);
        pending = false;
      }
    }
    if (BUF == 1) __syncthreads();
    store(blk[(half ^ 1) % BUF], rows, t0 + kC);
    load(rows, t0 + 2 * kC);
    __syncthreads();
  }
  if (pending) {
    const int blocks = (it.len + kC - 1) / kC;
    finish(pm[(blocks - 1) & 1][mine], (blocks - 1) * kC);
  }

  const int64_t size = int64_t(DK) * DV;
  float* to = AHEAD ? p.parts + (int64_t(it.part_out) * H + head) * size
                    : it.state_out >= 0 ? pool + (int64_t(it.state_out) * H + head) * size : nullptr;
  if (to) {
#pragma unroll
    for (int c = 0; c < CT; ++c)
#pragma unroll
      for (int r = 0; r < 4; ++r) to[(16 * c + 4 * g + r) * DV + col] = S[c][r];
  }
  if (AHEAD && part == 0 && lane == 0) p.part_decay[int64_t(it.part_out) * H + head] = total;
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
// column quad).  The outputs' sums over the rows are joined in LDS.  A token each of 128 requests, 64 heads of 128 x 128, is
// 1.08 GB of states read and written: 215 us, 5.0 TB/s, above a large copy's rate.  Few chains make up for their number by
// the four workgroups that share a state (4 requests, 32 heads of 128 x 64: 4 us).
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
  const LinItem it = item_at(p.steps + blockIdx.x / (DV / W) / H);
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

template <int DK, int DV, int HP>
void launch_blocks(const LinDevPlan& p, const __bf16* q, const __bf16* k, const __bf16* v, const float* alpha, float* pool,
                   __bf16* out, hipStream_t stream) {
  // a workgroup for every segment and HP heads, the segments' q/k heads padded to whole rounds of the L2 domains
  auto grid = [&](int segments) {
    return dim3((segments * p.num_qk_heads + kNumXcd - 1) / kNumXcd * kNumXcd * (p.num_heads / p.num_qk_heads / HP));
  };
  if (p.num_ahead)
    hipLaunchKernelGGL((lin_blocks_kernel<DK, DV, HP, true>), grid(p.num_ahead), dim3(4 * DV * HP), 0, stream, p, q, k, v,
                       alpha, pool, out);
  if (p.num_scans)
    hipLaunchKernelGGL(lin_scan_kernel, dim3(p.num_scans * p.num_heads, DK * DV / 1024), dim3(256), 0, stream, p, pool);
  if (p.num_segments)
    hipLaunchKernelGGL((lin_blocks_kernel<DK, DV, HP, false>), grid(p.num_segments), dim3(4 * DV * HP), 0, stream, p, q, k,
                       v, alpha, pool, out);
}

template <int DK, int DV>
hipError_t launch_dims(const LinDevPlan& p, const __bf16* q, const __bf16* k, const __bf16* v, const float* alpha,
                       float* pool, __bf16* out, hipStream_t stream) {
  if (p.num_steps)
    hipLaunchKernelGGL((lin_step_kernel<DK, DV>), dim3(p.num_steps * p.num_heads * (DV / 32)), dim3(256), 0, stream, p, q, k,
                       v, alpha, pool, out);
  if (DV == 64 && lin_heads(p.num_heads, p.num_qk_heads, DV) == 2)
    launch_blocks<DK, DV, DV == 64 ? 2 : 1>(p, q, k, v, alpha, pool, out, stream);
  else
    launch_blocks<DK, DV, 1>(p, q, k, v, alpha, pool, out, stream);
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
