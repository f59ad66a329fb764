// gfx950 (CDNA4) kernels of libwavepp_attn's 8-bit paged cache: the append that rounds, the way back to bf16 rows, and
// grouped-query attention over 8-bit pages.
//
// A value is an e4m3 code times the power of two 2^(e - 127) of its block of 16 tokens of one head, so it is exactly a bf16
// number and the attention multiplies bf16 operands that equal the cached values: nothing is lost after the append.
// gfx950 turns two codes into two scaled bf16 with one instruction (v_cvt_scalef32_pk_bf16_fp8).
#include <hip/hip_runtime.h>

#include "device.h"
#include "q8.h"

#include <algorithm>

namespace wavepp {
namespace {

typedef short i16x2 __attribute__((ext_vector_type(2)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

constexpr uint32_t kLargest = 0x7F60u;       // 1.75 * 2^127: the largest magnitude that a code and a scale of 246 hold

__device__ __forceinline__ float scale_of(uint32_t byte) { return __uint_as_float(byte << 23); }

// The eight values of two words of codes.
__device__ __forceinline__ bf16x8 q8_values(uint32_t lo, uint32_t hi, float s_lo, float s_hi) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s_lo, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, s_lo, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s_hi, false);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, s_hi, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The codes of eight bf16 numbers, in two words; their magnitudes over the scale are at most 448.  (A bit cast straight from
// a vector's element takes its first element, whichever is named.)
__device__ __forceinline__ u32x2 q8_codes(u32x4 y, float s) {
  const uint32_t w[4] = {y[0], y[1], y[2], y[3]};
  i16x2 lo = {0, 0}, hi = {0, 0};
  lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, __builtin_bit_cast(bf16x2, w[0]), s, false);
  lo = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(lo, __builtin_bit_cast(bf16x2, w[1]), s, true);
  hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, __builtin_bit_cast(bf16x2, w[2]), s, false);
  hi = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(hi, __builtin_bit_cast(bf16x2, w[3]), s, true);
  return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
}

// The wave's largest value (MAX) or smallest, on all lanes: within 16 lanes by lane moves, the four rows by the scalar unit.
template <bool MAX, int CTRL, typename T>
__device__ __forceinline__ T more_moved(T x) {
  const T y = T(__builtin_amdgcn_update_dpp(0, int(x), CTRL, 0xF, 0xF, true));
  return MAX ? max(x, y) : min(x, y);
}
template <bool MAX, typename T>
__device__ __forceinline__ T wave_most(T x) {
  x = more_moved<MAX, 0xB1>(x);              // lanes 1, 0, 3, 2 of each four
  x = more_moved<MAX, 0x4E>(x);              // lanes 2, 3, 0, 1
  x = more_moved<MAX, 0x141>(x);             // the other four of each eight, mirrored
  x = more_moved<MAX, 0x140>(x);             // the other eight of each row of 16, mirrored
  const T a = T(__builtin_amdgcn_readlane(x, 0)), b = T(__builtin_amdgcn_readlane(x, 16));
  const T c = T(__builtin_amdgcn_readlane(x, 32)), d = T(__builtin_amdgcn_readlane(x, 48));
  return MAX ? max(max(a, b), max(c, d)) : min(min(a, b), min(c, d));
}

// ---------------------------------------------------------------------------------------------
// Append and read.  A wave has one block of 16 slots of one head, of K or of V: all of its rows lie in registers, eight
// values a lane, so the block's scale is found and applied in one pass.  A workgroup has four blocks in a row of the same
// head, so mostly a page's, whose run it writes in one piece.  Bound by memory: 16,384 tokens of 8 heads of 128 from cold memory
// take 20.6 us stored and 17.4 read back, 4.8 and 5.7 TB/s where a large copy reaches 4.8; 64 single tokens 3.3 and 3.4,
// a launch.  The rows to store are read past the caches, as nothing reads them again: 24 us with the events around it for 29.
// (Stores past the caches make the next read of the codes wait: the read back 29 us for 20.)
// ---------------------------------------------------------------------------------------------
struct BlockPart {
  bool any, is_v;
  int head;
  Q8Block b;
  int lo, hi;          // new slots of the block
};
__device__ __forceinline__ BlockPart block_part(const DevPlan& p, const Q8Dev& x) {
  BlockPart u;
  const int per = 2 * p.num_kv_heads, part = blockIdx.x % per;
  const int i = 4 * (blockIdx.x / per) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  u.any = i < x.num_blocks;
  u.is_v = part & 1;
  u.head = part >> 1;
  const Q8Block* at = x.blocks + (u.any ? i : 0);
  u.b = {const_load(&at->page), const_load(&at->slot), const_load(&at->token), const_load(&at->span)};
  u.lo = u.b.span & 255;
  u.hi = u.b.span >> 8;
  return u;
}

template <int D>
__global__ __launch_bounds__(256) void q8_append_kernel(DevPlan p, Q8Dev x, const u32x4* __restrict__ k_new,
                                                        const u32x4* __restrict__ v_new, uint8_t* __restrict__ k_pool,
                                                        uint8_t* __restrict__ v_pool) {
  constexpr int LPR = D / 8, RPP = 64 / LPR, NP = kQ8Block / RPP;      // lanes of a row, rows a pass, passes
  const BlockPart u = block_part(p, x);          // in one trip with the header
  if (int(!meta_ok(p)) | int(!u.any) | int(u.lo >= u.hi)) return;
  const int Hkv = p.num_kv_heads, B = p.page_size, lane = threadIdx.x & 63, first = lane / LPR;
  const u32x4* rows = (u.is_v ? v_new : k_new) + (int64_t(u.b.token) * Hkv + u.head) * LPR + lane % LPR;
  uint8_t* run = (u.is_v ? v_pool : k_pool) + (int64_t(u.b.page) * Hkv + u.head) * (B * D + kQ8ScaleBytes);
  uint8_t* codes = run + (u.b.slot + first) * D + 8 * (lane % LPR);
  uint8_t* mark = run + B * D + u.b.slot / kQ8Block;
  u32x4 v[NP];
  u32x2 held[NP];
  int e_held = 0;
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int row = min(max(i * RPP + first, u.lo), u.hi - 1);         // others' rows stand in for those that are not new
    v[i] = __builtin_nontemporal_load(rows + int64_t(row - u.lo) * Hkv * LPR);
  }
  if (u.lo > 0) {                            // the block holds earlier tokens
#pragma unroll
    for (int i = 0; i < NP; ++i) held[i] = *reinterpret_cast<const u32x2*>(codes + i * RPP * D);
    e_held = __builtin_amdgcn_readfirstlane(*mark);
  }
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < NP; ++i)
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      // magnitudes of bf16 order like integers; NaN and infinities become the largest magnitude
      const uint32_t lo = min(v[i][w] & 0x7FFFu, kLargest), hi = min((v[i][w] >> 16) & 0x7FFFu, kLargest);
      v[i][w] = (v[i][w] & 0x80008000u) | lo | (hi << 16);
      top = max(top, max(lo, hi));
    }
  top = wave_most<true>(top);
  // top = 1.m * 2^(E - 127): the smallest s with top <= 1.75 * 2^8 s is 2^(E - 127 - 8), twice that where 1.m > 1.75
  const int e = max(max(int(top >> 7) - 8 + int((top & 0x7Fu) > 0x60u), 8), e_held);
  const float s = scale_of(uint32_t(e));
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int row = i * RPP + first;
    if (row >= u.lo && row < u.hi) *reinterpret_cast<u32x2*>(codes + i * RPP * D) = q8_codes(v[i], s);
  }
  if (u.lo > 0 && e > e_held) {
    const float was = scale_of(uint32_t(e_held));
#pragma unroll
    for (int i = 0; i < NP; ++i)
      if (i * RPP + first < u.lo)
        *reinterpret_cast<u32x2*>(codes + i * RPP * D) =
            q8_codes(__builtin_bit_cast(u32x4, q8_values(held[i][0], held[i][1], was, was)), s);
  }
  if (lane == 0) *mark = uint8_t(e);
}

template <int D>
__global__ __launch_bounds__(256) void q8_read_kernel(DevPlan p, Q8Dev x, const uint8_t* __restrict__ k_pool,
                                                      const uint8_t* __restrict__ v_pool, bf16x8* __restrict__ k_out,
                                                      bf16x8* __restrict__ v_out) {
  constexpr int LPR = D / 8, RPP = 64 / LPR, NP = kQ8Block / RPP;
  const BlockPart u = block_part(p, x);          // in one trip with the header
  if (int(!meta_ok(p)) | int(!u.any) | int(u.lo >= u.hi)) return;
  const int Hkv = p.num_kv_heads, B = p.page_size, lane = threadIdx.x & 63, first = lane / LPR;
  const uint8_t* run = (u.is_v ? v_pool : k_pool) + (int64_t(u.b.page) * Hkv + u.head) * (B * D + kQ8ScaleBytes);
  const uint8_t* codes = run + (u.b.slot + first) * D + 8 * (lane % LPR);
  bf16x8* rows = (u.is_v ? v_out : k_out) + (int64_t(u.b.token) * Hkv + u.head) * LPR + lane % LPR;
  u32x2 held[NP];
#pragma unroll
  for (int i = 0; i < NP; ++i) held[i] = *reinterpret_cast<const u32x2*>(codes + i * RPP * D);
  const float s = scale_of(run[B * D + u.b.slot / kQ8Block]);
#pragma unroll
  for (int i = 0; i < NP; ++i) {
    const int row = i * RPP + first;
    if (row >= u.lo && row < u.hi) rows[int64_t(row - u.lo) * Hkv * LPR] = q8_values(held[i][0], held[i][1], s, s);
  }
}

// ---------------------------------------------------------------------------------------------
// Scores.  Everything past a product's accumulator is in units of log2: a weight is 2 to the power of its score.
// ---------------------------------------------------------------------------------------------

// A weight is 2 to the power of its score less a reference m, which lies at most 8 under the largest.  The key that set m
// has a weight of 2^d, d being what m lost when it was rounded: nothing that matters up to 2^28, where d is 16 at most and
// the row's sum takes it out again; beyond, that weight could be anything.  So scores under -2^28 weigh nothing, like
// masked ones (a split may hold no others), and a reference over 2^28 gives a row of NaN.
constexpr float kFarScore = 0x1p28f;
__device__ __forceinline__ float reference(float m) { return m < -kFarScore ? 0.0f : m; }
// A row's sum of weights: 0 for a row of no weight, NaN for one that has no sum.
__device__ __forceinline__ float row_sum(float m, float l) { return m <= kFarScore ? l : NAN; }

// The weights meet V rounded to bf16.  Where an output is divided by the sum of the rounded ones, what a rounding does to a weight
// is taken out of that sum too, so a row that one key rules has that key's values, not up to 2^-8 off.  With few rows this
// costs nothing; with many 4 % (long_prefix 1,994 us, 2,076), which capped scores get, whose largest weights are any number, and
// others do without: there the largest is mostly 1, as the reference is the largest score of a row's first tiles.  The LSE is of
// the weights themselves in all of them.
__device__ __forceinline__ float plus_rounded(float sum, const bf16x8& w) {
  const bf16x2 one = {static_cast<__bf16>(1.0f), static_cast<__bf16>(1.0f)};
#pragma unroll
  for (int i = 0; i < 8; i += 2) sum = __builtin_amdgcn_fdot2_f32_bf16(bf16x2{w[i], w[i + 1]}, one, sum, false);
  return sum;
}

// What a kernel's scores are.  CAUSAL: softmax_scale q.k up to the row's own position.  LINEAR: with a slope on the distance, or
// an interval of keys.  CAPPED: with a cap of kFixedCap at most, and perhaps an interval.  MIXED: with a cap otherwise.
enum Form { CAUSAL, LINEAR, CAPPED, MIXED };

// Scores of CAPPED lie within c = cap log2 e of 0, so their weights need no running reference: they are taken against one fixed
// at min(c, 80 - c).  That leaves them within 2^-80 and 2^(2 c - 80), 2^65 at most: sums over 2^20 keys and their products with
// values within 2^-40 and 2^40 stay well inside fp32.
constexpr float kFixedCap = 50.0f;

// One lane's query row's scores.  A product's accumulator becomes a value x whose score is a x + b, so the weight is one fused
// multiply-add and one exp2 of x in every form:
//   * x = q.k less the slope over softmax_scale times the distance, a = softmax_scale log2 e; or
//   * x = -1 / (1 + e^2z), z = softmax_scale q.k / cap, a = 2 cap log2 e and b = cap log2 e, as tanh z = 1 - 2 / (1 + e^2z):
//     good to 2^-21 at all z, for a multiply, an addition, and an instruction of lower rate for each of exp2 and the reciprocal
//     (CAPPED); or
//   * the score itself (MIXED).  A cap over 128 multiplies that error beyond a score's own rounding: small z then take the
//     series, whose next term is 2^-26 of z at a quarter.
struct Scores {
  float a, b;
  float in, out;               // CAPPED: 2 log2 e softmax_scale / cap, cap log2 e
  float slope;                 // over softmax_scale where LINEAR, times log2 e where MIXED
  bool sloped, wide;
};
template <Form F>
__device__ __forceinline__ Scores scores_of(const DevPlan& p, const Q8Dev& x, int head) {
  Scores r{};
  r.a = p.softmax_scale * kLog2e;
  r.sloped = F != CAUSAL && x.slopes;
  if (r.sloped) r.slope = x.slopes[head] * (F == MIXED ? kLog2e : 1.0f / p.softmax_scale);
  if (F == CAPPED || F == MIXED) {
    r.in = 2.0f * kLog2e * p.softmax_scale / x.cap;
    r.out = x.cap * kLog2e;
    r.wide = x.cap > 128.0f;
    r.a = F == MIXED ? 1.0f : 2.0f * r.out;
    r.b = F == MIXED ? 0.0f : r.out;
  }
  return r;
}
__device__ __forceinline__ float fixed_reference(const Scores& r) { return fminf(r.out, 80.0f - r.out); }
// -1 / (1 + e^2z) of a product.
__device__ __forceinline__ float logistic_of(float s, const Scores& r) {
  return __builtin_amdgcn_rcpf(-1.0f - fast_exp2(s * r.in));
}
// cap log2 e tanh z of a product.
__device__ __forceinline__ float capped_of(float s, const Scores& r) {
  const float t = fmaf(2.0f, logistic_of(s, r), 1.0f);
  if (!r.wide) return r.out * t;
  const float z = s * r.in * (0.5f * kLn2), y = z * z;
  const float series = z * (1.0f + y * (-0x1.555556p-2f + y * (0x1.111112p-3f + y * (-0x1.ba1ba2p-5f + y * 0x1.664f48p-6f))));
  return r.out * (fabsf(z) < 0.25f ? series : t);
}

// ---------------------------------------------------------------------------------------------
// Attention of many rows.  The layout is that of the kernel over bf16 pages (kernels.hip): a workgroup of NW waves takes 32 NW
// query rows of one (request, KV head) and walks tiles of keys that all its rows share; scores S^T = K Q^T and
// O^T += V^T P^T on 32x32x16 matrix instructions, K from LDS rows, V by transposing LDS reads, the probabilities straight
// from the accumulators, rounded to bf16 for the second product.  A tile's codes are loaded (half of the bytes) before the
// MFMAs of the tile before it and turned into bf16 rows in the other LDS buffer after them: once for all NW waves.
// A wave stages 16 keys, which share a page and a scale: both are the wave's own scalars.
// Bound by the matrix instructions and the vector work of the softmax, which hardly overlap (of 7,470 clocks a tile of 128 keys,
// 4,060 and 3,660 a SIMD): 1,024 tokens behind 65,536, 64/8 heads of 128, 1,896-2,059 us on boxes of unlike clocks, 1.08-1.17
// PFLOP/s, where large library products reach 1.2-1.6.  With capped scores 2,560-2,630, three instructions of lower rate a score for
// one; 4 x 2,048 tokens behind 0-4,096, 32/8 heads: 474 us causal, 500 with slopes, 630-655 capped, 765 capped with slopes.
// ---------------------------------------------------------------------------------------------

// Where the 8-value piece c of a V row lies in its LDS row (stride 16 banks past a multiple of 64): the four pieces that a
// thread writes one by one exchange places by the thread's quarter of the row, so that all threads' pieces of one turn fall
// on distinct banks.
__device__ __forceinline__ int v_place(int c) { return 8 * (c ^ ((c >> 2) & 3)); }

template <int D, int NW, Form F>
__global__ __launch_bounds__(NW * 64, NW == 4 ? 2 : 1) void attn_q8_kernel(DevPlan p, Q8Dev x, const __bf16* __restrict__ q,
                                                                           const uint8_t* __restrict__ kpool,
                                                                           const uint8_t* __restrict__ vpool,
                                                                           __bf16* __restrict__ out,
                                                                           float* __restrict__ lse_out) {
  constexpr int KT = NW == 4 ? kKvTile / 2 : kKvTile;   // keys per tile
  constexpr int NKB = KT / 32;
  constexpr int KSTR = D + 8;          // K rows in LDS: 16-byte reads of 8 rows land on distinct banks
  constexpr int VSTR = D + 32;         // V rows: transposed reads of 4 rows x 2 groups x 32 bytes on distinct banks
  constexpr int W = D / 64;            // 16-byte pieces of codes per thread and tile, for K and for V: a quarter of a row
  constexpr int AHEAD = 2;             // CAPPED: LDS reads ahead of their products
  static_assert(KT * 4 == NW * 64, "four threads a key, 16 keys a wave");
  __shared__ __attribute__((aligned(16))) __bf16 ks[2][KT * KSTR];
  __shared__ __attribute__((aligned(16))) __bf16 vs[2][KT * VSTR];

  // the header, the item and its request in one trip to memory
  const WorkItem it = p.items[blockIdx.x];
  const Q8ItemReq rm = x.item_reqs[blockIdx.x];
  if (int(!meta_ok(p)) | int(it.rows <= 0)) return;
  const int Hq = p.num_q_heads, Hkv = p.num_kv_heads;
  const int G = Hq / Hkv;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 31, hf = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int last = it.kv_end - 1;                                // the last position to load
  const int32_t* __restrict__ bt = p.bt + rm.bt_row;
  const int B = p.page_size, shift = B == 64 ? 6 : 4;
  const int64_t page_bytes = B * D + kQ8ScaleBytes, page_stride = Hkv * page_bytes;
  const uint8_t* __restrict__ kpool_h = kpool + it.kv_head * page_bytes;
  const uint8_t* __restrict__ vpool_h = vpool + it.kv_head * page_bytes;

  // ---- K/V tile staging -----------------------------------------------------------------------
  // Thread tid has a quarter of key tid / 4's row.  Positions past the last that the item's rows see are clamped to that
  // one, those before the first to that: copies that the mask gives zero weight, so what nobody sees is never read.
  const int key = tid >> 2, part = tid & 3;
  u32x4 kreg[W], vreg[W];
  uint32_t kscale = 0, vscale = 0;
  // The page of this wave's keys is looked up one tile ahead.
  auto within = [&](int j) { return min(F == CAUSAL ? j : max(j, rm.first), last); };
  auto page_of = [&](int tile) { return const_load(bt + (within(tile * KT + wave * 16) >> shift)); };
  auto load_tile = [&](int tile, int page) {
    const int j = within(tile * KT + key), j0 = within(tile * KT + wave * 16);
    const int64_t at = int64_t(page) * page_stride;
    const uint32_t off = uint32_t(j & (B - 1)) * D + part * (W * 16);
    const uint32_t soff = uint32_t(B * D) + uint32_t((j0 & (B - 1)) >> 4);
#pragma unroll
    for (int i = 0; i < W; ++i) {
      kreg[i] = *reinterpret_cast<const u32x4*>(kpool_h + at + off + 16 * i);
      vreg[i] = *reinterpret_cast<const u32x4*>(vpool_h + at + off + 16 * i);
    }
    kscale = (kpool_h + at)[soff];
    vscale = (vpool_h + at)[soff];
  };
  const int t_begin = it.kv_begin / KT;
  const int t_end = (it.kv_end + KT - 1) / KT;
  if (t_begin < t_end) load_tile(t_begin, page_of(t_begin));       // under way while the rows are looked up

  // ---- this lane's query row -----------------------------------------------------------------
  const int lrow = wave * 32 + col;
  const bool row_ok = lrow < it.rows;
  const int prow = it.row0 + (row_ok ? lrow : 0);
  const int tok = prow / G;
  const int head = it.kv_head * G + (prow - tok * G);
  int begin = 0, end = rm.prefix + tok + 1;                      // keys that this row sees
  if (F != CAUSAL && x.ranges) {
    const TokenRange seen = x.ranges[rm.cu + tok];
    begin = seen.begin;
    end = seen.end;
  }
  bf16x8 qf[D / 16];
  {
    const __bf16* qrow = q + (int64_t(rm.cu + tok) * Hq + head) * D + 8 * hf;
#pragma unroll
    for (int s = 0; s < D / 16; ++s) qf[s] = row_ok ? *reinterpret_cast<const bf16x8*>(qrow + 16 * s) : bf16x8{};
  }
  const int wrow0 = wave * 32;
  const bool wave_active = wrow0 < it.rows;
  const int wrow_last = min(it.rows, wrow0 + 32) - 1;
  // Tiles in [wave_first, wave_end) have keys that a row of the wave sees; all rows see all keys of [all_first, all_end).
  int wave_first = 0, wave_end = rm.prefix + (it.row0 + max(wrow_last, wrow0)) / G + 1;
  int all_first = 0, all_end = rm.prefix + (it.row0 + wrow0) / G + 1;
  const Scores sc = scores_of<F>(p, x, head);
  if (F != CAUSAL) {
    if (x.ranges) {
      wave_first = row_ok && begin < end ? begin : INT32_MAX;
      wave_end = row_ok && begin < end ? end : 0;
      all_first = row_ok ? begin : 0;
      all_end = row_ok ? end : INT32_MAX;
      wave_first = wave_most<false>(wave_first);
      wave_end = wave_most<true>(wave_end);
      all_first = wave_most<true>(all_first);
      all_end = wave_most<false>(all_end);
    }
  }

  f32x16 oacc[D / 32];
#pragma unroll
  for (int db = 0; db < D / 32; ++db) oacc[db] = f32x16{};
  // The sum of the weights, and of the weights as rounded where that is kept: both of the lane's keys then, half of the row's.
  // (Joined at the end in the other forms too, long_prefix takes 1,978 us for 1,936: the compiler's schedule of a tile.)
  constexpr bool ROUNDED = F == CAPPED || F == MIXED;
  float m_run = F == CAPPED ? fixed_reference(sc) : -INFINITY, l_run = 0.0f, w_run = 0.0f;

  auto store_tile = [&](int buf) {
    __bf16* kd = &ks[buf][key * KSTR + part * (W * 16)];
    const float a = scale_of(kscale), b = scale_of(vscale);
#pragma unroll
    for (int i = 0; i < W; ++i)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        *reinterpret_cast<bf16x8*>(kd + 16 * i + 8 * u) = q8_values(kreg[i][2 * u], kreg[i][2 * u + 1], a, a);
        *reinterpret_cast<bf16x8*>(&vs[buf][key * VSTR + v_place(part * (2 * W) + 2 * i + u)]) =
            q8_values(vreg[i][2 * u], vreg[i][2 * u + 1], b, b);
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

  // A tile of CAPPED scores: with the reference fixed, nothing waits for a maximum, so the weights of one block of 32 keys are
  // worked out behind the products of the next one's scores and those of the last one's weights with V: an element of them
  // after each product.  The order is pinned: left to itself the compiler makes blocks of each.
  auto capped_tile = [&](int buf) {
    constexpr int M = D / 16;                    // products of a block's scores, and of its weights with V
    const float less = sc.b - m_run;
    const __bf16* kl = &ks[buf][k_lane];
    const __bf16* vl = &vs[buf][0];
    auto k_read = [&](int n) { return *reinterpret_cast<const bf16x8*>(kl + 32 * (n / M) * KSTR + 16 * (n % M)); };
    auto v_read = [&](int n) {                   // product n of a tile with V: step n / (D / 32), columns n % (D / 32)
      const __bf16* at = vl + v_lane[n % (D / 32)] + 16 * (n / (D / 32)) * VSTR;
      const bf16x4 lo = lds_read_tr(at), hi = lds_read_tr(at + 8 * VSTR);
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    f32x16 s = f32x16{}, next = f32x16{};
    bf16x8 kf[AHEAD], vf[AHEAD], pb[2];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) kf[i] = k_read(i);
#pragma unroll
    for (int i = 0; i < M; ++i) {
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[i % AHEAD], qf[i], s, 0, 0, 0);
      kf[i % AHEAD] = k_read(i + AHEAD);
    }
    // An element's weight is worked out in three parts, each behind the next product, so that no part waits for the one before.
    float one = 0.0f, two = 0.0f, e = 0.0f;
#pragma unroll
    for (int kb = 0; kb <= NKB; ++kb) {
      const bool scores = kb + 1 < NKB, weights = kb < NKB, values = kb > 0;
      if (values)
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) vf[i] = v_read((kb - 1) * M + i);
      next = f32x16{};
      bf16x8 pb_next[2];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        __builtin_amdgcn_sched_barrier(0);
        constexpr int per = 16 / M;              // elements of the weights for each product of a kind
        if (i % per == 0) {
          const int n = i / per;
          if (scores) {
            next = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[n % AHEAD], qf[n], next, 0, 0, 0);
            if ((kb + 1) * M + n + AHEAD < NKB * M) kf[n % AHEAD] = k_read((kb + 1) * M + n + AHEAD);
          }
        }
        const bool third = weights ? i >= 2 || kb > 0 : i < 2, second = weights ? i >= 1 || kb > 0 : i < 1;
        if (third) {
          e = fast_exp2(fmaf(two, sc.a, less));
          l_run += e;
          const int at = (i + 14) % 16;
          if (i >= 2) pb_next[at >> 3][at & 7] = static_cast<__bf16>(e);
          else pb[at >> 3][at & 7] = static_cast<__bf16>(e);
          if (i == 9) w_run = plus_rounded(w_run, pb_next[0]);
          if (i == 1) w_run = plus_rounded(w_run, pb[1]);
        }
        if (second) two = __builtin_amdgcn_rcpf(-1.0f - one);
        if (weights) one = fast_exp2(s[i] * sc.in);
        if (values && i % per == per - 1) {
          const int n = i / per, db = n % (D / 32);
          oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[n % AHEAD], pb[n / (D / 32)], oacc[db], 0, 0, 0);
          if (n + AHEAD < M) vf[n % AHEAD] = v_read((kb - 1) * M + n + AHEAD);
        }
      }
      s = next;
      pb[0] = pb_next[0];
      pb[1] = pb_next[1];
    }
  };

  // The same with a mask, block by block: a tile at the end of what a row sees.
  auto capped_edge = [&](int buf, int over, int under) {
    const float less = sc.b - m_run;
#pragma unroll 1
    for (int kb = 0; kb < NKB; ++kb) {
      const __bf16* kl = &ks[buf][k_lane + 32 * kb * KSTR];
      const __bf16* vl = &vs[buf][32 * kb * VSTR];
      f32x16 s = f32x16{};
#pragma unroll
      for (int i = 0; i < D / 16; ++i)
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*reinterpret_cast<const bf16x8*>(kl + 16 * i), qf[i], s, 0, 0, 0);
      bf16x8 pb[2];
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int c = 32 * kb + 8 * (r >> 2) + (r & 3);
        float e = fast_exp2(fmaf(logistic_of(s[r], sc), sc.a, less));
        if (c >= over || c < under) e = 0.0f;
        l_run += e;
        pb[r >> 3][r & 7] = static_cast<__bf16>(e);
      }
#pragma unroll
      for (int t = 0; t < 2; ++t) w_run = plus_rounded(w_run, pb[t]);
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
          const bf16x4 lo = lds_read_tr(vl + v_lane[db] + 16 * t * VSTR);
          const bf16x4 hi = lds_read_tr(vl + v_lane[db] + (16 * t + 8) * VSTR);
          const bf16x8 a = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
          oacc[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pb[t], oacc[db], 0, 0, 0);
        }
    }
  };

  int pg_nxt = 0;
  if (t_begin < t_end) {
    store_tile(0);
    pg_nxt = page_of(t_begin + 1);
  }
  __syncthreads();

  for (int tile = t_begin; tile < t_end; ++tile) {
    const int buf = (tile - t_begin) & 1;
    const bool has_next = tile + 1 < t_end;
    if (has_next) {
      load_tile(tile + 1, pg_nxt);
      pg_nxt = page_of(tile + 2);
    }
    const int kbase = tile * KT;
    const bool active = wave_active && kbase < wave_end && (F == CAUSAL || kbase + KT > wave_first);
    const bool mask_over = kbase + KT > all_end || kbase + KT > it.kv_end, mask_under = F != CAUSAL && kbase < all_first;
    const int over = min(end, it.kv_end) - kbase - 4 * hf, under = begin - kbase - 4 * hf;
    if (F == CAPPED && active) {
      if (mask_over || mask_under) capped_edge(buf, over, under);
      else capped_tile(buf);
    } else if (active) {
      // S^T[key][row] for the KT keys of the tile, as NKB 32-key blocks; accumulator element r of block kb holds key
      // 32*kb + 8*(r/4) + 4*hf + (r%4).  A slope without a cap is what the products are added to.
      f32x16 sacc[NKB];
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb) sacc[kb] = f32x16{};
      const float from = float(rm.prefix + tok - kbase - 4 * hf);
      if (F == LINEAR && sc.sloped) {
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) sacc[kb][r] = -sc.slope * fabsf(from - float(32 * kb + 8 * (r >> 2) + (r & 3)));
      }
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
      if (F == MIXED) {
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb) {
#pragma unroll
          for (int r = 0; r < 16; ++r)
            sacc[kb][r] = fmaf(-sc.slope, fabsf(from - float(32 * kb + 8 * (r >> 2) + (r & 3))), capped_of(sacc[kb][r], sc));
          __builtin_amdgcn_sched_barrier(0);       // block by block: fewer registers
        }
      }
      if (mask_over) {
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (32 * kb + 8 * (r >> 2) + (r & 3) >= over) sacc[kb][r] = -INFINITY;
      }
      if (mask_under) {
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if (32 * kb + 8 * (r >> 2) + (r & 3) < under) sacc[kb][r] = -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sacc[kb][r]);
      mx = fmaf(halves_max(mx), sc.a, sc.b);
      // The reference max only moves when the tile's max exceeds it by more than 2^8, so most tiles
      // skip rescaling the accumulators; probabilities stay below 256, which bf16/fp32 represent as
      // well as values below 1.  The final normalization uses the same reference.
      const bool bump = mx > m_run + 8.0f;
      const float m_new = bump ? mx : m_run;
      const float m_use = reference(m_new);
      const float less = sc.b - m_use;
      float rs = 0.0f;
      bf16x8 pb[2 * NKB];
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float e = fast_exp2(fmaf(sacc[kb][r], sc.a, less));
          rs += e;
          pb[2 * kb + (r >> 3)][r & 7] = static_cast<__bf16>(e);
        }
      if (!ROUNDED) rs = halves_sum(rs);
      if (__any(bump)) {
        const float alpha = fast_exp2(m_run - m_use);
        l_run *= alpha;
        w_run *= alpha;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) oacc[db][r] *= alpha;
      }
      l_run += rs;
#pragma unroll
      for (int i = 0; ROUNDED && i < 2 * NKB; ++i) w_run = plus_rounded(w_run, pb[i]);
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

  // ---- epilogue: O = O^T / w, lse = ln(l) + m (natural log) ------------------------------------
  if (ROUNDED) {
    l_run = halves_sum(l_run);
    w_run = halves_sum(w_run);
  }
  if (!row_ok) return;
  const float sum = row_sum(m_run, l_run), rounded = row_sum(m_run, ROUNDED ? w_run : l_run);
  const float inv_l = sum == 0.0f ? 0.0f : 1.0f / rounded;
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
// Attention of few rows: up to 32 query rows for each (request, KV head), so one token of up to 32 heads a group or a few
// tokens.  The cache is read once and hardly computed with, so the work is to keep loads in flight: the four waves of a
// workgroup each take every fourth block of 32 keys with all the rows, straight from memory into registers, and join
// their sums at the end.  Products are on 16x16x32 matrix instructions, so rows come in RT tiles of 16: one token of up to 16
// heads a group costs half of what two tiles do.
//   * K needs no LDS: a lane has 16-byte pieces of the row that it feeds to the matrix instruction.  Any order of the
//     contraction over the head dim will do, so step 2 i + u takes half u of piece 4 i + g (g = lane / 16), and Q's rows
//     are loaded in that order.
//   * V needs transposing: its codes go as they are through rows in LDS that belong to the wave alone, without barriers, and
//     come back by transposing reads of eight codes, which are turned into bf16 in registers.
// The accumulator of a block's scores, element r of key tile kt, holds key 16 kt + 4 g + r: with the keys of the second
// product in the order (g, kt, r), the probabilities are its operand where they lie.
// Bound by memory: a token each behind 64 x 1-32 K cached (64/8 heads of 128, pages of 64) 361 us, 5.95 TB/s, where reads alone reach
// 6.1; 377 through the caches.  128 tokens behind 16-4,000 (24/4 heads of 64, pages of 16) 32 us: runs of 1,040 bytes
// begin and end inside lines, 156 MB are read for 137.  One token behind 8,191: 7 us, and 3.5 for the join of its splits.
// ---------------------------------------------------------------------------------------------

// 16 bytes, where STREAM without a place in the caches.
template <bool STREAM>
__device__ __forceinline__ u32x4 load16(const uint8_t* at) {
  if constexpr (STREAM) return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(at));
  else return *reinterpret_cast<const u32x4*>(at);
}

// Largest value, and the sum, over the four lanes l % 16 + 16 g of a query row.
__device__ __forceinline__ float quarters_max(float v) {
  const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return halves_max(fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1])));
}
__device__ __forceinline__ float quarters_sum(float v) {
  const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return halves_sum(__uint_as_float(s[0]) + __uint_as_float(s[1]));
}

template <int D, int RT, Form F, bool STREAM>
__global__ __launch_bounds__(256, 2) void attn_q8_few_kernel(DevPlan p, Q8Dev x, const __bf16* __restrict__ q,
                                                             const uint8_t* __restrict__ kpool,
                                                             const uint8_t* __restrict__ vpool, __bf16* __restrict__ out,
                                                             float* __restrict__ lse_out) {
  constexpr int NK = D / 64, NV = D / 32;        // 16-byte pieces per lane: of K for each key tile, of V
  constexpr int PPR = D / 16;                    // pieces of a row
  constexpr int VSTR = D + 16;                   // bytes of a V row in LDS: transposing reads of 32 rows on distinct banks
  constexpr int OSTR = D + 4;                    // floats per row while the waves' sums are joined
  constexpr int VBYTES = 32 * VSTR, JOIN = 4 * 16 * OSTR * 4;
  __shared__ __attribute__((aligned(16))) unsigned char smem[4 * VBYTES > JOIN ? 4 * VBYTES : JOIN];
  __shared__ float wave_m[4][16 * RT], wave_l[4][16 * RT], wave_w[4][16 * RT];

  // the header, the item and its request in one trip to memory
  const WorkItem it = p.items[blockIdx.x];
  const Q8ItemReq rm = x.item_reqs[blockIdx.x];
  if (int(!meta_ok(p)) | int(it.rows <= 0)) return;
  const int Hq = p.num_q_heads, Hkv = p.num_kv_heads;
  const int G = Hq / Hkv;
  const int tid = threadIdx.x, lane = tid & 63, col = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int last = it.kv_end - 1;                // the last position to load
  const int32_t* __restrict__ bt = p.bt + rm.bt_row;
  const int B = p.page_size, shift = B == 64 ? 6 : 4;
  const int64_t page_bytes = B * D + kQ8ScaleBytes, page_stride = Hkv * page_bytes;
  const uint8_t* __restrict__ kpool_h = kpool + it.kv_head * page_bytes;
  const uint8_t* __restrict__ vpool_h = vpool + it.kv_head * page_bytes;

  int begin[RT], end[RT], pos[RT];               // keys that this lane's rows see, the rows' positions
  bf16x8 qf[RT][D / 32];
  Scores sc[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int lrow = 16 * t + col;
    const bool row_ok = lrow < it.rows;
    const int prow = it.row0 + (row_ok ? lrow : 0);
    const int tok = prow / G, head = it.kv_head * G + (prow - tok * G);
    pos[t] = rm.prefix + tok;
    begin[t] = 0;
    end[t] = pos[t] + 1;
    if (F != CAUSAL && x.ranges) {
      const TokenRange seen = x.ranges[rm.cu + tok];
      begin[t] = seen.begin;
      end[t] = seen.end;
    }
    sc[t] = scores_of<F>(p, x, head);
    const __bf16* qrow = q + (int64_t(rm.cu + tok) * Hq + head) * D;
#pragma unroll
    for (int s = 0; s < D / 32; ++s)
      qf[t][s] = row_ok ? *reinterpret_cast<const bf16x8*>(qrow + 16 * (4 * (s >> 1) + g) + 8 * (s & 1)) : bf16x8{};
  }
  // all rows see all keys from all_first to before all_end
  const int all_first = F != CAUSAL && x.ranges ? INT32_MAX : 0;
  const int all_end = F != CAUSAL && x.ranges ? 0 : rm.prefix + it.row0 / G + 1;

  struct Block {                                 // 32 keys
    u32x4 k[2][NK], v[NV];
    uint32_t scales;                             // lanes 0..3: K's bytes of both key tiles, V's
  };
  // Positions that no row of the item sees are clamped to those that one does, as above.
  auto within = [&](int j) { return min(F == CAUSAL ? j : max(j, rm.first), last); };
  auto load = [&](Block& b, int block) {
    const int kbase = 32 * block;
    const int64_t at[2] = {int64_t(const_load(bt + (within(kbase) >> shift))) * page_stride,
                           int64_t(const_load(bt + (within(kbase + 16) >> shift))) * page_stride};
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const uint32_t off = uint32_t(within(kbase + 16 * kt + col) & (B - 1)) * D + 16 * g;
#pragma unroll
      for (int i = 0; i < NK; ++i) b.k[kt][i] = load16<STREAM>(kpool_h + at[kt] + off + 64 * i);
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int piece = lane + 64 * i;
      const uint32_t off = uint32_t(within(kbase + piece / PPR) & (B - 1)) * D + 16 * (piece % PPR);
      b.v[i] = load16<STREAM>(vpool_h + at[64 * i / D] + off);
    }
    const uint8_t* pool = lane & 2 ? vpool_h : kpool_h;
    const int j = within(kbase + 16 * (lane & 1));
    b.scales = (pool + (lane & 1 ? at[1] : at[0]))[uint32_t(B * D) + uint32_t((j & (B - 1)) >> 4)];
  };

  unsigned char* const vs = smem + wave * VBYTES;
  // transposing reads: lanes 2 m and 2 m + 1 of 16 address the two halves of 16 bytes of the m-th of their eight keys
  const unsigned char* const vl = vs + (16 * (col >> 3) + 4 * g + ((col >> 1) & 3)) * VSTR + 8 * (lane & 1);
  f32x4 oacc[RT][D / 16];
  float m_run[RT], l_run[RT], w_run[RT];         // the sums of this lane's keys alone
#pragma unroll
  for (int t = 0; t < RT; ++t) {
#pragma unroll
    for (int db = 0; db < D / 16; ++db) oacc[t][db] = f32x4{};
    m_run[t] = -INFINITY;
    l_run[t] = w_run[t] = 0.0f;
  }

  auto attend = [&](const Block& b, int block) {
    const int kbase = 32 * block;
    f32x4 s[RT][2];
#pragma unroll
    for (int t = 0; t < RT; ++t) s[t][0] = s[t][1] = f32x4{};
    float scale[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) scale[i] = scale_of(__builtin_amdgcn_readlane(b.scales, i));
#pragma unroll
    for (int i = 0; i < NK; ++i)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int kt = 0; kt < 2; ++kt) {
          const bf16x8 a = q8_values(b.k[kt][i][2 * u], b.k[kt][i][2 * u + 1], scale[kt], scale[kt]);
#pragma unroll
          for (int t = 0; t < RT; ++t) s[t][kt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, qf[t][2 * i + u], s[t][kt], 0, 0, 0);
        }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int piece = lane + 64 * i;
      *reinterpret_cast<u32x4*>(vs + piece / PPR * VSTR + 16 * (piece % PPR)) = b.v[i];
    }
    bf16x8 pb[RT];
    bool bump[RT];
    float alpha[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      if (F != CAUSAL) {
        const float from = float(pos[t] - kbase - 4 * g);
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float v = s[t][kt][r];
            if (F == CAPPED) v = logistic_of(v, sc[t]);
            if (F == MIXED) v = capped_of(v, sc[t]);
            s[t][kt][r] = F != CAPPED && sc[t].sloped ? fmaf(-sc[t].slope, fabsf(from - float(16 * kt + r)), v) : v;
          }
      }
      if (kbase + 32 > all_end || kbase + 32 > it.kv_end || (F != CAUSAL && kbase < all_first)) {
        const int over = min(end[t], it.kv_end) - kbase - 4 * g, under = begin[t] - kbase - 4 * g;
#pragma unroll
        for (int kt = 0; kt < 2; ++kt)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            if (16 * kt + r >= over || (F != CAUSAL && 16 * kt + r < under)) s[t][kt][r] = -INFINITY;
      }
      float mx = -INFINITY;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[t][kt][r]);
      mx = fmaf(quarters_max(mx), sc[t].a, sc[t].b);
      bump[t] = mx > m_run[t] + 8.0f;            // as in the kernel above
      const float m_new = bump[t] ? mx : m_run[t];
      const float m_use = reference(m_new);
      alpha[t] = fast_exp2(m_run[t] - m_use);
      const float less = sc[t].b - m_use;
      float rs = 0.0f;
#pragma unroll
      for (int kt = 0; kt < 2; ++kt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float e = fast_exp2(fmaf(s[t][kt][r], sc[t].a, less));
          rs += e;
          pb[t][4 * kt + r] = static_cast<__bf16>(e);
        }
      if (__any(bump[t])) {
        l_run[t] *= alpha[t];
        w_run[t] *= alpha[t];
#pragma unroll
        for (int db = 0; db < D / 16; ++db)
#pragma unroll
          for (int r = 0; r < 4; ++r) oacc[t][db][r] *= alpha[t];
      }
      l_run[t] += rs;
      w_run[t] = plus_rounded(w_run[t], pb[t]);
      m_run[t] = m_new;
    }
#pragma unroll
    for (int db = 0; db < D / 16; ++db) {
      const i32x2 c = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)(vl + 16 * db));
      const bf16x8 a = q8_values(uint32_t(c[0]), uint32_t(c[1]), scale[2], scale[3]);
#pragma unroll
      for (int t = 0; t < RT; ++t) oacc[t][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pb[t], oacc[t][db], 0, 0, 0);
    }
  };

  // Two blocks are in flight.  Loads are not branched around (a last block is loaded again instead), so the compiler
  // knows their number and waits for the older block alone.
  const int end_block = (it.kv_end + 31) / 32;
  int block = it.kv_begin / 32 + wave;
  if (block < end_block) {
    Block b0, b1;
    load(b0, block);
    __builtin_amdgcn_sched_barrier(0);
    load(b1, min(block + 4, end_block - 1));
    for (;;) {
      attend(b0, block);
      load(b0, min(block + 8, end_block - 1));
      if (block + 4 >= end_block) break;
      attend(b1, block + 4);
      load(b1, min(block + 12, end_block - 1));
      block += 8;
      if (block >= end_block) break;
    }
  }

  // ---- the waves' sums joined -------------------------------------------------------------------
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    l_run[t] = quarters_sum(l_run[t]);
    w_run[t] = quarters_sum(w_run[t]);
    if (g == 0) {
      wave_m[wave][16 * t + col] = m_run[t];
      wave_l[wave][16 * t + col] = l_run[t];
      wave_w[wave][16 * t + col] = w_run[t];
    }
  }
  float* const join = reinterpret_cast<float*>(smem);
  constexpr int N = D / 16;                      // values of a row that a thread joins
  const int row16 = tid >> 4, c0 = N * (tid & 15);
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    __syncthreads();                             // the waves are done with smem, their sums are there
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) m = fmaxf(m, wave_m[w][16 * t + col]);
    const float mine = m_run[t] == -INFINITY ? 0.0f : fast_exp2(m_run[t] - m);
#pragma unroll
    for (int db = 0; db < D / 16; ++db) {
      f32x4 v;
#pragma unroll
      for (int k = 0; k < 4; ++k) v[k] = oacc[t][db][k] * mine;
      *reinterpret_cast<f32x4*>(join + (wave * 16 + col) * OSTR + 16 * db + 4 * g) = v;
    }
    __syncthreads();
    const int row = 16 * t + row16;
    if (row >= it.rows) continue;
    float top = -INFINITY, l = 0.0f, rounded = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w) top = fmaxf(top, wave_m[w][row]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      // a sum of NaN stays so whatever its share, that of a wave which saw no other score included
      const float share = wave_l[w][row] == 0.0f ? 0.0f : fast_exp2(wave_m[w][row] - top);
      l += wave_l[w][row] * share;
      rounded += wave_w[w][row] * share;
    }
    l = row_sum(top, l);
    const float inv_l = l == 0.0f ? 0.0f : 1.0f / row_sum(top, rounded);
    const float lse_v = l == 0.0f ? -INFINITY : (top + __log2f(l)) * kLn2;
    const int prow = it.row0 + row, tok = prow / G;
    const int64_t orow = int64_t(rm.cu + tok) * Hq + it.kv_head * G + (prow - tok * G);
    float a[N];
#pragma unroll
    for (int k = 0; k < N; ++k) a[k] = 0.0f;
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int k = 0; k < N; k += 4) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(join + (w * 16 + row16) * OSTR + c0 + k);
#pragma unroll
        for (int j = 0; j < 4; ++j) a[k + j] += v[j];
      }
    if (it.part < 0) {
#pragma unroll
      for (int k = 0; k < N; k += 4) {
        bf16x4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = static_cast<__bf16>(a[k + j] * inv_l);
        *reinterpret_cast<bf16x4*>(out + orow * D + c0 + k) = o;
      }
      if (lse_out && (tid & 15) == 0) lse_out[orow] = lse_v;
    } else {
      float* to = p.opart + int64_t(it.part + row) * D + c0;
#pragma unroll
      for (int k = 0; k < N; k += 4) {
        f32x4 o;
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] = a[k + j] * inv_l;
        *reinterpret_cast<f32x4*>(to + k) = o;
      }
      if ((tid & 15) == 0) p.lpart[it.part + row] = lse_v;
    }
  }
}

}  // namespace

// ---------------------------------------------------------------------------------------------
// Launchers
// ---------------------------------------------------------------------------------------------
hipError_t launch_q8_append(const DevPlan& p, const Q8Dev& x, const void* k_new, const void* v_new, void* k_pool,
                            void* v_pool, hipStream_t stream) {
  const int64_t groups = q8_moves(x.num_blocks, p.num_kv_heads);
  if (groups > kQ8MostMoves) return hipErrorInvalidValue;
  auto kn = static_cast<const u32x4*>(k_new);
  auto vn = static_cast<const u32x4*>(v_new);
  auto kp = static_cast<uint8_t*>(k_pool);
  auto vp = static_cast<uint8_t*>(v_pool);
  if (p.head_dim_qk == 128)
    hipLaunchKernelGGL((q8_append_kernel<128>), dim3(groups), dim3(256), 0, stream, p, x, kn, vn, kp, vp);
  else if (p.head_dim_qk == 64)
    hipLaunchKernelGGL((q8_append_kernel<64>), dim3(groups), dim3(256), 0, stream, p, x, kn, vn, kp, vp);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

hipError_t launch_q8_read(const DevPlan& p, const Q8Dev& x, const void* k_pool, const void* v_pool, void* k_out, void* v_out,
                          hipStream_t stream) {
  const int64_t groups = q8_moves(x.num_blocks, p.num_kv_heads);
  if (groups > kQ8MostMoves) return hipErrorInvalidValue;
  auto kp = static_cast<const uint8_t*>(k_pool);
  auto vp = static_cast<const uint8_t*>(v_pool);
  auto ko = static_cast<bf16x8*>(k_out);
  auto vo = static_cast<bf16x8*>(v_out);
  if (p.head_dim_qk == 128)
    hipLaunchKernelGGL((q8_read_kernel<128>), dim3(groups), dim3(256), 0, stream, p, x, kp, vp, ko, vo);
  else if (p.head_dim_qk == 64)
    hipLaunchKernelGGL((q8_read_kernel<64>), dim3(groups), dim3(256), 0, stream, p, x, kp, vp, ko, vo);
  else
    return hipErrorInvalidValue;
  return hipGetLastError();
}

hipError_t launch_q8_attention(const DevPlan& p, const Q8Dev& x, int32_t num_few, const void* q, const void* k_pool,
                               const void* v_pool, void* out, float* lse, hipStream_t stream) {
  if (p.num_items == 0) return hipSuccess;
  auto qq = static_cast<const __bf16*>(q);
  auto kp = static_cast<const uint8_t*>(k_pool);
  auto vp = static_cast<const uint8_t*>(v_pool);
  auto oo = static_cast<__bf16*>(out);
  const int32_t num_many = p.num_items - num_few;
  if (num_many > kQ8MostMany || num_few > kQ8MostFew) return hipErrorInvalidValue;
  const bool w8 = p.rows_per_item == kGqaRowsPerItem, one = x.few_rows <= 16;
  const Form form = x.cap > 0.0f ? (x.cap <= kFixedCap && !x.slopes ? CAPPED : MIXED) : x.ranges || x.slopes ? LINEAR : CAUSAL;
  if (num_many && !w8 && p.rows_per_item != kGqaRowsPerItem / 2) return hipErrorInvalidValue;
  DevPlan few = p;
  Q8Dev xf = x;
  few.items += num_many;
  xf.item_reqs += num_many;
#define WAVEPP_Q8_FEW(D_, RT_, F_)                                                                                     \
  if (x.stream)                                                                                                        \
    hipLaunchKernelGGL((attn_q8_few_kernel<D_, RT_, F_, true>), dim3(num_few), dim3(256), 0, stream, few, xf, qq, kp, vp, oo, \
                       lse);                                                                                           \
  else                                                                                                                 \
    hipLaunchKernelGGL((attn_q8_few_kernel<D_, RT_, F_, false>), dim3(num_few), dim3(256), 0, stream, few, xf, qq, kp, vp, oo, \
                       lse);
#define WAVEPP_Q8(D_, F_)                                                                                          \
  if (num_many && w8)                                                                                                  \
    hipLaunchKernelGGL((attn_q8_kernel<D_, 8, F_>), dim3(num_many), dim3(512), 0, stream, p, x, qq, kp, vp, oo, lse);  \
  else if (num_many)                                                                                                   \
    hipLaunchKernelGGL((attn_q8_kernel<D_, 4, F_>), dim3(num_many), dim3(256), 0, stream, p, x, qq, kp, vp, oo, lse);  \
  if (num_few && one) {                                                                                                \
    WAVEPP_Q8_FEW(D_, 1, F_)                                                                                           \
  } else if (num_few) {                                                                                                \
    WAVEPP_Q8_FEW(D_, 2, F_)                                                                                           \
  }
  if (p.head_dim_qk == 128 && form == CAUSAL) {
    WAVEPP_Q8(128, CAUSAL)
  } else if (p.head_dim_qk == 128 && form == LINEAR) {
    WAVEPP_Q8(128, LINEAR)
  } else if (p.head_dim_qk == 128 && form == CAPPED) {
    WAVEPP_Q8(128, CAPPED)
  } else if (p.head_dim_qk == 128) {
    WAVEPP_Q8(128, MIXED)
  } else if (p.head_dim_qk == 64 && form == CAUSAL) {
    WAVEPP_Q8(64, CAUSAL)
  } else if (p.head_dim_qk == 64 && form == LINEAR) {
    WAVEPP_Q8(64, LINEAR)
  } else if (p.head_dim_qk == 64 && form == CAPPED) {
    WAVEPP_Q8(64, CAPPED)
  } else if (p.head_dim_qk == 64) {
    WAVEPP_Q8(64, MIXED)
  } else {
    return hipErrorInvalidValue;
  }
#undef WAVEPP_Q8
#undef WAVEPP_Q8_FEW
  return hipGetLastError();
}

}  // namespace wavepp
