// Tree attention over a KV pool held in 4 bits (layout: kv4.cuh) for work items with at most eight
// query rows; wider ones go to attn_q4_wide.cu.
//
// A unit is one work item and one kv head.  Twelve warps per SM each work
// through units of their own, from first to last block, with no barrier between them: a warp
// streams the tiles of its blocks (K and V of one block: 2560 bytes) through a private ring with
// cp.async, and the copies run ahead *across* units - the next unit's description, query rows and
// first blocks are on their way while the current one is computed.  (A CTA per unit whose four
// warps share its blocks spends some 5 us per unit on the chain item -> table -> tile and on the
// fold.)  Units are dealt out in the planner's order, longest first, forwards and backwards in turn, so no counter
// in memory is needed and the kernel can be captured and replayed as it is.
//
// Products run on mma.sync m16n8k16 (f16) with the *cache* as the 16-row operand and the queries
// as the 8-column one, so that a call with few rows per block wastes little of a product, and the
// codes of a block are turned into operand registers once.  A code is used as it lies in the
// word: four bits in the low end of a 16-bit lane are the subnormal f16 number c * 2^-24, and
// four bits higher up c * 2^-20, both exact in the tensor core, so a pair of codes costs one AND
// (and every other pair no shift).  The powers of two come out again for nothing:
//   S^T = K Q^T     A = K codes, 16 tokens x 16 dims.  B = the query row in f16, scaled by the power
//                   of two that brings its largest value to 2^14 (exact, but for values 2^-38 of
//                   the largest), and by another 2^-4 where codes stand four bits higher.  A
//                   group of 32 dims is two products, and its scale is applied to the 32-bit sums:
//                   score = sum_j s_j acc_j + sum_j lo_j qsum_j, with qsum_j the sum of the query over
//                   the group; the powers of two are part of the softmax scale.  The second sum is
//                   one more product: lo_j is a bf16 number, and qsum_j the sum of three, so
//                   that four groups fill a k of 16.  Scores are exact to 32 bits.
//   O^T += V^T P^T  A = V codes less 7.5, 16 dims x 16 tokens (one fused multiply-add a pair, exact).
//                   B = P s_j, one operand per group, rounded once to f16: it is below 2^16 by the
//                   choice of reference.  The middles lo_j + 7.5 s_j are summed in 32 bits on the
//                   side, once per group and row.  Codes as they lie, 0..15, would make of both sums
//                   numbers that grow with the length and cancel: over 32768 tokens of equal
//                   weight what the tensor core cuts off its sums, always the same way, and
//                   the rounding of one and the same weight came to 1.8 % of the result.  Less
//                   their middle they leave 0.16 %, the output's own rounding.
// The reference subtracted in the exponent is the running maximum of score + log2(largest
// scale of the token's V row), not of the score: P s_j is then bounded whatever the scales are,
// and f16's narrow exponent is spent on the largest terms of the sum.  It moves lazily (kSlack), and
// to a little below the maximum (kHeadroom): f16 numbers are normal from 2^-14 to 2^16, and in a
// long context most of the sum is in weights far below the largest.
//
// The C fragment of S^T holds tokens in rows, the B operand wants them in the k index: a
// movmatrix of the 8 x 8 halves brings one into the other.
//
// Measured: four contexts of 125 k tokens, 32 query heads over 8 (646 MB): 133 us, 4.9 TB/s, 0.74 of
// a copy (129 before the codes went less their middle; then, with the arithmetic taken out, 97 us, and
// with the loads taken out 113).  128 tails of 190 tokens and 32 prompts of 512 under 32 heads
// (210 MB): 59 us, 3.6 TB/s.  What bounds it is issue: a block is some 320 instructions of a warp, most
// of them on the integer pipe, and twelve warps are what the registers (168) allow.
#include <algorithm>
#include <climits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "apar_internal.h"
#include "kv4.cuh"
#include "ptx.cuh"

namespace apar {
namespace {

constexpr int kRows = kQ4Rows;                       // query rows of a unit
constexpr int kWarps = kQ4Streams;
constexpr int kStep = 2;                             // blocks computed together
constexpr int kTile = 2 * kQ4TileBytes;              // K and V of one block
constexpr int kSlot = kStep * kTile;
constexpr int kDepth = 3;                            // slots of a warp's ring
constexpr int kHdrs = 4;                             // unit descriptions a warp holds
constexpr int kHdrInts = 32;
constexpr int kOffQ = kWarps * kDepth * kSlot;       // the next unit's query rows, per warp
constexpr int kOffHdr = kOffQ + kWarps * kRows * kDim * 2;
constexpr int kSmemQ4 = kOffHdr + kWarps * kHdrs * kHdrInts * 4;
static_assert(kSmemQ4 <= 227 * 1024, "shared memory");
constexpr float kHeadroom = 12.f;                    // largest weight when the reference is set: 2^12
constexpr float kSlack = 15.5f;                      // and when it has to move: 2^15.5 (times 2^0.1)
constexpr float kNoRef = -3e38f;                      // of a row that has seen nothing (finite: a
                                                     // masked score less this is still -inf)
constexpr float kCodeUnit = 1.f / 16777216.f;        // what a code of 1 counts as in a product: 2^-24
constexpr uint32_t kEven = 0x000f000fu;             // nibbles 0 and 4 of a word: f16 pair c * 2^-24
constexpr uint32_t kOdd = 0x00f000f0u;              // nibbles 1 and 5: c * 2^-20
constexpr uint32_t kUpEven = 0x78007800u, kUpOdd = 0x68006800u;   // f16 pairs 2^15 and 2^11: bring
                                                     // c * 2^-24 and c * 2^-20 to c * 2^-9
constexpr uint32_t kLessMiddle = 0xa380a380u;        // f16 pair -7.5 * 2^-9
constexpr float kValueUnit = 512.f;                  // 2^9
constexpr float kMinScaleLog2 = -60.f;               // V scales below 2^-60 count as 2^-60

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                        uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                         uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
      "{%8,%9}, {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  __half2 h = __floats2half2_rn(lo, hi);
  return *(uint32_t*)&h;
}
__device__ __forceinline__ uint32_t fma_f16(uint32_t a, uint32_t b, uint32_t c) {
  __half2 r = __hfma2(*(__half2*)&a, *(__half2*)&b, *(__half2*)&c);
  return *(uint32_t*)&r;
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a));
  return v;
}

// words of a unit description; query and slot of row r at H_QUERY + r, H_SLOT + r
enum { H_ROW = 0, H_BEGIN = 1, H_TOK = 2, H_NUSERS = 4, H_ADD = 5, H_KVH = 9, H_BID = 10, H_TAB = 12,
       H_QUERY = 16, H_SLOT = 24 };                  // (H_BID: the first two block ids)

// One warp's share of the units of a launch.
//
// kNarrow: units of at most four rows.  Columns 0-3 carry the rows over a step's first block,
// columns 4-7 the same rows over its second one, as if they were other rows (they meet at the end
// of the unit): S^T of both blocks comes out of one accumulator, because each block is
// multiplied with the queries in its own columns and zeros in the others, and everything that is
// done per score is done once for both.  A lane's block is q / 2.  For O^T the weights of the other
// block's columns are masked out of the B operand.
template <bool kNarrow>
__device__ __forceinline__ void stream_units(const AttnArgs& a, const Q4Units& units, uint8_t* smem) {
  constexpr int kSets = kNarrow ? 2 : 1;             // query operands
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, q = lane & 3;
  const int G = a.shape.group, HQ = a.shape.num_q_heads, HKV = a.shape.num_kv_heads;
  const uint32_t ring = s32(smem) + warp * kDepth * kSlot;
  const uint32_t qrows = s32(smem) + kOffQ + warp * kRows * kDim * 2;
  int* const hdrs = (int*)(smem + kOffHdr) + warp * kHdrs * kHdrInts;
  auto hdr = [&](int seq) { return hdrs + (seq & (kHdrs - 1)) * kHdrInts; };
  const int n_units = kNarrow ? units.narrow_units : units.mid_units;

  // ---- descriptions, one phase per call: item; its users, first block ids and length; stored
  int f_seq = 0, f_phase = 0, f_pass = 0;            // units described so far; pass over the list
  bool f_end = n_units == 0;
  int t0 = 0, t1 = 0, t2 = 0, t4 = 0, f_kvh = 0;
  uint2 t3 = make_uint2(0u, 0u);
  auto fetch_step = [&]() {
    if (f_phase == 0) {
      const int W = gridDim.x * kWarps, w = warp * gridDim.x + blockIdx.x;
      const int u = f_pass * W + ((f_pass & 1) ? W - 1 - w : w);
      ++f_pass;
      if (u >= n_units) {
        f_end = (long long)f_pass * W >= n_units;    // (a backward pass may start past the end)
        return;
      }
      f_kvh = u % HKV;
      t0 = lane < 8 ? __ldg((const int*)(a.d_items + (kNarrow ? units.narrow_begin : units.mid_begin) +
                                         u / HKV) + lane) : 0;
      f_phase = 1;
    } else if (f_phase == 1) {
      const int row = __shfl_sync(0xffffffffu, t0, 0), begin = __shfl_sync(0xffffffffu, t0, 1);
      const int end = __shfl_sync(0xffffffffu, t0, 2), ub = __shfl_sync(0xffffffffu, t0, 3);
      const int R = __shfl_sync(0xffffffffu, t0, 4) * G;
      t1 = (end < 0 ? a.d_lens[row] : end) - begin;
      const int32_t* tab = a.d_tables + (size_t)row * a.shape.table_stride;
      t2 = tab[begin / kBlock];
      t4 = tab[min(begin / kBlock + 1, a.shape.table_stride - 1)];   // (unused if there is none)
      const int r = lane & 7;
      t3 = make_uint2(0u, 0u);
      if (r < R) t3 = *(const uint2*)(a.d_users + ub + r / G);
      f_phase = 2;
    } else {
      int* h = hdr(f_seq);
      const int row = __shfl_sync(0xffffffffu, t0, 0), begin = __shfl_sync(0xffffffffu, t0, 1);
      if (lane < 8 && lane != H_TOK) h[lane] = t0;
      if (lane == 8) {
        h[H_TOK] = t1;
        h[H_KVH] = f_kvh;
        h[H_BID] = t2;
        h[H_BID + 1] = t4;
        *(const int32_t**)(h + H_TAB) = a.d_tables + (size_t)row * a.shape.table_stride + begin / kBlock;
      }
      if (lane >= 16) h[lane] = lane < 24 ? (int)t3.x : (int)t3.y;
      __syncwarp();
      ++f_seq;
      f_phase = 0;
    }
  };

  // ---- loads: at most one unit ahead of the one that is computed, and not before that one's
  // query rows have been read (the next unit's take their place)
  int c_seq = 0, k = 0;                              // the unit being computed; its next block
  int l_seq = -1, l_k = 0, l_n = 0, l_bid = 0, l_bid1 = 0;
  int issue_slot = 0, use_slot = 0, ahead = 0;       // steps requested and not computed
  auto issue_block = [&](int bid, uint32_t dst) {
    const size_t tile = ((size_t)bid * HKV + hdr(l_seq)[H_KVH]) * kQ4TileBytes + lane * 16;
    const uint8_t* kt = (const uint8_t*)a.k_pool + tile;
    const uint8_t* vt = (const uint8_t*)a.v_pool + tile - kQ4TileBytes;
    cp_async16(dst, kt);
    cp_async16(dst + 512, kt + 512);
    cp_async16(dst + 1024, (lane < 16 ? kt : vt) + 1024);
    cp_async16(dst + 1536, vt + 1536);
    cp_async16(dst + 2048, vt + 2048);
  };
  auto issue = [&]() {                               // blocks l_k and l_k + 1 of the loads' unit
    const uint32_t dst = ring + issue_slot * kSlot + lane * 16;
    issue_block(l_bid, dst);
    if (l_k + 1 < l_n) issue_block(l_bid1, dst + kTile);
    asm volatile("cp.async.commit_group;" ::: "memory");
    issue_slot = issue_slot == kDepth - 1 ? 0 : issue_slot + 1;
    ++ahead;
    l_k += kStep;
    if (l_k < l_n) {                                 // (arrive while a step is computed)
      const int32_t* tab = *(const int32_t**)(hdr(l_seq) + H_TAB);
      l_bid = tab[l_k];
      l_bid1 = tab[min(l_k + 1, l_n - 1)];
    }
  };
  auto next_unit = [&]() -> bool {                   // moves the loads on to it
    if (l_seq > c_seq || (l_seq == c_seq && k == 0)) return false;
    while (f_seq <= l_seq + 1 && !f_end) fetch_step();
    if (f_seq <= l_seq + 1) return false;            // no more units
    const int* h = hdr(++l_seq);
    l_n = (h[H_TOK] + kBlock - 1) / kBlock;
    l_k = 0;
    l_bid = h[H_BID];
    l_bid1 = h[H_BID + 1];
    // the query rows, committed with the first tile: half a warp copies one
    const int rows = h[H_NUSERS] * G;
#pragma unroll
    for (int j = 0; j < (kNarrow ? kRows / 4 : kRows / 2); ++j) {
      const int r = 2 * j + (lane >> 4);
      if (r < rows)
        cp_async16(qrows + r * kDim * 2 + (lane & 15) * 16,
                   (const uint4*)a.q + ((size_t)h[H_QUERY + r] * HQ + h[H_KVH] * G + r % G) * 16 + (lane & 15));
    }
    return true;
  };

  // ---- state of the unit being computed
  uint32_t qb[kSets][4][4];      // the column's row, dims 32 j + 8 q .. + 7, as B fragments
  uint32_t qsum[kSets][2];       // its sum over group q as three bf16 numbers
  float unit[2];                 // rows 2 q, 2 q + 1: scale * 2^24 / their factor
  float o[8][4], lsum[4][2], ref[2], l[2];

#pragma unroll 1
  for (;;) {
    __syncwarp();                // (the tiles and the description read last may be overwritten)
    if (k < 4 * kStep && !f_end && f_seq < c_seq + kHdrs) fetch_step();
#pragma unroll 1
    do {                         // (once, but for the start and units too short to run ahead of)
      if (l_k >= l_n && !next_unit()) break;
      issue();
    } while (ahead < kDepth);
    if (ahead == 0) break;
    if (ahead == kDepth) asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 1) : "memory");
    else asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();

    if (k == 0) {                // ---- a unit begins
      const int rows = hdr(c_seq)[H_NUSERS] * G;
      const int r = kNarrow ? g & 3 : g;
      uint32_t top = 0;          // bits of the row's largest magnitude, without the sign
      uint4 v[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        v[j] = make_uint4(0u, 0u, 0u, 0u);
        if (r < rows) v[j] = lds128(qrows + r * kDim * 2 + (32 * j + 8 * q) * 2);
        const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
#pragma unroll
        for (int p = 0; p < 4; ++p) top = max(top, max(w[p] << 17, (w[p] & 0x7fff0000u) << 1));
      }
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      // the factor 2^lift; a row of zeros or subnormal numbers has it at its limit
      const int lift = min(126, 14 + 127 - (int)(top >> 24));
      const float f = __uint_as_float((uint32_t)(lift + 127) << 23);
      float mine = 0.f;          // the sum over group q
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t w[4] = {v[j].x, v[j].y, v[j].z, v[j].w};
        float x = 0.f;
#pragma unroll
        for (int p = 0; p < 4; ++p) {
          const float e0 = bf16_lo(w[p]) * f, e1 = bf16_hi(w[p]) * f;
          x += e0 + e1;
          const uint32_t b = (p & 1) ? pack_f16(e0 * 0.0625f, e1 * 0.0625f) : pack_f16(e0, e1);
          qb[0][j][p] = kNarrow && g >= 4 ? 0u : b;
          if (kNarrow) qb[kSets - 1][j][p] = g >= 4 ? b : 0u;
        }
        x += __shfl_xor_sync(0xffffffffu, x, 1);
        x += __shfl_xor_sync(0xffffffffu, x, 2);
        if (j == q) mine = x * kCodeUnit;
      }
      const float m0 = __bfloat162float(__float2bfloat16_rn(mine)), m1 = mine - m0;
      const uint32_t s0 = pack2(m0, m1);
      const uint32_t s1 = pack2(m1 - __bfloat162float(__float2bfloat16_rn(m1)), 0.f);
      qsum[0][0] = kNarrow && g >= 4 ? 0u : s0;
      qsum[0][1] = kNarrow && g >= 4 ? 0u : s1;
      if (kNarrow) {
        qsum[kSets - 1][0] = g >= 4 ? s0 : 0u;
        qsum[kSets - 1][1] = g >= 4 ? s1 : 0u;
      }
      // score * log2(e) * scale = (what the products give) * unit; never 0, so that the -inf of
      // a masked score stays one
      float u = a.scale_log2e * (1.f / kCodeUnit) * __uint_as_float((uint32_t)(127 - lift) << 23);
      if (fabsf(u) < 1.17549435e-38f) u = 1.17549435e-38f;
      unit[0] = __shfl_sync(0xffffffffu, u, 8 * q);
      unit[1] = __shfl_sync(0xffffffffu, u, 8 * q + 4);
#pragma unroll
      for (int m = 0; m < 8; ++m)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[m][e] = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) lsum[j][0] = lsum[j][1] = 0.f;
      ref[0] = ref[1] = kNoRef;
      l[0] = l[1] = 0.f;
    }
    const uint32_t tile0 = ring + use_slot * kSlot;
    const int nv = hdr(c_seq)[H_TOK] - k * kBlock;   // tokens from this step on

    // ---- pieces of a step.  Scores are those of tokens g and g + 8 of a block for rows 2 q and
    // 2 q + 1, up to the factor `unit`.
    auto offsets = [&](uint32_t kt, int n, const uint32_t (&sum)[2], float (&x)[4]) {
      uint32_t lo0 = lds32(kt + g * kQ4RowBytes + kQ4CodeBytes + 4 * q);
      uint32_t lo1 = lds32(kt + (g + 8) * kQ4RowBytes + kQ4CodeBytes + 4 * q);
      if (kNarrow && n < kBlock) {   // (unspecified bits may be NaN, and meet the other columns' zeros)
        if (g >= n) lo0 = 0u;
        if (g + 8 >= n) lo1 = 0u;
      }
      const uint32_t a0 = __byte_perm(lo0, 0u, 0x3232), a1 = __byte_perm(lo1, 0u, 0x3232);
      mma_bf16(x, a0, a1, a0, a1, sum[0], sum[1]);
    };
    auto dot = [&](uint32_t w0, uint32_t w1, const uint32_t (&b)[4], float (&acc)[4]) {
      const uint32_t h0 = w0 >> 8, h1 = w1 >> 8;
      mma_f16(acc, w0 & kEven, w1 & kEven, w0 & kOdd, w1 & kOdd, b[0], b[1]);
      mma_f16(acc, h0 & kEven, h1 & kEven, h0 & kOdd, h1 & kOdd, b[2], b[3]);
    };
    auto scale_add = [&](uint32_t s0, uint32_t s1, const float (&acc)[4], float (&x)[4]) {
      const float sa = bf16_lo(s0), sb = bf16_lo(s1);
      x[0] = fmaf(sa, acc[0], x[0]);
      x[1] = fmaf(sa, acc[1], x[1]);
      x[2] = fmaf(sb, acc[2], x[2]);
      x[3] = fmaf(sb, acc[3], x[3]);
    };
    // V scales of the same tokens; rows past the length hold unspecified bits.  n: tokens that count
    auto v_scales = [&](uint32_t vt, int n, uint32_t (&z)[2][4], float (&x)[4]) {
      const uint32_t at = vt + (g >> 1) * kQ4PairBytes + 2 * kQ4CodeBytes + 16 * (g & 1);
      const uint4 v0 = lds128(at), v1 = lds128(at + 4 * kQ4PairBytes);
      z[0][0] = v0.x; z[0][1] = v0.y; z[0][2] = v0.z; z[0][3] = v0.w;
      z[1][0] = v1.x; z[1][1] = v1.y; z[1][2] = v1.z; z[1][3] = v1.w;
      if (n < kBlock) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
          if (g + 8 * e >= n) {
            x[2 * e] = copysignf(INFINITY, -unit[0]);
            x[2 * e + 1] = copysignf(INFINITY, -unit[1]);
            z[e][0] = z[e][1] = z[e][2] = z[e][3] = 0u;
          }
      }
    };
    // score + log2 of the token's largest scale (from the bits of the number, below by at most 0.09)
    auto tops = [&](const uint32_t (&z)[2][4], const float (&x)[4], float& y0, float& y1) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int top = max(max(max((int)(z[e][0] << 16), (int)(z[e][1] << 16)),
                                (int)(z[e][2] << 16)), (int)(z[e][3] << 16));
        const float sl = fmaxf(fmaf((float)top, 1.f / 8388608.f, -127.f), kMinScaleLog2);
        y0 = fmaxf(y0, fmaf(x[2 * e], unit[0], sl));
        y1 = fmaxf(y1, fmaf(x[2 * e + 1], unit[1], sl));
      }
    };
    auto move_reference = [&](float y0, float y1) {
      if (!__any_sync(0xffffffffu, y0 > ref[0] + kSlack || y1 > ref[1] + kSlack)) return;
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) {
        y0 = fmaxf(y0, __shfl_xor_sync(0xffffffffu, y0, d));
        y1 = fmaxf(y1, __shfl_xor_sync(0xffffffffu, y1, d));
      }
      y0 = fmaxf(y0 - kHeadroom, ref[0]);
      y1 = fmaxf(y1 - kHeadroom, ref[1]);
      const float f0 = ex2(ref[0] - y0), f1 = ex2(ref[1] - y1);
      ref[0] = y0;
      ref[1] = y1;
      l[0] *= f0;
      l[1] *= f1;
#pragma unroll
      for (int m = 0; m < 8; ++m) {
        o[m][0] *= f0; o[m][1] *= f1; o[m][2] *= f0; o[m][3] *= f1;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        lsum[j][0] *= f0;
        lsum[j][1] *= f1;
      }
    };
    auto weights = [&](float (&x)[4]) {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = ex2(fmaf(x[e], unit[e & 1], -ref[e & 1]));
      l[0] += x[0] + x[2];
      l[1] += x[1] + x[3];
    };
    // the B operand of group j, and the middles' share
    auto weights_b = [&](uint32_t z0, uint32_t z1, const float (&p)[4], int j, uint32_t& b0,
                         uint32_t& b1) {
      const float sa = bf16_lo(z0), sb = bf16_lo(z1);
      b0 = transpose8x8(pack_f16(p[0] * sa, p[1] * sa));
      b1 = transpose8x8(pack_f16(p[2] * sb, p[3] * sb));
      const float la = fmaf(7.5f, sa, bf16_hi(z0)), lb = fmaf(7.5f, sb, bf16_hi(z1));
      lsum[j][0] = fmaf(p[0], la, fmaf(p[2], lb, lsum[j][0]));
      lsum[j][1] = fmaf(p[1], la, fmaf(p[3], lb, lsum[j][1]));
    };
    auto accumulate = [&](uint32_t xl, uint32_t xh, uint32_t b0, uint32_t b1, float (&d0)[4],
                          float (&d1)[4]) {
      const uint32_t hl = xl >> 8, hh = xh >> 8;
      auto even = [](uint32_t w) { return fma_f16(w & kEven, kUpEven, kLessMiddle); };
      auto odd = [](uint32_t w) { return fma_f16(w & kOdd, kUpOdd, kLessMiddle); };
      mma_f16(d0, even(xl), odd(xl), even(xh), odd(xh), b0, b1);
      mma_f16(d1, even(hl), odd(hl), even(hh), odd(hh), b0, b1);
    };
    auto k_words = [&](uint32_t kt, uint4& w0, uint4& w1) {
      w0 = lds128(kt + g * kQ4RowBytes + q * 16);
      w1 = lds128(kt + (g + 8) * kQ4RowBytes + q * 16);
    };
    auto v_words = [&](uint32_t vt, uint4& w0, uint4& w1) {      // pairs q and q + 4
      w0 = lds128(vt + q * kQ4PairBytes + g * 16);
      w1 = lds128(vt + (q + 4) * kQ4PairBytes + g * 16);
    };

    if (kNarrow) {
      const uint32_t mine = tile0 + (q >> 1) * kTile;
      float x[4] = {0.f, 0.f, 0.f, 0.f};
      offsets(tile0, nv, qsum[0], x);
      offsets(tile0 + kTile, nv - kBlock, qsum[kSets - 1], x);
      {
        uint4 a0, a1, c0, c1;
        k_words(tile0, a0, a1);
        k_words(tile0 + kTile, c0, c1);
        const uint4 s0 = lds128(mine + g * kQ4RowBytes + kQ4CodeBytes);
        const uint4 s1 = lds128(mine + (g + 8) * kQ4RowBytes + kQ4CodeBytes);
        const uint32_t wa[4] = {a0.x, a0.y, a0.z, a0.w}, wb[4] = {a1.x, a1.y, a1.z, a1.w};
        const uint32_t wc[4] = {c0.x, c0.y, c0.z, c0.w}, wd[4] = {c1.x, c1.y, c1.z, c1.w};
        const uint32_t sa[4] = {s0.x, s0.y, s0.z, s0.w}, sb[4] = {s1.x, s1.y, s1.z, s1.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float acc[4] = {};
          dot(wa[j], wb[j], qb[0][j], acc);
          dot(wc[j], wd[j], qb[kSets - 1][j], acc);
          scale_add(sa[j], sb[j], acc, x);
        }
      }
      uint32_t z[2][4];
      v_scales(mine + kQ4TileBytes, nv - (q >> 1) * kBlock, z, x);
      float y0 = -INFINITY, y1 = -INFINITY;
      tops(z, x, y0, y1);
      move_reference(y0, y1);
      weights(x);
      uint4 v0, v1, v2, v3;
      v_words(tile0 + kQ4TileBytes, v0, v1);
      v_words(tile0 + kTile + kQ4TileBytes, v2, v3);
      const uint32_t al[4] = {v0.x, v0.y, v0.z, v0.w}, ah[4] = {v1.x, v1.y, v1.z, v1.w};
      const uint32_t cl[4] = {v2.x, v2.y, v2.z, v2.w}, ch[4] = {v3.x, v3.y, v3.z, v3.w};
      const uint32_t first_columns = g < 4 ? ~0u : 0u;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t b0, b1;
        weights_b(z[0][j], z[1][j], x, j, b0, b1);
        const uint32_t c0 = b0 & first_columns, c1 = b1 & first_columns;
        accumulate(al[j], ah[j], c0, c1, o[2 * j], o[2 * j + 1]);
        accumulate(cl[j], ch[j], b0 ^ c0, b1 ^ c1, o[2 * j], o[2 * j + 1]);
      }
    } else {
      float x[kStep][4];
      uint32_t z[kStep][2][4];
      float y0 = -INFINITY, y1 = -INFINITY;
#pragma unroll
      for (int b = 0; b < kStep; ++b) {
        const uint32_t kt = tile0 + b * kTile;
        uint4 w0, w1;
        k_words(kt, w0, w1);
        const uint4 s0 = lds128(kt + g * kQ4RowBytes + kQ4CodeBytes);
        const uint4 s1 = lds128(kt + (g + 8) * kQ4RowBytes + kQ4CodeBytes);
        const uint32_t wa[4] = {w0.x, w0.y, w0.z, w0.w}, wb[4] = {w1.x, w1.y, w1.z, w1.w};
        const uint32_t sa[4] = {s0.x, s0.y, s0.z, s0.w}, sb[4] = {s1.x, s1.y, s1.z, s1.w};
        x[b][0] = x[b][1] = x[b][2] = x[b][3] = 0.f;
        offsets(kt, nv - b * kBlock, qsum[0], x[b]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          float acc[4] = {};
          dot(wa[j], wb[j], qb[0][j], acc);
          scale_add(sa[j], sb[j], acc, x[b]);
        }
      }
#pragma unroll
      for (int b = 0; b < kStep; ++b) {
        v_scales(tile0 + b * kTile + kQ4TileBytes, nv - b * kBlock, z[b], x[b]);
        tops(z[b], x[b], y0, y1);
      }
      move_reference(y0, y1);
#pragma unroll
      for (int b = 0; b < kStep; ++b) weights(x[b]);
#pragma unroll
      for (int b = 0; b < kStep; ++b) {
        uint4 w0, w1;
        v_words(tile0 + b * kTile + kQ4TileBytes, w0, w1);
        const uint32_t xl[4] = {w0.x, w0.y, w0.z, w0.w}, xh[4] = {w1.x, w1.y, w1.z, w1.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          uint32_t b0, b1;
          weights_b(z[b][0][j], z[b][1][j], x[b], j, b0, b1);
          accumulate(xl[j], xh[j], b0, b1, o[2 * j], o[2 * j + 1]);
        }
      }
    }
    --ahead;
    use_slot = use_slot == kDepth - 1 ? 0 : use_slot + 1;
    k += kStep;
    if (nv > kStep * kBlock) continue;

    // ---- end of the unit: sums over the lanes that hold other tokens of the same rows
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) {
      l[0] += __shfl_xor_sync(0xffffffffu, l[0], d);
      l[1] += __shfl_xor_sync(0xffffffffu, l[1], d);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        lsum[j][0] += __shfl_xor_sync(0xffffffffu, lsum[j][0], d);
        lsum[j][1] += __shfl_xor_sync(0xffffffffu, lsum[j][1], d);
      }
    }
    if (kNarrow) {               // row r over the first blocks and over the second: lanes q and q ^ 2
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float other = __shfl_xor_sync(0xffffffffu, ref[e], 2);
        const float m = fmaxf(ref[e], other);
        const float f = ref[e] == m ? 1.f : ex2(ref[e] - m);   // (no second block: kNoRef and zeros)
        ref[e] = m;
        l[e] *= f;
        l[e] += __shfl_xor_sync(0xffffffffu, l[e], 2);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          lsum[j][e] *= f;
          lsum[j][e] += __shfl_xor_sync(0xffffffffu, lsum[j][e], 2);
        }
#pragma unroll
        for (int m8 = 0; m8 < 8; ++m8)
#pragma unroll
          for (int x = e; x < 4; x += 2) {
            o[m8][x] *= f;
            o[m8][x] += __shfl_xor_sync(0xffffffffu, o[m8][x], 2);
          }
      }
    }
    // ---- row 2 q + e: dims 32 j + 4 g .. + 3, to the output or to a partial result
    const int* h = hdr(c_seq);
    const int rows = h[H_NUSERS] * G;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = 2 * q + e;
      if (r >= rows) continue;
      const int head = h[H_KVH] * G + r % G;
      const int query = h[H_QUERY + r], slot = h[H_SLOT + r];
      const float inv = slot < 0 ? 1.f / l[e] : 1.f;
      const size_t prow = (size_t)(slot + h[H_ADD]) * HQ + head;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float4 v = make_float4(fmaf(o[2 * j][e], kValueUnit, lsum[j][e]) * inv,
                                     fmaf(o[2 * j][2 + e], kValueUnit, lsum[j][e]) * inv,
                                     fmaf(o[2 * j + 1][e], kValueUnit, lsum[j][e]) * inv,
                                     fmaf(o[2 * j + 1][2 + e], kValueUnit, lsum[j][e]) * inv);
        if (slot < 0)
          *(uint2*)((__nv_bfloat16*)a.out + ((size_t)query * HQ + head) * kDim + 32 * j + 4 * g) =
              make_uint2(pack2(v.x, v.y), pack2(v.z, v.w));
        else
          *(float4*)(a.part_o + prow * kDim + 32 * j + 4 * g) = v;
      }
      if (slot >= 0 && g == 0) a.part_ml[prow] = make_float2(ref[e], l[e]);
    }
    ++c_seq;
    k = 0;
  }
}

__global__ void __launch_bounds__(32 * kWarps, 1)
attn_q4_kernel(const AttnArgs a, const Q4Units units) {
  extern __shared__ __align__(128) uint8_t smem[];
  pdl_launch_dependents();
  stream_units<false>(a, units, smem);
  __syncwarp();
  stream_units<true>(a, units, smem);
  pdl_wait();                        // "this grid has completed" implies the one before it has
}

// End of a verification, one warp per candidate and kHeads heads of one kv head: the candidates it
// sees, read straight from the 4-bit pool, and the partial results of the committed tokens before
// them, folded into the output.  The halves of the warp take the set bits of the mask in turn (a
// candidate of a tree sees few others), and the partial results too; lane c of a half holds dims
// 8 c .. 8 c + 7.  What it reads first depends on nothing the attention kernels write, so it may
// start before them.  Turning the rows into numbers is what costs: heads that share them share it.
template <int kHeads>
__global__ void __launch_bounds__(128) q4_verify_finish_kernel(const AttnArgs a,
                                                               const VerifyDesc* __restrict__ descs) {
  const VerifyDesc d = descs[blockIdx.x];
  const int G = a.shape.group, HQ = a.shape.num_q_heads, HKV = a.shape.num_kv_heads;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int half = lane >> 4, c = lane & 15;
  const int head0 = (blockIdx.y * 4 + warp) * kHeads;
  if (head0 >= HQ) return;
  const int kvh = head0 / G;
  const int32_t* table = a.d_tables + (size_t)d.row * a.shape.table_stride;
  float qf[kHeads][8], o[kHeads][8], m[kHeads], l[kHeads];   // m, l of this half
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    const uint4 qv = __ldg((const uint4*)a.q + ((size_t)d.query * HQ + head0 + h) * 16 + c);
    const uint32_t w[4] = {qv.x, qv.y, qv.z, qv.w};
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      qf[h][2 * x] = bf16_lo(w[x]) * a.scale_log2e;
      qf[h][2 * x + 1] = bf16_hi(w[x]) * a.scale_log2e;
      o[h][2 * x] = o[h][2 * x + 1] = 0.f;
    }
    m[h] = -INFINITY;
    l[h] = 0.f;
  }
  uint64_t left = d.mask;
  while (left) {
    // two candidates per half at a time
    constexpr int kSums = 2 * kHeads;                // sum n * kHeads + h: candidate n, head h
    float t[kSums], vf[2][8];
    bool on[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      const int i_first = __ffsll((long long)left) - 1;
      const bool any = left != 0;
      left &= left - 1;                              // (0 stays 0)
      const int i_second = __ffsll((long long)left) - 1;
      const bool two = left != 0;
      left &= left - 1;
      on[n] = half ? two : any;
#pragma unroll
      for (int h = 0; h < kHeads; ++h) t[n * kHeads + h] = 0.f;
#pragma unroll
      for (int x = 0; x < 8; ++x) vf[n][x] = 0.f;
      if (on[n]) {
        const int pos = d.base + (half ? i_second : i_first);
        const size_t tile = ((size_t)table[pos >> 4] * HKV + kvh) * kQ4TileBytes;
        float kf[8];
        q4_load8_k((const uint8_t*)a.k_pool + tile, pos & (kBlock - 1), c, kf);
        q4_load8_v((const uint8_t*)a.v_pool + tile, pos & (kBlock - 1), c, vf[n]);
#pragma unroll
        for (int h = 0; h < kHeads; ++h)
#pragma unroll
          for (int x = 0; x < 8; ++x) t[n * kHeads + h] = fmaf(qf[h][x], kf[x], t[n * kHeads + h]);
      }
    }
    // sums over the 16 lanes: each step halves the sums a lane carries, then lane i 16 / kSums has i
#pragma unroll
    for (int x = 8, left_of = kSums; x; x >>= 1) {
      left_of >>= 1;
      if (left_of) {
#pragma unroll
        for (int i = 0; i < kSums / 2; ++i)
          if (i < left_of) {
            const bool up = c & x;
            const float give = up ? t[i] : t[i + left_of], keep = up ? t[i + left_of] : t[i];
            t[i] = keep + __shfl_xor_sync(0xffffffffu, give, x);
          }
      } else {
        t[0] += __shfl_xor_sync(0xffffffffu, t[0], x);
      }
    }
    const float own = t[0];
#pragma unroll
    for (int i = 0; i < kSums; ++i) {
      t[i] = __shfl_sync(0xffffffffu, own, i * (16 / kSums), 16);
      if (!on[i / kHeads]) t[i] = -INFINITY;
    }
#pragma unroll
    for (int h = 0; h < kHeads; ++h) {
      const float t0 = t[h], t1 = t[kHeads + h];
      const float mn = fmaxf(m[h], fmaxf(t0, t1));
      const float corr = m[h] == -INFINITY ? 0.f : ex2(m[h] - mn);
      const float p0 = on[0] ? ex2(t0 - mn) : 0.f, p1 = on[1] ? ex2(t1 - mn) : 0.f;
      m[h] = mn;
      l[h] = fmaf(l[h], corr, p0 + p1);
#pragma unroll
      for (int x = 0; x < 8; ++x) o[h][x] = fmaf(p0, vf[0][x], fmaf(p1, vf[1][x], o[h][x] * corr));
    }
  }
  pdl_wait();                                        // partial results of the attention kernels
#pragma unroll
  for (int h = 0; h < kHeads; ++h) {
    const int head = head0 + h;
    for (int j0 = half; j0 < d.parts; j0 += 4) {     // two per half at a time
      float2 ml[2];
      float4 x0[2], x1[2];
      float mn = m[h];
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const int j = j0 + 2 * n;
        ml[n] = make_float2(-INFINITY, 0.f);
        x0[n] = x1[n] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (j < d.parts) {
          const size_t prow = (size_t)(d.slot - d.parts + j) * HQ + head;
          ml[n] = a.part_ml[prow];
          const float4* src = (const float4*)(a.part_o + prow * kDim) + 2 * c;
          x0[n] = src[0];
          x1[n] = src[1];
        }
      }
#pragma unroll
      for (int n = 0; n < 2; ++n) mn = fmaxf(mn, ml[n].x);
      const float corr = m[h] == -INFINITY ? 0.f : ex2(m[h] - mn);
      m[h] = mn;
      l[h] *= corr;
#pragma unroll
      for (int x = 0; x < 8; ++x) o[h][x] *= corr;
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        const float w = ml[n].x == -INFINITY ? 0.f : ex2(ml[n].x - mn);
        l[h] = fmaf(ml[n].y, w, l[h]);
        o[h][0] = fmaf(x0[n].x, w, o[h][0]); o[h][1] = fmaf(x0[n].y, w, o[h][1]);
        o[h][2] = fmaf(x0[n].z, w, o[h][2]); o[h][3] = fmaf(x0[n].w, w, o[h][3]);
        o[h][4] = fmaf(x1[n].x, w, o[h][4]); o[h][5] = fmaf(x1[n].y, w, o[h][5]);
        o[h][6] = fmaf(x1[n].z, w, o[h][6]); o[h][7] = fmaf(x1[n].w, w, o[h][7]);
      }
    }
    __syncwarp();
    const float M = fmaxf(m[h], __shfl_xor_sync(0xffffffffu, m[h], 16));
    const float f = m[h] == -INFINITY ? 0.f : ex2(m[h] - M);   // (a half may have seen nothing)
    l[h] *= f;
    l[h] += __shfl_xor_sync(0xffffffffu, l[h], 16);
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      o[h][x] *= f;
      o[h][x] += __shfl_xor_sync(0xffffffffu, o[h][x], 16);
    }
    const float inv = 1.f / l[h];                    // (a candidate sees itself)
    if (half == 0)
      *((uint4*)((__nv_bfloat16*)a.out + ((size_t)d.query * HQ + head) * kDim) + c) =
          make_uint4(pack2(o[h][0] * inv, o[h][1] * inv), pack2(o[h][2] * inv, o[h][3] * inv),
                     pack2(o[h][4] * inv, o[h][5] * inv), pack2(o[h][6] * inv, o[h][7] * inv));
  }
}

// out = sum_j o_j 2^(m_j - M) / sum_j l_j 2^(m_j - M) over the partial results of one (query, head).
// kWarpsPerRow warps share a row's parts (1: four rows to a CTA); (m, l) and o of kRound parts a warp
// are requested together, so that a row of few parts costs one trip to memory.
template <int kWarpsPerRow, int kRound>
__global__ void __launch_bounds__(128) q4_merge_kernel(const AttnArgs a,
                                                       const MergeRef* __restrict__ merges) {
  __shared__ float sm_m[4], sm_l[4];
  __shared__ __align__(16) float sm_o[kWarpsPerRow > 1 ? 4 : 1][kDim];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int HQ = a.shape.num_q_heads;
  const int head = kWarpsPerRow == 1 ? blockIdx.y * 4 + warp : blockIdx.y;
  const MergeRef mr = merges[blockIdx.x];
  pdl_wait();                                        // (the attention launch before this one)
  if (head >= HQ) return;                            // (whole warps, and only where rows are warps)
  float M = -INFINITY, L = 0.f;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int j0 = kWarpsPerRow == 1 ? 0 : warp; j0 < mr.n; j0 += kRound * kWarpsPerRow) {
    float2 ml[kRound];
    float4 o[kRound];
#pragma unroll
    for (int k = 0; k < kRound; ++k) {
      const int j = j0 + k * kWarpsPerRow;
      ml[k] = make_float2(-INFINITY, 0.f);
      o[k] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (j < mr.n) {
        const size_t prow = (size_t)(mr.slot_begin + j) * HQ + head;
        ml[k] = a.part_ml[prow];
        o[k] = ((const float4*)(a.part_o + prow * kDim))[lane];
      }
    }
    float m = M;
#pragma unroll
    for (int k = 0; k < kRound; ++k) m = fmaxf(m, ml[k].x);
    const float f = M == -INFINITY ? 0.f : ex2(M - m);
    M = m;
    L *= f;
    acc.x *= f; acc.y *= f; acc.z *= f; acc.w *= f;
#pragma unroll
    for (int k = 0; k < kRound; ++k) {
      const float w = ml[k].x == -INFINITY ? 0.f : ex2(ml[k].x - m);
      L = fmaf(ml[k].y, w, L);
      acc.x = fmaf(o[k].x, w, acc.x); acc.y = fmaf(o[k].y, w, acc.y);
      acc.z = fmaf(o[k].z, w, acc.z); acc.w = fmaf(o[k].w, w, acc.w);
    }
  }
  if (kWarpsPerRow > 1) {
    if (lane == 0) {
      sm_m[warp] = M;
      sm_l[warp] = L;
    }
    *(float4*)&sm_o[warp][4 * lane] = acc;
    __syncthreads();
    if (warp > 0) return;
    const float m = fmaxf(fmaxf(sm_m[0], sm_m[1]), fmaxf(sm_m[2], sm_m[3]));
    L = 0.f;
    acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = sm_m[w] == -INFINITY ? 0.f : ex2(sm_m[w] - m);
      const float4 v = *(const float4*)&sm_o[w][4 * lane];
      L = fmaf(sm_l[w], f, L);
      acc.x = fmaf(v.x, f, acc.x); acc.y = fmaf(v.y, f, acc.y);
      acc.z = fmaf(v.z, f, acc.z); acc.w = fmaf(v.w, f, acc.w);
    }
  }
  const float inv = 1.f / L;
  *((uint2*)((__nv_bfloat16*)a.out + ((size_t)mr.query * HQ + head) * kDim) + lane) =
      make_uint2(pack2(acc.x * inv, acc.y * inv), pack2(acc.z * inv, acc.w * inv));
}

}  // namespace

cudaError_t launch_q4_merge(const AttnArgs& a, const MergeRef* d_merge, int n_merge, int max_parts,
                            cudaStream_t st) {
  if (n_merge <= 0) return cudaSuccess;
  const int HQ = a.shape.num_q_heads;
  // One warp takes a row unless the parts of some row need more than one round of its loads; rounds of
  // eight are mostly empty slots where no row has more than two (32768 rows of two parts: 10 us,
  // 34 MB at 3.4 TB/s, against 17).
  if (max_parts <= 8) {
    auto* kernel = max_parts <= 2 ? q4_merge_kernel<1, 2> : q4_merge_kernel<1, 8>;
    return launch_kernel(kernel, dim3(n_merge, (HQ + 3) / 4), dim3(128), 0, st, a.pdl != 0, a, d_merge);
  }
  return launch_kernel(q4_merge_kernel<4, 8>, dim3(n_merge, HQ), dim3(128), 0, st, a.pdl != 0, a, d_merge);
}

cudaError_t launch_attention_q4(const AttnArgs& a, const Q4Items& it, cudaStream_t st) {
  const int64_t mid = (int64_t)it.n_mid * a.shape.num_kv_heads;
  const int64_t narrow = (int64_t)it.n_narrow * a.shape.num_kv_heads;
  if (mid + narrow == 0) return cudaSuccess;
  if (std::max(mid, narrow) > INT32_MAX - (1 << 20)) return cudaErrorInvalidValue;
  const Q4Units u = {it.n_wide, (int32_t)mid, it.n_wide + it.n_mid, (int32_t)narrow};
  static bool configured[64] = {};
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!configured[dev]) {
    cudaError_t e = cudaFuncSetAttribute(attn_q4_kernel,
                                         cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemQ4);
    if (e != cudaSuccess) return e;
    configured[dev] = true;
  }
  const int ctas = (int)std::min<int64_t>(mid + narrow, a.num_sms);
  return launch_kernel(attn_q4_kernel, dim3(ctas), dim3(32 * kWarps), kSmemQ4, st, a.pdl != 0, a, u);
}

cudaError_t launch_q4_verify_finish(const AttnArgs& a, const VerifyDesc* d_desc, int n_desc,
                                    cudaStream_t st) {
  if (n_desc <= 0) return cudaSuccess;
  // Heads of one warp, two where two share a kv head: 2496 candidates x 32 heads took 57 us, with one
  // head 72, with four (122 registers) 64.  (Now 54.)
  const int heads = a.shape.group % 2 == 0 ? 2 : 1;
  auto* kernel = heads == 2 ? q4_verify_finish_kernel<2> : q4_verify_finish_kernel<1>;
  return launch_kernel(kernel, dim3(n_desc, (a.shape.num_q_heads + 4 * heads - 1) / (4 * heads)),
                       dim3(128), 0, st, a.pdl != 0, a, d_desc);
}

}  // namespace apar
