// Tree attention over a KV pool held in 4 bits (layout: kv4.cuh).
//
// A unit is eight query rows of one work item and one kv head; its CTA's four warps take every
// fourth block of the item, each with its own ring of tiles (K and V of one block: 2560 bytes)
// filled with cp.async, and fold their (reference, l, O) at the end.
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
//                   group of 32 dims is two products; its scale and offset are applied to the
//                   32-bit sums: score = sum_j s_j acc_j + lo_j qsum_j, with qsum_j the sum of the
//                   query over the group, and the powers of two are part of the softmax scale.
//                   Scores are exact to 32 bits.
//   O^T += V^T P^T  A = V codes, 16 dims x 16 tokens.  B = P s_j, one operand per group, rounded
//                   once to f16: it is below 2^10 by the choice of reference, and 11 bits against
//                   bf16's eight keep the result as good as 32-bit arithmetic rounded to bf16.
//                   The offsets lo_j are summed in 32 bits on the side, once per group and row.
// The reference subtracted in the exponent is the running maximum of score + log2(largest
// scale of the token's V row), not of the score: P s_j is then bounded whatever the scales are,
// and f16's narrow exponent is spent on the largest terms of the sum.  It moves lazily (kSlack).
//
// The C fragment of S^T holds tokens in rows, the B operand wants them in the k index: a
// movmatrix of the 8 x 8 halves brings one into the other.
#include <algorithm>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "apar_internal.h"
#include "kv4.cuh"
#include "ptx.cuh"

namespace apar {
namespace {

constexpr int kRows = 8;                             // query rows of a unit
constexpr int kDepth = 5;                            // tiles in flight per warp
constexpr int kWarps = 4;
constexpr int kSlot = 2 * kQ4TileBytes;              // K and V of one block
constexpr int kRing = kDepth * kSlot;
constexpr int kFoldFloats = kRows * kDim;            // one warp's O when it is folded
constexpr int kSmemQ4 = kWarps * kRing;
static_assert(kWarps * kFoldFloats * 4 <= kSmemQ4, "the fold takes the place of the rings");
constexpr float kSlack = 8.f;                        // the reference moves only past 2^8
constexpr float kCodeUnit = 1.f / 16777216.f;        // what a code of 1 counts as in a product: 2^-24
constexpr float kMinScaleLog2 = -60.f;               // V scales below 2^-60 count as 2^-60

__device__ __forceinline__ void mma_f16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                        uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, "
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
// nibbles n and n + 4 of w as an f16 pair: c * 2^-24 for even n, c * 2^-20 for odd n
__device__ __forceinline__ uint32_t codes_f16(uint32_t w, int n) {
  return (n < 2 ? w : w >> 8) & ((n & 1) ? 0x00f000f0u : 0x000f000fu);
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
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}

__global__ void __launch_bounds__(32 * kWarps, 4)
attn_q4_kernel(const AttnArgs a, const Q4Grid grid) {
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float fold_m[kWarps][kRows], fold_l[kWarps][kRows];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, q = lane & 3;
  const int kvh = blockIdx.y;
  const int G = a.shape.group, HQ = a.shape.num_q_heads, HKV = a.shape.num_kv_heads;

  // the CTA's item and row tile: items of a class have the same number of row tiles
  int cls = 0;
  while (cls < 3 && (int)blockIdx.x >= grid.cta_end[cls]) ++cls;
  const int cta = (int)blockIdx.x - (cls ? grid.cta_end[cls - 1] : 0);
  const WorkItem it = a.d_items[grid.item_begin[cls] + cta / grid.tiles[cls]];
  const int r0 = cta % grid.tiles[cls] * kRows;
  const int R = it.n_users * G;
  if (r0 >= R) return;                               // (an item narrower than its class)

  const int tok_end = it.tok_end < 0 ? a.d_lens[it.table_row] : it.tok_end;
  const int n_tok = tok_end - it.tok_begin;
  const int n_blk = (n_tok + kBlock - 1) / kBlock;
  const int32_t* table = a.d_tables + (size_t)it.table_row * a.shape.table_stride +
                         it.tok_begin / kBlock;
  const uint32_t ring = s32(smem) + warp * kRing;

  // ---- loads: this warp's k-th block is block warp + 4 k of the item
  const int my_blk = n_blk > warp ? (n_blk - warp + kWarps - 1) / kWarps : 0;
  auto issue = [&](int k, int bid) {
    const size_t tile = ((size_t)bid * HKV + kvh) * kQ4TileBytes;
    const uint8_t* kt = (const uint8_t*)a.k_pool + tile;
    const uint8_t* vt = (const uint8_t*)a.v_pool + tile - kQ4TileBytes;
    const uint32_t dst = ring + (k % kDepth) * kSlot;
#pragma unroll
    for (int j = 0; j < 2 * kQ4TileBytes / 512; ++j) {
      const int x = (j * 32 + lane) * 16;
      cp_async16(dst + x, (x < kQ4TileBytes ? kt : vt) + x);
    }
  };
#pragma unroll
  for (int k = 0; k < kDepth - 1; ++k) {
    if (k < my_blk) issue(k, table[warp + kWarps * k]);
    asm volatile("cp.async.commit_group;" ::: "memory");
  }
  int next_bid = kDepth - 1 < my_blk ? table[warp + kWarps * (kDepth - 1)] : 0;

  // ---- queries: row r0 + g, dims 32 j + 8 q .. + 7, as B fragments
  uint32_t qb[4][4];
  float qs[4][2], unit[2];       // of rows 2 q, 2 q + 1: sums over each group; 2^24 / their factor
  {
    const int r = r0 + g;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int p = 0; p < 4; ++p) qb[j][p] = 0u;
    if (r < R) {
      const int query = a.d_users[it.user_begin + r / G].query;
      const uint4* src = (const uint4*)a.q + ((size_t)query * HQ + kvh * G + r % G) * 16 + q;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint4 v = __ldg(src + 4 * j);
        qb[j][0] = v.x; qb[j][1] = v.y; qb[j][2] = v.z; qb[j][3] = v.w;
      }
    }
    uint32_t top = 0;            // bits of the row's largest magnitude (bf16, in the high half)
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int p = 0; p < 4; ++p)
        top = max(top, max(qb[j][p] << 17, (qb[j][p] & 0x7fff0000u) << 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
    // the factor 2^k; a row of zeros or subnormal numbers has k at its limit
    const int k = min(126, 14 + 127 - (int)(top >> 24));
    const float f = __uint_as_float((uint32_t)(k + 127) << 23);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float x = 0.f;
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const float e0 = bf16_lo(qb[j][p]) * f, e1 = bf16_hi(qb[j][p]) * f;
        x += e0 + e1;
        qb[j][p] = (p & 1) ? pack_f16(e0 * 0.0625f, e1 * 0.0625f) : pack_f16(e0, e1);
      }
      x += __shfl_xor_sync(0xffffffffu, x, 1);
      x += __shfl_xor_sync(0xffffffffu, x, 2);
      qs[j][0] = __shfl_sync(0xffffffffu, x, 8 * q) * kCodeUnit;
      qs[j][1] = __shfl_sync(0xffffffffu, x, 8 * q + 4) * kCodeUnit;
    }
    // score * log2(e) * scale = (what the products give) * unit
    const float u = a.scale_log2e * (1.f / kCodeUnit) * __uint_as_float((uint32_t)(127 - k) << 23);
    unit[0] = __shfl_sync(0xffffffffu, u, 8 * q);
    unit[1] = __shfl_sync(0xffffffffu, u, 8 * q + 4);
  }

  float o[8][4], lsum[4][2], ref[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
  for (int m = 0; m < 8; ++m)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[m][e] = 0.f;
#pragma unroll
  for (int j = 0; j < 4; ++j) lsum[j][0] = lsum[j][1] = 0.f;

  for (int k = 0; k < my_blk; ++k) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kDepth - 2) : "memory");
    __syncwarp();
    const uint32_t kt = ring + (k % kDepth) * kSlot, vt = kt + kQ4TileBytes;
    // the slot after the last one in flight was read in the previous pass: refill it
    if (k + kDepth - 1 < my_blk) issue(k + kDepth - 1, next_bid);
    asm volatile("cp.async.commit_group;" ::: "memory");
    next_bid = k + kDepth < my_blk ? table[warp + kWarps * (k + kDepth)] : 0;

    // ---- scores of tokens g and g + 8 for rows 2 q and 2 q + 1
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    {
      const uint4 k0 = lds128(kt + g * kQ4RowBytes + q * 16);
      const uint4 k1 = lds128(kt + (g + 8) * kQ4RowBytes + q * 16);
      const uint4 s0 = lds128(kt + g * kQ4RowBytes + kQ4CodeBytes);
      const uint4 s1 = lds128(kt + (g + 8) * kQ4RowBytes + kQ4CodeBytes);
      const uint32_t w0[4] = {k0.x, k0.y, k0.z, k0.w}, w1[4] = {k1.x, k1.y, k1.z, k1.w};
      const uint32_t t0[4] = {s0.x, s0.y, s0.z, s0.w}, t1[4] = {s1.x, s1.y, s1.z, s1.w};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
        mma_f16(acc, codes_f16(w0[j], 0), codes_f16(w1[j], 0), codes_f16(w0[j], 1),
                codes_f16(w1[j], 1), qb[j][0], qb[j][1]);
        mma_f16(acc, codes_f16(w0[j], 2), codes_f16(w1[j], 2), codes_f16(w0[j], 3),
                codes_f16(w1[j], 3), qb[j][2], qb[j][3]);
        const float sa = bf16_lo(t0[j]), sb = bf16_lo(t1[j]);
        const float la = bf16_hi(t0[j]), lb = bf16_hi(t1[j]);
        x[0] = fmaf(sa, acc[0], fmaf(la, qs[j][0], x[0]));
        x[1] = fmaf(sa, acc[1], fmaf(la, qs[j][1], x[1]));
        x[2] = fmaf(sb, acc[2], fmaf(lb, qs[j][0], x[2]));
        x[3] = fmaf(sb, acc[3], fmaf(lb, qs[j][1], x[3]));
      }
    }
    x[0] *= unit[0];
    x[1] *= unit[1];
    x[2] *= unit[0];
    x[3] *= unit[1];

    // ---- V scales of tokens g and g + 8; rows past the length hold unspecified bits
    uint4 v0 = lds128(vt + g * kQ4RowBytes + kQ4CodeBytes);
    uint4 v1 = lds128(vt + (g + 8) * kQ4RowBytes + kQ4CodeBytes);
    const int nv = n_tok - (warp + kWarps * k) * kBlock;
    if (nv < kBlock) {
      if (g >= nv) {
        x[0] = x[1] = -INFINITY;
        v0 = make_uint4(0u, 0u, 0u, 0u);
      }
      if (g + 8 >= nv) {
        x[2] = x[3] = -INFINITY;
        v1 = make_uint4(0u, 0u, 0u, 0u);
      }
    }
    const uint32_t z0[4] = {v0.x, v0.y, v0.z, v0.w}, z1[4] = {v1.x, v1.y, v1.z, v1.w};
    // log2 of a token's largest scale, from the bits of the number (below by at most 0.09)
    auto scale_log2 = [](const uint32_t (&z)[4]) {
      const int top = max(max((int)(z[0] << 16), (int)(z[1] << 16)),
                          max((int)(z[2] << 16), (int)(z[3] << 16)));
      return fmaxf(fmaf((float)top, 1.f / 8388608.f, -127.f), kMinScaleLog2);
    };
    const float e0 = scale_log2(z0), e1 = scale_log2(z1);
    const float y0 = fmaxf(x[0] + e0, x[2] + e1), y1 = fmaxf(x[1] + e0, x[3] + e1);
    if (__any_sync(0xffffffffu, y0 > ref[0] + kSlack || y1 > ref[1] + kSlack)) {
      float m0 = y0, m1 = y1;
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) {
        m0 = fmaxf(m0, __shfl_xor_sync(0xffffffffu, m0, d));
        m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, d));
      }
      m0 = fmaxf(m0, ref[0]);
      m1 = fmaxf(m1, ref[1]);
      const float f0 = ref[0] == -INFINITY ? 0.f : ex2(ref[0] - m0);
      const float f1 = ref[1] == -INFINITY ? 0.f : ex2(ref[1] - m1);
      ref[0] = m0;
      ref[1] = m1;
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
    }
    const float p0 = ex2(x[0] - ref[0]), p1 = ex2(x[1] - ref[1]);
    const float p2 = ex2(x[2] - ref[0]), p3 = ex2(x[3] - ref[1]);
    l[0] += p0 + p2;
    l[1] += p1 + p3;

    // ---- O^T += V^T P^T
    const uint2 t0 = lds64(vt + (2 * q) * kQ4RowBytes + 8 * g);
    const uint2 t1 = lds64(vt + (2 * q + 1) * kQ4RowBytes + 8 * g);
    const uint2 t2 = lds64(vt + (2 * q + 8) * kQ4RowBytes + 8 * g);
    const uint2 t3 = lds64(vt + (2 * q + 9) * kQ4RowBytes + 8 * g);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float sa = bf16_lo(z0[j]), sb = bf16_lo(z1[j]);
      const uint32_t b0 = transpose8x8(pack_f16(p0 * sa, p1 * sa));
      const uint32_t b1 = transpose8x8(pack_f16(p2 * sb, p3 * sb));
      const float la = bf16_hi(z0[j]), lb = bf16_hi(z1[j]);
      lsum[j][0] = fmaf(p0, la, fmaf(p2, lb, lsum[j][0]));
      lsum[j][1] = fmaf(p1, la, fmaf(p3, lb, lsum[j][1]));
      const uint32_t sel = (j & 1) ? 0x7632 : 0x5410;
      const uint32_t xl = __byte_perm(j < 2 ? t0.x : t0.y, j < 2 ? t1.x : t1.y, sel);
      const uint32_t xh = __byte_perm(j < 2 ? t2.x : t2.y, j < 2 ? t3.x : t3.y, sel);
      mma_f16(o[2 * j], codes_f16(xl, 0), codes_f16(xl, 1), codes_f16(xh, 0), codes_f16(xh, 1),
              b0, b1);
      mma_f16(o[2 * j + 1], codes_f16(xl, 2), codes_f16(xl, 3), codes_f16(xh, 2), codes_f16(xh, 3),
              b0, b1);
    }
  }
  asm volatile("cp.async.wait_all;" ::: "memory");

  // ---- sums over the lanes that hold other tokens of the same rows
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
  // ---- fold of the four warps (the rings are no longer needed)
  __syncthreads();
  float* fo = (float*)smem;
  constexpr float kLow = 1.f / kCodeUnit, kHigh = kLow / 16.f;   // (odd nibbles counted 16 times)
  if (g == 0) {
    fold_m[warp][2 * q] = ref[0];
    fold_m[warp][2 * q + 1] = ref[1];
    fold_l[warp][2 * q] = l[0];
    fold_l[warp][2 * q + 1] = l[1];
  }
#pragma unroll
  for (int e = 0; e < 2; ++e)                      // row 2 q + e: dims 32 j + 4 g .. + 3
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *(float4*)(fo + warp * kFoldFloats + (2 * q + e) * kDim + 32 * j + 4 * g) =
          make_float4(fmaf(o[2 * j][e], kLow, lsum[j][e]), fmaf(o[2 * j][2 + e], kHigh, lsum[j][e]),
                      fmaf(o[2 * j + 1][e], kLow, lsum[j][e]),
                      fmaf(o[2 * j + 1][2 + e], kHigh, lsum[j][e]));
  __syncthreads();
#pragma unroll
  for (int rr = 0; rr < kRows / kWarps; ++rr) {
    const int row = warp + kWarps * rr, r = r0 + row;
    if (r >= R) continue;
    float M = fold_m[0][row];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) M = fmaxf(M, fold_m[w][row]);
    float L = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float4 v = *(const float4*)(fo + w * kFoldFloats + row * kDim + 4 * lane);
      // (a warp without blocks has -inf and zeros; a row of NaN scores has l = NaN)
      const float f = fold_m[w][row] == M ? 1.f : ex2(fold_m[w][row] - M);
      L = fmaf(fold_l[w][row], f, L);
      acc.x = fmaf(v.x, f, acc.x); acc.y = fmaf(v.y, f, acc.y);
      acc.z = fmaf(v.z, f, acc.z); acc.w = fmaf(v.w, f, acc.w);
    }
    const UserRef ur = a.d_users[it.user_begin + r / G];
    const int head = kvh * G + r % G;
    if (ur.slot < 0) {
      const float inv = 1.f / L;
      *((uint2*)((__nv_bfloat16*)a.out + ((size_t)ur.query * HQ + head) * kDim) + lane) =
          make_uint2(pack2(acc.x * inv, acc.y * inv), pack2(acc.z * inv, acc.w * inv));
    } else {
      const size_t prow = (size_t)(ur.slot + it.slot_add) * HQ + head;
      *((float4*)(a.part_o + prow * kDim) + lane) = acc;
      if (lane == 0) a.part_ml[prow] = make_float2(M, L);
    }
  }
}

// Candidate tokens of a verification: as verify_tail_kernel, rows read from the 4-bit pool.
__global__ void __launch_bounds__(128) q4_verify_tail_kernel(const AttnArgs a,
                                                             const VerifyDesc* __restrict__ descs) {
  const VerifyDesc d = descs[blockIdx.x];
  const int kvh = blockIdx.y;
  const int G = a.shape.group, HQ = a.shape.num_q_heads, HKV = a.shape.num_kv_heads;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int half = lane >> 4, c = lane & 15;
  const int32_t* table = a.d_tables + (size_t)d.row * a.shape.table_stride;
  for (int hg = warp; hg < G; hg += 4) {
    const int head = kvh * G + hg;
    float qf[8], o[8];
    {
      const uint4 qv = __ldg((const uint4*)a.q + ((size_t)d.query * HQ + head) * 16 + c);
      const uint32_t w[4] = {qv.x, qv.y, qv.z, qv.w};
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        qf[2 * x] = bf16_lo(w[x]) * a.scale_log2e;
        qf[2 * x + 1] = bf16_hi(w[x]) * a.scale_log2e;
        o[2 * x] = o[2 * x + 1] = 0.f;
      }
    }
    float m = -INFINITY, l = 0.f;
    for (int i0 = 0; i0 < d.n_cand; i0 += 2) {
      const int i = i0 + half;
      const bool on = i < d.n_cand && ((d.mask >> i) & 1ull);
      float t = 0.f, vf[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
      if (on) {
        const int pos = d.base + i;
        const size_t row = (((size_t)table[pos >> 4] * HKV + kvh) * kBlock + (pos & (kBlock - 1)));
        float kf[8];
        q4_load8_k((const uint8_t*)a.k_pool + row * kQ4RowBytes, c, kf);
        q4_load8_v((const uint8_t*)a.v_pool + row * kQ4RowBytes, c, vf);
#pragma unroll
        for (int x = 0; x < 8; ++x) t = fmaf(qf[x], kf[x], t);
      }
#pragma unroll
      for (int x = 8; x; x >>= 1) t += __shfl_xor_sync(0xffffffffu, t, x);
      const float s = on ? t : -INFINITY;
      const float other = __shfl_xor_sync(0xffffffffu, s, 16);
      const bool other_on = __shfl_xor_sync(0xffffffffu, (int)on, 16) != 0;
      if (!on && !other_on) continue;              // both tokens masked
      const float mn = fmaxf(m, fmaxf(s, other));
      const float corr = m == -INFINITY ? 0.f : ex2(m - mn);
      const float p = on ? ex2(s - mn) : 0.f;
      l = l * corr + p + (other_on ? ex2(other - mn) : 0.f);   // identical in both halves
      m = mn;
#pragma unroll
      for (int x = 0; x < 8; ++x) o[x] = fmaf(p, vf[x], o[x] * corr);
    }
#pragma unroll
    for (int x = 0; x < 8; ++x) o[x] += __shfl_xor_sync(0xffffffffu, o[x], 16);
    if (half == 0) {
      if (d.slot < 0) {
        const float inv = 1.f / l;                 // (a candidate sees itself)
        *((uint4*)((__nv_bfloat16*)a.out + ((size_t)d.query * HQ + head) * kDim) + c) =
            make_uint4(pack2(o[0] * inv, o[1] * inv), pack2(o[2] * inv, o[3] * inv),
                       pack2(o[4] * inv, o[5] * inv), pack2(o[6] * inv, o[7] * inv));
      } else {
        const size_t prow = (size_t)d.slot * HQ + head;
        float4* dst = (float4*)(a.part_o + prow * kDim) + 2 * c;
        dst[0] = make_float4(o[0], o[1], o[2], o[3]);
        dst[1] = make_float4(o[4], o[5], o[6], o[7]);
        if (c == 0) a.part_ml[prow] = make_float2(m, l);
      }
    }
  }
}

}  // namespace

cudaError_t launch_attention_q4(const AttnArgs& a, const int32_t n_items[4],
                                const int32_t max_rows[4], cudaStream_t st) {
  // classes as the planner orders them: items of 4, 3, 2 and 1 tiles of 16 rows
  Q4Grid g;
  int ctas = 0, items = 0;
  for (int k = 0; k < 4; ++k) {
    const int n = n_items[3 - k];
    g.tiles[k] = std::max(1, (max_rows[3 - k] + kRows - 1) / kRows);
    g.item_begin[k] = items;
    items += n;
    ctas += n * g.tiles[k];
    g.cta_end[k] = ctas;
  }
  if (ctas == 0) return cudaSuccess;
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
  attn_q4_kernel<<<dim3(ctas, a.shape.num_kv_heads), 32 * kWarps, kSmemQ4, st>>>(a, g);
  return cudaGetLastError();
}

cudaError_t launch_q4_verify_tail(const AttnArgs& a, const VerifyDesc* d_desc, int n_desc,
                                  cudaStream_t st) {
  if (n_desc <= 0) return cudaSuccess;
  q4_verify_tail_kernel<<<dim3(n_desc, a.shape.num_kv_heads), 128, 0, st>>>(a, d_desc);
  return cudaGetLastError();
}

}  // namespace apar
