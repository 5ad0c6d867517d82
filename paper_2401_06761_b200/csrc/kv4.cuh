// Layout and arithmetic of a KV pool held in 4 bits (APAR_KV_Q4).
//
// A row (one token of one kv head, of K or of V) is 128 values in four groups of 32 consecutive
// dims.  A group keeps lo = min(x) and s = bf16((max(x) - lo) / 15); x becomes the integer
// c = round_half_even((x - lo) / s) in 0..15 and stands for lo + s * c.  lo is a value of the row
// itself, hence exact in bf16; s is rounded once, which moves the top of the range by at most
// 15 s / 2^9 = 0.03 s, far below the half step that the rounding to c costs anyway.  Both the
// difference and the quotient are taken in 32 bits.  A group whose scale would be below 2^-100
// stores s = 0 and c = 0 (every value reads as lo; the residuals below stay exact above that); a group with a NaN or an infinity, or whose
// range overflows, stores NaN for s and lo (all of it reads as NaN, nothing else is touched).
//
// 80 bytes per row: 64 of codes and, per group, {s, lo} as two bf16.  A (block, kv head) tile is 1280
// contiguous bytes (a bf16 tile: 4096).  The order inside it is the one in which the attention
// kernel's matrix fragments want it, so that a lane turns a 32-bit word into four operand
// registers with little more than one logical instruction each:
//   K  16 rows of 80 bytes, codes first.  A lane of a 16 x 16 operand holds dims 2 p, 2 p + 1 of its
//      row in one register, so the two nibbles p and p + 4, 16 bits apart, are neighbours: dim
//      32 j + 8 x + e (e = 0..7) is nibble e / 2 + 4 (e & 1) of word j of the 16 bytes at 16 x.
//   V  8 pairs of rows of 160 bytes.  There a register holds one dim of two tokens, so the pair's
//      rows are interleaved 16 bits at a time: dims 32 G + 4 g + i (i = 0..3) of the row with
//      parity e are the nibbles of the 16 bits at byte 4 (4 g + G) + 2 e; then {s, lo} of the even row
//      (16 bytes) and of the odd one.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace apar {

constexpr int kQ4RowBytes = 80;                  // 64 of codes + 4 x (s, lo)
constexpr int kQ4PairBytes = 160;                // two rows of V
constexpr int kQ4CodeBytes = 64;
constexpr int kQ4TileBytes = 16 * kQ4RowBytes;   // one (block, kv head) of K or of V
constexpr float kQ4MinScale = 7.888609052210118e-31f;   // 2^-100
constexpr int kQ4RowVec = kQ4RowBytes / 16;

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// The eight values of dims 8 c .. 8 c + 7 (c = 0..15) of row `off` of a tile, as floats.
__device__ __forceinline__ void q4_load8_k(const uint8_t* tile, int off, int c, float* f) {
  const uint8_t* row = tile + off * kQ4RowBytes;
  const uint32_t w = *(const uint32_t*)(row + (c & 3) * 16 + (c >> 2) * 4);
  const uint32_t sl = *(const uint32_t*)(row + kQ4CodeBytes + (c >> 2) * 4);
  const float s = bf16_lo(sl), lo = bf16_hi(sl);
#pragma unroll
  for (int e = 0; e < 8; ++e)
    f[e] = fmaf(s, (float)((w >> (4 * ((e >> 1) + 4 * (e & 1)))) & 15u), lo);
}
// byte offset, in a V tile, of the 16 bits of piece g and group G of row `off`; of its scales
__device__ __forceinline__ int q4_v_piece(int off, int g, int G) {
  return (off >> 1) * kQ4PairBytes + 4 * (4 * g + G) + 2 * (off & 1);
}
__device__ __forceinline__ int q4_v_scales(int off) {
  return (off >> 1) * kQ4PairBytes + 2 * kQ4CodeBytes + 16 * (off & 1);
}
__device__ __forceinline__ void q4_load8_v(const uint8_t* tile, int off, int c, float* f) {
  const uint8_t* p = tile + q4_v_piece(off, 2 * (c & 3), c >> 2);
  const uint32_t w = (uint32_t)*(const uint16_t*)p | ((uint32_t)*(const uint16_t*)(p + 16) << 16);
  const uint32_t sl = *(const uint32_t*)(tile + q4_v_scales(off) + (c >> 2) * 4);
  const float s = bf16_lo(sl), lo = bf16_hi(sl);
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = fmaf(s, (float)((w >> (4 * e)) & 15u), lo);
}

}  // namespace apar
