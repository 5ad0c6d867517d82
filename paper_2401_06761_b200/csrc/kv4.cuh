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
// 80 bytes per row: 64 of codes, then per group {s, lo} as two bf16.  The rows of a (block, kv
// head) follow each other, so a tile is 1280 contiguous bytes (a bf16 tile: 4096), a new row is
// one contiguous write, and a fork copies the first r * 80 bytes.
//
// The order of the codes inside a row is the one in which the attention kernel's matrix
// fragments want them, so that a lane turns a 32-bit word into four operand registers with one
// logical instruction each:
//   K  dim 32 j + 8 x + e (e = 0..7): word j of the 16 bytes at 16 x, nibble e / 2 + 4 (e & 1)
//      (a lane of a 16 x 16 operand holds dims 2 p, 2 p + 1 of its row in one register: the two
//      nibbles p and p + 4 are 16 bits apart)
//   V  dim 32 G + 4 g + i (i = 0..3): nibble i of the 16 bits at byte 8 g + 2 G
//      (there a register holds one dim of two tokens; the lane joins the 16-bit pieces of two
//      rows first)
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace apar {

constexpr int kQ4RowBytes = 80;                  // 64 of codes + 4 x (s, lo)
constexpr int kQ4CodeBytes = 64;
constexpr int kQ4TileBytes = 16 * kQ4RowBytes;   // one (block, kv head) of K or of V
constexpr float kQ4MinScale = 7.888609052210118e-31f;   // 2^-100
constexpr int kQ4RowVec = kQ4RowBytes / 16;

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// The eight values of dims 8 c .. 8 c + 7 (c = 0..15) of one row, as floats.
__device__ __forceinline__ void q4_load8_k(const uint8_t* row, int c, float* f) {
  const uint32_t w = *(const uint32_t*)(row + (c & 3) * 16 + (c >> 2) * 4);
  const uint32_t sl = *(const uint32_t*)(row + kQ4CodeBytes + (c >> 2) * 4);
  const float s = bf16_lo(sl), lo = bf16_hi(sl);
#pragma unroll
  for (int e = 0; e < 8; ++e)
    f[e] = fmaf(s, (float)((w >> (4 * ((e >> 1) + 4 * (e & 1)))) & 15u), lo);
}
__device__ __forceinline__ void q4_load8_v(const uint8_t* row, int c, float* f) {
  const uint8_t* p = row + (c & 3) * 16 + (c >> 2) * 2;
  const uint32_t w = (uint32_t)*(const uint16_t*)p | ((uint32_t)*(const uint16_t*)(p + 8) << 16);
  const uint32_t sl = *(const uint32_t*)(row + kQ4CodeBytes + (c >> 2) * 4);
  const float s = bf16_lo(sl), lo = bf16_hi(sl);
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = fmaf(s, (float)((w >> (4 * e)) & 15u), lo);
}

}  // namespace apar
