// Kernels that move rows of a 4-bit KV pool (layout and arithmetic: kv4.cuh): the quantising
// scatter of new rows, the copy of a partial block at fork, the moves of accepted candidate rows,
// and the reading of rows back as bf16 values (which also serves bf16 pools).
// Measured: 22 k rows of 32 kv heads: append 113 us for 471 MB, 4.2 TB/s, 0.63 of a copy (the arithmetic
// of the quantiser, some 8 instructions a value, keeps it from more); read 96 us for the same
// bytes, 4.9 TB/s, three quarters of them written.  4096 rows of 8 heads: 12 and 9 us.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "apar_internal.h"
#include "kv4.cuh"

namespace apar {
namespace {

// ------------------------------------------------------------------ append: quantise and scatter
// Eight lanes hold one row, sixteen dims (32 bytes) each, half a group of 32: enough values to
// spread the division and the reciprocal of a group's scale over.
struct Q4Half {           // one lane's share of a row: sixteen codes and its group's scale word
  uint32_t w0, w1, scale;
};

// Nibble order of each word's eight codes: K e / 2 + 4 (e & 1), V e.
template <bool kV>
__device__ __forceinline__ Q4Half q4_quantise(const uint4& xa, const uint4& xb) {
  const uint32_t xs[8] = {xa.x, xa.y, xa.z, xa.w, xb.x, xb.y, xb.z, xb.w};
  // the NaN-propagating minimum lets a NaN reach the scale
  __nv_bfloat162 mn = *(__nv_bfloat162*)&xs[0], mx = mn;
#pragma unroll
  for (int e = 1; e < 8; ++e) {
    mn = __hmin2_nan(mn, *(__nv_bfloat162*)&xs[e]);
    mx = __hmax2_nan(mx, *(__nv_bfloat162*)&xs[e]);
  }
  {
    uint32_t a = __shfl_xor_sync(0xffffffffu, *(uint32_t*)&mn, 1);
    uint32_t b = __shfl_xor_sync(0xffffffffu, *(uint32_t*)&mx, 1);
    mn = __hmin2_nan(mn, *(__nv_bfloat162*)&a);
    mx = __hmax2_nan(mx, *(__nv_bfloat162*)&b);
  }
  const float lo = __bfloat162float(__hmin_nan(mn.x, mn.y));
  const float hi = __bfloat162float(__hmax_nan(mx.x, mx.y));
  const float range = hi - lo;
  float s = __bfloat162float(__float2bfloat16_rn(__fdiv_rn(range, 15.f)));
  const bool bad = !(range <= 3.402823466e38f);        // NaN, or an infinity
  if (!(s >= kQ4MinScale)) s = 0.f;
  // c = round((x - lo) / s).  The quotient is correctly rounded, as a division would give it: one
  // residual step on a correctly rounded reciprocal (Markstein 1990; the divisor has eight
  // significant bits, so the theorem's one exception, a significand of all ones, cannot occur).
  // Adding 1.5 * 2^23 leaves the integer, ties to even, in the low bits of a number whose other
  // bits are known: they are summed along and taken off once per word.
  const float inv = s > 0.f ? __frcp_rn(s) : 0.f;
  constexpr uint32_t kMagicBits = 0x4b400000u;
  uint32_t w[2];
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    uint32_t sum = 0, known = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const uint32_t x = xs[4 * n + (e >> 1)];
      const float d = ((e & 1) ? bf16_hi(x) : bf16_lo(x)) - lo;
      const float q = d * inv;
      const float t = fmaf(fmaf(-q, s, d), inv, q);
      const uint32_t at = 1u << (kV ? 4 * e : 4 * ((e >> 1) + 4 * (e & 1)));
      sum += __float_as_uint(t + 12582912.f) * at;
      known += kMagicBits * at;
    }
    w[n] = sum - known;
  }
  // (a NaN scale carries the sign bit: integer comparisons of scales rank it below all others)
  if (bad) return Q4Half{0u, 0u, 0xffc0ffc0u};
  return Q4Half{w[0], w[1], (__float_as_uint(s) >> 16) | (__float_as_uint(lo) & 0xffff0000u)};
}

template <bool kV>
__device__ __forceinline__ void q4_append_rows(uint8_t* __restrict__ pool, const uint4* __restrict__ rows,
                                               const int32_t* __restrict__ slots, long long first_row,
                                               int n_rows, int num_kv_heads) {
  const uint32_t rh = blockIdx.x * (blockDim.x / 8) + (threadIdx.x >> 3);   // (row, head) < 2^31
  const int c = threadIdx.x & 7;
  bool on = rh < (uint32_t)n_rows * (uint32_t)num_kv_heads;
  const int r = on ? (int)(rh / (uint32_t)num_kv_heads) : 0;
  const int h = on ? (int)(rh - (uint32_t)r * (uint32_t)num_kv_heads) : 0;
  const int slot = slots[r];
  const bool pair = on && !(slot & 1) && r + 1 < n_rows && slots[r + 1] == slot + 1;
  if ((slot & 1) && r > 0 && slots[r - 1] == slot - 1) on = false;
  if (!__any_sync(0xffffffffu, on)) return;
  const uint4* src = rows + ((first_row + r) * num_kv_heads + h) * 16 + 2 * c;
  uint4 x[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = make_uint4(0u, 0u, 0u, 0u);
  if (on) {
    x[0] = __ldg(src);
    x[1] = __ldg(src + 1);
  }
  if (pair) {
    x[2] = __ldg(src + (size_t)num_kv_heads * 16);
    x[3] = __ldg(src + (size_t)num_kv_heads * 16 + 1);
  }
  const Q4Half a = q4_quantise<kV>(x[0], x[1]), b = q4_quantise<kV>(x[2], x[3]);
  if (!on) return;
  uint8_t* tile = pool + ((size_t)(slot >> 4) * num_kv_heads + h) * kQ4TileBytes;
  const int off = slot & 15, G = c >> 1;
  if (kV) {
    uint8_t* p = tile + q4_v_piece(off, 4 * (c & 1), G);     // pieces 4 (c & 1) .. + 3
    if (pair) {
      *(uint32_t*)p = __byte_perm(a.w0, b.w0, 0x5410);
      *(uint32_t*)(p + 16) = __byte_perm(a.w0, b.w0, 0x7632);
      *(uint32_t*)(p + 32) = __byte_perm(a.w1, b.w1, 0x5410);
      *(uint32_t*)(p + 48) = __byte_perm(a.w1, b.w1, 0x7632);
    } else {
      *(uint16_t*)p = (uint16_t)a.w0;
      *(uint16_t*)(p + 16) = (uint16_t)(a.w0 >> 16);
      *(uint16_t*)(p + 32) = (uint16_t)a.w1;
      *(uint16_t*)(p + 48) = (uint16_t)(a.w1 >> 16);
    }
    if (!(c & 1)) {
      *(uint32_t*)(tile + q4_v_scales(off) + 4 * G) = a.scale;
      if (pair) *(uint32_t*)(tile + q4_v_scales(off + 1) + 4 * G) = b.scale;
    }
  } else {
    uint8_t* row = tile + off * kQ4RowBytes + (c & 1) * 32 + G * 4;    // word G of pieces 2 (c & 1), + 1
    *(uint32_t*)row = a.w0;
    *(uint32_t*)(row + 16) = a.w1;
    if (pair) {
      *(uint32_t*)(row + kQ4RowBytes) = b.w0;
      *(uint32_t*)(row + kQ4RowBytes + 16) = b.w1;
    }
    if (!(c & 1)) {
      uint8_t* sc = tile + off * kQ4RowBytes + kQ4CodeBytes + 4 * G;
      *(uint32_t*)sc = a.scale;
      if (pair) *(uint32_t*)(sc + kQ4RowBytes) = b.scale;
    }
  }
}

// Two rows that are neighbours in the pool, an even one and the odd one after it, are written by
// the lanes of the first, so that the pair's interleaved V codes leave as whole words; the lanes
// of the second have nothing to do.  blockIdx.y selects K or V.  The kernel reads 256 bytes and
// writes 80 for each row.
__global__ void __launch_bounds__(256) q4_append_kernel(uint8_t* __restrict__ k_pool,
                                                        uint8_t* __restrict__ v_pool,
                                                        const uint4* __restrict__ k_new,
                                                        const uint4* __restrict__ v_new,
                                                        const int32_t* __restrict__ slots,
                                                        long long first_row, int n_rows,
                                                        int num_kv_heads) {
  if (blockIdx.y)
    q4_append_rows<true>(v_pool, v_new, slots, first_row, n_rows, num_kv_heads);
  else
    q4_append_rows<false>(k_pool, k_new, slots, first_row, n_rows, num_kv_heads);
}

// ------------------------------------------------------------------ fork: copy r rows
__global__ void __launch_bounds__(96) q4_cow_copy_kernel(uint4* __restrict__ k_pool,
                                                         uint4* __restrict__ v_pool,
                                                         const CowCopy* __restrict__ copies,
                                                         int num_kv_heads) {
  const CowCopy c = copies[blockIdx.x];
  uint4* pool = blockIdx.z ? v_pool : k_pool;
  const size_t tile = kQ4TileBytes / 16;
  const uint4* src = pool + ((size_t)c.src_block * num_kv_heads + blockIdx.y) * tile;
  uint4* dst = pool + ((size_t)c.dst_block * num_kv_heads + blockIdx.y) * tile;
  // (V rows lie in pairs: the partner of an odd last row is copied along, unspecified as it is)
  const int rows = blockIdx.z ? (c.rows + 1) & ~1 : c.rows;
  for (int i = threadIdx.x; i < rows * kQ4RowVec; i += blockDim.x) dst[i] = src[i];
}

// ------------------------------------------------------------------ accepted candidates: row moves
// As row_move_kernel: every source row of a group is read before the first one is written.  A
// row is 32 pieces of 16 bits and 16 bytes of scales, which holds for K and V rows alike.
__global__ void __launch_bounds__(256) q4_row_move_kernel(uint8_t* __restrict__ k_pool,
                                                          uint8_t* __restrict__ v_pool,
                                                          const RowMove* __restrict__ moves,
                                                          const int32_t* __restrict__ group_begin,
                                                          int num_kv_heads) {
  __shared__ uint16_t rows[64 * kQ4RowBytes / 2];
  constexpr int kPieces = kQ4RowBytes / 2, kCodes = kQ4CodeBytes / 2;
  const int m0 = group_begin[blockIdx.x], n = group_begin[blockIdx.x + 1] - m0;
  const bool is_v = blockIdx.z != 0;
  uint8_t* pool = is_v ? v_pool : k_pool;
  const int h = blockIdx.y;
  auto at = [&](int slot, int i) {
    uint8_t* tile = pool + ((size_t)(slot >> 4) * num_kv_heads + h) * kQ4TileBytes;
    const int off = slot & 15;
    if (!is_v) return (uint16_t*)(tile + off * kQ4RowBytes) + i;
    if (i >= kCodes) return (uint16_t*)(tile + q4_v_scales(off)) + (i - kCodes);
    return (uint16_t*)(tile + q4_v_piece(off, i >> 2, i & 3));
  };
  for (int x = threadIdx.x; x < n * kPieces; x += blockDim.x)
    rows[x] = *at(moves[m0 + x / kPieces].src_slot, x % kPieces);
  __syncthreads();
  for (int x = threadIdx.x; x < n * kPieces; x += blockDim.x)
    *at(moves[m0 + x / kPieces].dst_slot, x % kPieces) = rows[x];
}

// ------------------------------------------------------------------ rows read back as bf16
// One thread per sixteen dims of a row; blockIdx.y selects K or V.  A 4-bit row reads as
// bf16(lo + s * c), the sum taken in 32 bits and rounded once more to the output's type.
template <bool kQ4>
__global__ void __launch_bounds__(256) read_rows_kernel(const uint8_t* __restrict__ k_pool,
                                                        const uint8_t* __restrict__ v_pool,
                                                        uint4* __restrict__ k_out,
                                                        uint4* __restrict__ v_out,
                                                        const int32_t* __restrict__ slots,
                                                        long long first_row, int n_rows,
                                                        int num_kv_heads) {
  const uint32_t rh = blockIdx.x * (blockDim.x / 8) + (threadIdx.x >> 3);   // (row, head) < 2^31
  if (rh >= (uint32_t)n_rows * (uint32_t)num_kv_heads) return;
  const int c = threadIdx.x & 7;
  const int r = (int)(rh / (uint32_t)num_kv_heads);
  const int h = (int)(rh - (uint32_t)r * (uint32_t)num_kv_heads);
  const int slot = slots[r];
  const size_t tile = (size_t)(slot >> 4) * num_kv_heads + h;
  const uint8_t* pool = blockIdx.y ? v_pool : k_pool;
  uint4 out[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (kQ4) {
      float f[8];
      if (blockIdx.y) q4_load8_v(pool + tile * kQ4TileBytes, slot & 15, 2 * c + i, f);
      else q4_load8_k(pool + tile * kQ4TileBytes, slot & 15, 2 * c + i, f);
      uint32_t w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * e], f[2 * e + 1]);
        w[e] = *(uint32_t*)&p;
      }
      out[i] = make_uint4(w[0], w[1], w[2], w[3]);
    } else {
      out[i] = ((const uint4*)pool)[(tile * kBlock + (slot & 15)) * 16 + 2 * c + i];
    }
  }
  uint4* dst = (blockIdx.y ? v_out : k_out) + (first_row * num_kv_heads + rh) * 16 + 2 * c;
  dst[0] = out[0];
  dst[1] = out[1];
}

}  // namespace

cudaError_t launch_q4_append(void* k_pool, void* v_pool, const void* k_new, const void* v_new,
                             const int32_t* d_slots, int64_t first_row, int n_rows,
                             int num_kv_heads, cudaStream_t st) {
  if (n_rows <= 0) return cudaSuccess;
  const long long total = (long long)n_rows * num_kv_heads * 8;
  q4_append_kernel<<<dim3((unsigned)((total + 255) / 256), 2), 256, 0, st>>>(
      (uint8_t*)k_pool, (uint8_t*)v_pool, (const uint4*)k_new, (const uint4*)v_new, d_slots,
      (long long)first_row, n_rows, num_kv_heads);
  return cudaGetLastError();
}

cudaError_t launch_q4_cow_copy(void* k_pool, void* v_pool, const CowCopy* d_copies, int n,
                               int num_kv_heads, cudaStream_t st) {
  if (n <= 0) return cudaSuccess;
  q4_cow_copy_kernel<<<dim3(n, num_kv_heads, 2), 96, 0, st>>>((uint4*)k_pool, (uint4*)v_pool,
                                                              d_copies, num_kv_heads);
  return cudaGetLastError();
}

cudaError_t launch_q4_row_moves(void* k_pool, void* v_pool, const RowMove* d_moves,
                                const int32_t* d_group_begin, int n_groups, int num_kv_heads,
                                cudaStream_t st) {
  if (n_groups <= 0) return cudaSuccess;
  q4_row_move_kernel<<<dim3(n_groups, num_kv_heads, 2), 256, 0, st>>>(
      (uint8_t*)k_pool, (uint8_t*)v_pool, d_moves, d_group_begin, num_kv_heads);
  return cudaGetLastError();
}

cudaError_t launch_read_rows(bool q4, const void* k_pool, const void* v_pool, void* k_out,
                             void* v_out, const int32_t* d_slots, int64_t first_row, int n_rows,
                             int num_kv_heads, cudaStream_t st) {
  if (n_rows <= 0) return cudaSuccess;
  const long long total = (long long)n_rows * num_kv_heads * 8;
  const dim3 grid((unsigned)((total + 255) / 256), 2);
  auto kernel = q4 ? read_rows_kernel<true> : read_rows_kernel<false>;
  kernel<<<grid, 256, 0, st>>>((const uint8_t*)k_pool, (const uint8_t*)v_pool, (uint4*)k_out,
                               (uint4*)v_out, d_slots, (long long)first_row, n_rows, num_kv_heads);
  return cudaGetLastError();
}

}  // namespace apar
