// apar_rope: rotary positions applied to query and key rows.
//
// Pair i of a head (i < rotary_dim / 2) is turned by the angle position * theta_i:
//     (a, b) -> m * (a cos - b sin, b cos + a sin)
// with (a, b) = dims (i, rotary_dim / 2 + i) in the half layout and (2 i, 2 i + 1) in the
// interleaved one; dims from rotary_dim on are copied.  The kernel moves every row once in each
// direction and does little else: it is bound by HBM, so the angles, which all heads of a token
// share, are computed once per token into shared memory.  They need 64 bits: position * theta_i
// in 32 bits is off by 2^-24 of itself, a sixteenth of a radian at position 2^20.  The product
// is reduced to [-pi, pi] in 64 bits and only the remainder is handed to sincosf.
// Measured: 16384 tokens of 80 heads (671 MB): 110 us, 6.1 TB/s, 0.93 of a copy; 4095 tokens of 72
// heads, half of each turned (151 MB): 28 us, 5.4 TB/s; three tokens: 4 us.  Element by element (rows off
// the 16-byte grid, 20 turned dims) 4095 tokens of 72 heads take 71 us against 36.
#include <algorithm>
#include <cmath>

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "../../include/apar.h"
#include "apar_internal.h"

namespace apar {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kMaxTokens = 2;                    // tokens whose angles a CTA holds

struct RopeArgs {
  double theta[kDim / 2];
  float magnitude;
  int32_t rd, interleaved, heads[2];             // q, k
  const void* in[2];
  void* out[2];
  long long in_stride[2], out_stride[2];         // elements from one token to the next
  const int32_t* positions;
  int32_t n;
};

__device__ __forceinline__ void rope_angles(const RopeArgs& a, int t0, int nt,
                                            float2 (*cs)[kDim / 2]) {
  const int half = a.rd / 2;
  for (int x = threadIdx.x; x < nt * half; x += kRopeThreads) {
    const int t = x / half, i = x % half;
    const double angle = (double)a.positions[t0 + t] * a.theta[i];
    const double turns = rint(angle * 0.15915494309189535);      // 1 / (2 pi)
    float s, c;
    sincosf((float)fma(turns, -6.283185307179586, angle), &s, &c);
    cs[t][i] = make_float2(c * a.magnitude, s * a.magnitude);
  }
  __syncthreads();
}

// One pair turned; the roundings are written out so that both kernels give the same numbers.
__device__ __forceinline__ float2 turn_pair(float a, float b, float c, float s) {
  return make_float2(fmaf(a, c, -__fmul_rn(b, s)), fmaf(b, c, __fmul_rn(a, s)));
}

// 16-byte pieces.  An item is 16 dims of one row: in the half layout the piece of 8 dims at 8 p
// and its partner at rd / 2 + 8 p (or 16 dims past rotary_dim, copied), in the interleaved one the
// 16 dims at 16 p.  Needs 16-byte aligned rows and, in the half layout, rd a multiple of 16.
__global__ void __launch_bounds__(kRopeThreads) rope_vec_kernel(const __grid_constant__ RopeArgs a,
                                                                int tokens) {
  __shared__ float2 cs[kMaxTokens][kDim / 2];
  const int t0 = blockIdx.x * tokens, nt = min(tokens, a.n - t0);
  rope_angles(a, t0, nt, cs);
  const int heads = a.heads[0] + a.heads[1], half = a.rd / 2;
  const int items = nt * heads * 8;
  for (int x = threadIdx.x; x < items; x += kRopeThreads) {
    const int p = x & 7, row = x >> 3;
    const int t = row / heads, hh = row % heads;
    const int which = hh >= a.heads[0], h = which ? hh - a.heads[0] : hh;
    const __nv_bfloat16* src = (const __nv_bfloat16*)a.in[which] +
                               (long long)(t0 + t) * a.in_stride[which] + h * kDim;
    __nv_bfloat16* dst = (__nv_bfloat16*)a.out[which] +
                         (long long)(t0 + t) * a.out_stride[which] + h * kDim;
    int d0, d1, i0;                              // the two pieces and the first pair
    bool turn;
    if (a.interleaved) {
      d0 = 16 * p;
      d1 = d0 + 8;
      i0 = 8 * p;
      turn = d0 < a.rd;
    } else {
      turn = 8 * p < half;
      d0 = turn ? 8 * p : 16 * p;                // (past the pairs: dims rd + 16 (p - half / 8))
      d1 = turn ? half + 8 * p : d0 + 8;
      i0 = 8 * p;
    }
    if (!turn && src == dst) continue;           // in place: nothing to copy
    uint4 u = *(const uint4*)(src + d0), v = *(const uint4*)(src + d1);
    if (turn) {
      uint32_t uw[4] = {u.x, u.y, u.z, u.w}, vw[4] = {v.x, v.y, v.z, v.w};
      if (a.interleaved) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          uint32_t& w = e < 4 ? uw[e] : vw[e - 4];
          if (i0 + e < half) {
            const float2 r = cs[t][i0 + e];
            const float fa = __uint_as_float(w << 16), fb = __uint_as_float(w & 0xffff0000u);
            const float2 y = turn_pair(fa, fb, r.x, r.y);
            __nv_bfloat162 o = __floats2bfloat162_rn(y.x, y.y);
            w = *(uint32_t*)&o;
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float4 r = *(const float4*)&cs[t][i0 + 2 * e];
          const float a0 = __uint_as_float(uw[e] << 16), a1 = __uint_as_float(uw[e] & 0xffff0000u);
          const float b0 = __uint_as_float(vw[e] << 16), b1 = __uint_as_float(vw[e] & 0xffff0000u);
          const float2 y0 = turn_pair(a0, b0, r.x, r.y), y1 = turn_pair(a1, b1, r.z, r.w);
          __nv_bfloat162 oa = __floats2bfloat162_rn(y0.x, y1.x);
          __nv_bfloat162 ob = __floats2bfloat162_rn(y0.y, y1.y);
          uw[e] = *(uint32_t*)&oa;
          vw[e] = *(uint32_t*)&ob;
        }
      }
      u = make_uint4(uw[0], uw[1], uw[2], uw[3]);
      v = make_uint4(vw[0], vw[1], vw[2], vw[3]);
    }
    *(uint4*)(dst + d0) = u;
    *(uint4*)(dst + d1) = v;
  }
}

// Any even rotary_dim, any alignment: single elements.  Slot i < rd / 2 of a row is a pair, the
// slots after it are two copied dims each.
__global__ void __launch_bounds__(kRopeThreads) rope_any_kernel(const __grid_constant__ RopeArgs a,
                                                                int tokens) {
  __shared__ float2 cs[kMaxTokens][kDim / 2];
  const int t0 = blockIdx.x * tokens, nt = min(tokens, a.n - t0);
  rope_angles(a, t0, nt, cs);
  const int heads = a.heads[0] + a.heads[1], half = a.rd / 2;
  const int slots = nt * heads * (kDim / 2);
  for (int x = threadIdx.x; x < slots; x += kRopeThreads) {
    const int i = x & (kDim / 2 - 1), row = x / (kDim / 2);
    const int t = row / heads, hh = row % heads;
    const int which = hh >= a.heads[0], h = which ? hh - a.heads[0] : hh;
    const __nv_bfloat16* src = (const __nv_bfloat16*)a.in[which] +
                               (long long)(t0 + t) * a.in_stride[which] + h * kDim;
    __nv_bfloat16* dst = (__nv_bfloat16*)a.out[which] +
                         (long long)(t0 + t) * a.out_stride[which] + h * kDim;
    const bool turn = i < half;
    const int d0 = a.interleaved || !turn ? 2 * i : i;
    const int d1 = a.interleaved || !turn ? d0 + 1 : half + i;
    __nv_bfloat16 u = src[d0], v = src[d1];
    if (turn) {
      const float2 r = cs[t][i];
      const float fa = __bfloat162float(u), fb = __bfloat162float(v);
      const float2 y = turn_pair(fa, fb, r.x, r.y);
      u = __float2bfloat16_rn(y.x);
      v = __float2bfloat16_rn(y.y);
    }
    dst[d0] = u;
    dst[d1] = v;
  }
}

// theta_i of every pair, in 64 bits.  Returns false for parameters out of range.
bool rope_thetas(const apar_rope_config* c, double* theta) {
  const int half = c->rotary_dim / 2;
  const double two_pi = 6.283185307179586;
  auto finite_pos = [](double x) { return x > 0.0 && std::isfinite(x); };
  if (!finite_pos(c->base)) return false;
  for (int i = 0; i < half; ++i) theta[i] = std::pow(c->base, -2.0 * i / c->rotary_dim);
  if (c->scaling == APAR_ROPE_PLAIN) return true;
  if (!finite_pos(c->factor)) return false;
  if (c->scaling == APAR_ROPE_LINEAR) {
    for (int i = 0; i < half; ++i) theta[i] /= c->factor;
    return true;
  }
  if (c->original_len <= 0 || !finite_pos(c->low) || !finite_pos(c->high) || !(c->low < c->high))
    return false;
  const double len = c->original_len;
  if (c->scaling == APAR_ROPE_BANDS) {
    for (int i = 0; i < half; ++i) {
      const double turns = len * theta[i] / two_pi;      // of this pair over the trained length
      const double t = std::min(1.0, std::max(0.0, (turns - c->low) / (c->high - c->low)));
      theta[i] = (1.0 - t) * theta[i] / c->factor + t * theta[i];
    }
    return true;
  }
  if (!(c->base > 1.0)) return false;
  auto index = [&](double turns) {                       // the pair that makes so many turns
    return c->rotary_dim * std::log(len / (turns * two_pi)) / (2.0 * std::log(c->base));
  };
  const double first = std::max(0.0, std::floor(index(c->high)));
  const double last = std::min(c->rotary_dim - 1.0, std::ceil(index(c->low)));
  for (int i = 0; i < half; ++i) {
    const double r = std::min(1.0, std::max(0.0, (i - first) / std::max(last - first, 0.001)));
    theta[i] = theta[i] / c->factor * r + theta[i] * (1.0 - r);
  }
  return true;
}

}  // namespace
}  // namespace apar

using namespace apar;

extern "C" apar_status apar_rope(const apar_rope_config* cfg, int32_t n, const int32_t* positions,
                                 int32_t num_q_heads, const void* q, int64_t q_stride, void* q_out,
                                 int64_t q_out_stride, int32_t num_kv_heads, const void* k,
                                 int64_t k_stride, void* k_out, int64_t k_out_stride,
                                 void* cuda_stream) {
  if (!cfg || n < 0 || num_q_heads < 0 || num_kv_heads < 0) return APAR_ERR_INVALID_ARG;
  if (cfg->head_dim != kDim) return APAR_ERR_UNSUPPORTED;
  if (cfg->rotary_dim < 2 || cfg->rotary_dim > kDim || cfg->rotary_dim % 2 ||
      cfg->layout < APAR_ROPE_HALF || cfg->layout > APAR_ROPE_INTERLEAVED ||
      cfg->scaling < APAR_ROPE_PLAIN || cfg->scaling > APAR_ROPE_YARN ||
      !std::isfinite(cfg->attn_scale))
    return APAR_ERR_INVALID_ARG;
  RopeArgs a;
  if (!rope_thetas(cfg, a.theta)) return APAR_ERR_INVALID_ARG;
  a.magnitude = (float)cfg->attn_scale;
  a.rd = cfg->rotary_dim;
  a.interleaved = cfg->layout == APAR_ROPE_INTERLEAVED;
  a.positions = positions;
  a.n = n;
  const void* in[2] = {q, k};
  void* out[2] = {q_out, k_out};
  const int32_t heads[2] = {num_q_heads, num_kv_heads};
  const int64_t in_stride[2] = {q_stride, k_stride}, out_stride[2] = {q_out_stride, k_out_stride};
  bool vec = a.interleaved || a.rd % 16 == 0;
  for (int w = 0; w < 2; ++w) {
    const int64_t row = (int64_t)heads[w] * kDim;
    a.heads[w] = heads[w];
    a.in[w] = in[w];
    a.out[w] = out[w];
    a.in_stride[w] = in_stride[w] ? in_stride[w] : row;
    a.out_stride[w] = out_stride[w] ? out_stride[w] : row;
    if (heads[w] == 0 || n == 0) continue;
    if (!in[w] || !out[w] || a.in_stride[w] < row || a.out_stride[w] < row)
      return APAR_ERR_INVALID_ARG;
    if (((uintptr_t)in[w] | (uintptr_t)out[w]) & 1) return APAR_ERR_INVALID_ARG;
    // in place means the same rows; any other overlap would read what was already turned
    const uintptr_t i0 = (uintptr_t)in[w], i1 = i0 + 2 * ((uintptr_t)(n - 1) * a.in_stride[w] + row);
    const uintptr_t o0 = (uintptr_t)out[w], o1 = o0 + 2 * ((uintptr_t)(n - 1) * a.out_stride[w] + row);
    if (!(i0 == o0 && a.in_stride[w] == a.out_stride[w]) && i0 < o1 && o0 < i1)
      return APAR_ERR_INVALID_ARG;
    if ((i0 | o0) & 15 || a.in_stride[w] % 8 || a.out_stride[w] % 8) vec = false;
  }
  const int64_t total_heads = (int64_t)num_q_heads + num_kv_heads;
  if (n == 0 || total_heads == 0) return APAR_OK;
  if (!positions || ((uintptr_t)positions & 3)) return APAR_ERR_INVALID_ARG;
  if (total_heads > 65536) return APAR_ERR_INVALID_ARG;
  // Two tokens to a CTA once there are enough of them to fill the machine that way: one / two / four
  // took 37 / 34 / 35 us for 4096 tokens of 72 heads, 117 / 113 / 119 for 16384 of 80, 32 / 27 / 25 for 16384
  // of 10; for 2048 of 72 and of 80 23 / 21 / 23 and 23 / 23 / 25, for 1024 14 / 15 / 17 and 14 / 16 / 18.
  const int tokens = n >= 4096 ? kMaxTokens : 1;
  const unsigned grid = (unsigned)((n + (int64_t)tokens - 1) / tokens);
  // (the launch's own status: an error that an earlier call left is neither taken for it nor lost)
  const cudaError_t e = launch_kernel(vec ? rope_vec_kernel : rope_any_kernel, dim3(grid),
                                      dim3(kRopeThreads), 0, (cudaStream_t)cuda_stream, false, a, tokens);
  if (e == cudaSuccess) return APAR_OK;
  note_cuda_error(e);
  return APAR_ERR_CUDA;
}
