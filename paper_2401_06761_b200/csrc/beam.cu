// Beam search's selection: of all (beam, token) pairs of a sequence the num_select with the highest
// score[b] + x[b][v] - lse(x[b]), where lse is the log-sum-exp of the beam's row of logits.
//
// Within one row the order of the pairs is the order of the logits, so one pass over the logits is
// enough: it keeps, per piece of a row, the num_select largest logits and the piece's maximum and sum
// of exponentials, and a second small kernel puts the pieces of a sequence's rows together.
//
// beam_scan_kernel   one CTA of eight warps per piece; the warps run on their own.  A warp reads 256
//     consecutive elements at a time, eight per lane, and compares them with a threshold that at least
//     num_select of its elements are above or equal to; the few that pass go into a buffer of 128 in
//     shared memory, which is sorted and cut back to num_select when it fills up, and the threshold
//     rises.  The first threshold is the num_select-th largest of the maxima of 64 groups of sixteen
//     elements.  A key is (ordered bits of the logit, complement of the token): of equal logits the
//     lower token is kept.
// beam_pick_kernel   one warp per sequence: each lane looks after the heads of some of the sorted
//     lists, num_select rounds of a maximum over the warp.  Scores of different beams are compared in
//     64 bits: their difference goes through two log-sum-exps, and 32 bits would round it.
#include <algorithm>
#include <climits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "../../include/apar.h"
#include "apar_internal.h"
#include "ptx.cuh"

namespace apar {
namespace {

constexpr int kWarps = 8;                     // of a scanning CTA
constexpr int kBuf = 128;                     // keys a warp holds
constexpr int kMaxSelect = 64, kMaxBeams = 64;
constexpr int kMaxPieces = 16;                // of a row
constexpr int kMaxLists = 128;                // pieces of a sequence's rows
constexpr float kLog2e = 1.4426950408889634f;
constexpr unsigned kAll = 0xffffffffu;
typedef unsigned long long u64;

__device__ __forceinline__ uint32_t ordered(float x) {   // (-0 counts as 0)
  const uint32_t b = __float_as_uint(x + 0.f);
  return b ^ (uint32_t)((int32_t)b >> 31 | 0x80000000);
}
__device__ __forceinline__ float unordered(uint32_t o) {
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}

__device__ __forceinline__ float number(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float number(__half x) { return __half2float(x); }
__device__ __forceinline__ float number(float x) { return x; }

__device__ __forceinline__ void numbers(const uint32_t* w, const __nv_bfloat16*, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void numbers(const uint32_t* w, const __half*, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = __half22float2(*(const __half2*)&w[i]);
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
__device__ __forceinline__ void numbers(const uint32_t* w, const float*, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(w[i]);
}

// Elements 8 at .. 8 at + 7 of a row; -inf past its end.  Groups are counted from the row's first
// element wherever that lies, so that two equal rows are summed in the same order and tie exactly:
// a row that begins off a 16-byte boundary (`off` elements behind one) is read in the aligned pieces
// that cover the group, which are then shifted into place.
template <typename T>
__device__ __forceinline__ void load_group(const T* row, int vocab, int off, int at, float (&x)[8]) {
  constexpr int kWords = 2 * (int)sizeof(T);           // of a group
  constexpr int kPiece = 16 / (int)sizeof(T);          // elements of 16 bytes
  const T* p = row + (int64_t)at * 8;
  if (off == 0 && at * 8 + 8 <= vocab) {
    uint32_t w[kWords];
#pragma unroll
    for (int i = 0; i < kWords / 4; ++i) *(uint4*)(w + 4 * i) = __ldg((const uint4*)p + i);
    numbers(w, row, x);
  } else if (off != 0 && at > 0 && at * 8 + 8 + kPiece - off <= vocab) {
    uint32_t w[kWords + 4];                            // (all of it inside the row)
#pragma unroll
    for (int i = 0; i < kWords / 4 + 1; ++i) *(uint4*)(w + 4 * i) = __ldg((const uint4*)(p - off) + i);
    const int words = sizeof(T) == 4 ? off : off >> 1;
    if (words & 2) {
#pragma unroll
      for (int i = 0; i < kWords + 2; ++i) w[i] = w[i + 2];
    }
    if (words & 1) {
#pragma unroll
      for (int i = 0; i < kWords + 1; ++i) w[i] = w[i + 1];
    }
    if (sizeof(T) == 2 && (off & 1)) {
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
    }
    numbers(w, row, x);
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = at * 8 + e < vocab ? number(__ldg(p + e)) : -INFINITY;
  }
}

// Sorts N keys, element N / 32 * lane + i in v[i], largest first.
template <int N, typename T>
__device__ __forceinline__ void warp_sort(T (&v)[N / 32], int lane) {
  constexpr int P = N / 32;
#pragma unroll
  for (int size = 2; size <= N; size *= 2) {
#pragma unroll
    for (int d = size / 2; d > 0; d /= 2) {
      if (d >= P) {
#pragma unroll
        for (int i = 0; i < P; ++i) {
          const T o = __shfl_xor_sync(kAll, v[i], d / P);
          const int at = lane * P + i;
          const bool big = ((at & d) == 0) == ((at & size) == 0);   // keeps the larger of the two
          v[i] = (o > v[i]) == big ? o : v[i];
        }
      } else {
#pragma unroll
        for (int i = 0; i < P; ++i) {
          if (i & d) continue;
          const bool down = ((lane * P + i) & size) == 0;
          const T a = v[i], b = v[i | d];
          const bool swap = (b > a) == down;
          v[i] = swap ? b : a;
          v[i | d] = swap ? a : b;
        }
      }
    }
  }
}

struct BeamArgs {
  const void* logits;
  int64_t seq_stride, beam_stride;   // elements
  int32_t n_seq, beams, vocab, select, pieces;
  const float* scores;
  const uint8_t* finished;
  int32_t eos;
  u64* keys;                         // [n_seq * beams * pieces][select], largest first, 0 = none
  float2* stats;                     // [n_seq * beams * pieces]: maximum, sum of 2^((x - max) log2 e)
  float* out_score;
  int32_t *out_beam, *out_token;
};

// What a warp knows of its part of a row.
struct Held {
  u64* buf;                          // kBuf keys in shared memory
  int n = 0;                         // of them in use
  float tau = -INFINITY;             // smaller elements are of no interest,
  u64 last = 0;                      // nor keys below this one
  float m = -INFINITY, l = 0.f;      // of this lane's elements
};

__device__ __forceinline__ void cut_back(Held& h, int select, int lane) {
  u64 v[kBuf / 32];
#pragma unroll
  for (int i = 0; i < kBuf / 32; ++i) {
    const int at = lane * (kBuf / 32) + i;
    v[i] = at < h.n ? h.buf[at] : 0ull;
  }
  __syncwarp();
  warp_sort<kBuf>(v, lane);
#pragma unroll
  for (int i = 0; i < kBuf / 32; ++i) h.buf[lane * (kBuf / 32) + i] = v[i];
  __syncwarp();
  if (h.n >= select) {
    h.n = select;
    h.last = h.buf[select - 1];
    h.tau = unordered((uint32_t)(h.last >> 32));
  }
}

// One element per lane; -inf where a lane has none.
__device__ __forceinline__ void offer(Held& h, float x, int token, int select, int lane) {
  const u64 key = (u64)ordered(x) << 32 | (uint32_t)~token;
  auto wanted = [&] { return x >= h.tau && x > -INFINITY && key > h.last; };   // (a NaN is not)
  unsigned who = __ballot_sync(kAll, wanted());
  if (who == 0) return;
  if (h.n + 32 > kBuf) {                       // (more than num_select are held: cut back to that many)
    cut_back(h, select, lane);
    who = __ballot_sync(kAll, wanted());
  }
  if (who >> lane & 1) h.buf[h.n + __popc(who & ((1u << lane) - 1))] = key;
  h.n += __popc(who);
  __syncwarp();
}

template <typename T>
__global__ void __launch_bounds__(kWarps * 32) beam_scan_kernel(const BeamArgs a) {
  __shared__ u64 bufs[kWarps][kBuf];
  __shared__ int counts[kWarps];
  __shared__ float2 sums[kWarps];
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int row = blockIdx.x / a.pieces, piece = blockIdx.x % a.pieces;
  const int seq = row / a.beams, beam = row % a.beams;
  const T* x = (const T*)a.logits + seq * a.seq_stride + beam * a.beam_stride;
  Held h;
  h.buf = bufs[warp];
  const bool skip = a.finished && a.finished[row];   // (has its one continuation, see the other kernel)
  if (!skip) {
    const int off = (int)((uintptr_t)x & 15) / (int)sizeof(T);
    const int groups = (a.vocab + 7) / 8;
    const int per_piece = (groups + a.pieces - 1) / a.pieces;
    const int per_warp = ((per_piece + kWarps - 1) / kWarps + 31) / 32 * 32;
    const int end = min(groups, (piece + 1) * per_piece);
    const int g0 = piece * per_piece + warp * per_warp, g1 = min(end, g0 + per_warp);
    bool first = true;
    for (int g = g0; g < g1; g += 128) {       // up to four groups a lane in flight
      float v[4][8];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int at = g + 32 * u + lane;
        if (at < g1) {
          load_group(x, a.vocab, off, at, v[u]);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) v[u][e] = -INFINITY;
        }
      }
      if (first) {
        // each group is half of what the lane holds
        uint32_t top[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float t = v[2 * k][0];
#pragma unroll
          for (int u = 2 * k; u < 2 * k + 2; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) t = fmaxf(t, v[u][e]);
          top[k] = ordered(t == t ? t : -INFINITY);
        }
        warp_sort<64>(top, lane);
        const int at = a.select - 1;           // (at least num_select elements are not below that one)
        const uint32_t t0 = __shfl_sync(kAll, top[0], at >> 1), t1 = __shfl_sync(kAll, top[1], at >> 1);
        h.tau = fmaxf(h.tau, unordered(at & 1 ? t1 : t0));
        first = false;
      }
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        float top = v[u][0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = fmaxf(top, v[u][e]);
        if (top > h.m) {
          h.l *= ex2((h.m - top) * kLog2e);
          h.m = top;
        }
        // (x - m before the factor: rounding m log2 e would be the same error in every term)
        const float ref = h.m == -INFINITY ? 0.f : h.m;
        float part = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) part += ex2((v[u][e] - ref) * kLog2e);
        h.l += part;
        if (__any_sync(kAll, top >= h.tau)) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            offer(h, v[u][e], (g + 32 * u + lane) * 8 + e, a.select, lane);
        }
      }
    }
    cut_back(h, a.select, lane);
    h.n = min(h.n, a.select);
  }
  // maximum and sum of the warp
  float m = h.m;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(kAll, m, o));
  float l = h.m == -INFINITY ? h.l : h.l * ex2((h.m - m) * kLog2e);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(kAll, l, o);
  if (lane == 0) {
    counts[warp] = h.n;
    sums[warp] = make_float2(m, l);
  }
  __syncthreads();
  if (warp != 0) return;
  // the warps' sorted lists become one
  const int mine = lane < kWarps ? lane : 0;
  int at = 0, n = lane < kWarps ? counts[mine] : 0;
  u64* out = a.keys + (size_t)blockIdx.x * a.select;
  for (int k = 0; k < a.select; ++k) {
    const u64 head = at < n ? bufs[mine][at] : 0ull;
    u64 best = head;
#pragma unroll
    for (int o = kWarps / 2; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(kAll, best, o));
    if (best != 0 && head == best) ++at;
    if (lane == 0) out[k] = best;
  }
  float2 s = sums[mine];
  float M = s.x;
#pragma unroll
  for (int o = kWarps / 2; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(kAll, M, o));
  float L = s.x == -INFINITY ? s.y : s.y * ex2((s.x - M) * kLog2e);
#pragma unroll
  for (int o = kWarps / 2; o > 0; o >>= 1) L += __shfl_xor_sync(kAll, L, o);
  if (lane == 0) a.stats[blockIdx.x] = make_float2(M, L);
}

// A pair's place in the order: larger value first, then lower beam, then lower token.
struct Pair {
  double value;
  uint32_t beam, token;
};
__device__ __forceinline__ bool before(const Pair& a, const Pair& b) {
  if (a.value != b.value) return a.value > b.value;
  return a.beam != b.beam ? a.beam < b.beam : a.token < b.token;
}

__global__ void __launch_bounds__(32) beam_pick_kernel(const BeamArgs a) {
  extern __shared__ u64 lists[];                       // [beams * pieces][select]
  __shared__ double base[kMaxBeams];                   // score - lse; NaN: the beam has no pairs
  const int lane = threadIdx.x, seq = blockIdx.x, n_lists = a.beams * a.pieces;
  pdl_wait();                                          // (the scan has written its lists)
  const u64* src = a.keys + (size_t)seq * n_lists * a.select;
  for (int i = lane; i < n_lists * a.select; i += 32) lists[i] = src[i];
  for (int b = lane; b < a.beams; b += 32) {
    const int row = seq * a.beams + b;
    const float score = a.scores[row];
    double to = NAN;
    if (score - score == 0.f) {                        // finite
      if (a.finished && a.finished[row]) {
        to = score;
      } else {
        float M = -INFINITY;
        for (int p = 0; p < a.pieces; ++p) M = fmaxf(M, a.stats[row * a.pieces + p].x);
        double L = 0.0;
        for (int p = 0; p < a.pieces; ++p) {
          const float2 s = a.stats[row * a.pieces + p];
          L += s.x == -INFINITY ? (double)s.y : (double)s.y * exp((double)s.x - (double)M);
        }
        const double lse = (double)M + log(L);
        if (lse - lse == 0.0) to = (double)score - lse;
      }
    }
    base[b] = to;
  }
  __syncwarp();
  // this lane's lists are lane, lane + 32, ...; at[j] is how far list j has been used
  int at[kMaxLists / 32];
#pragma unroll
  for (int j = 0; j < kMaxLists / 32; ++j) at[j] = 0;
  for (int k = 0; k < a.select; ++k) {
    Pair best{-INFINITY, 0xffffffffu, 0xffffffffu};
    int from = -1;
#pragma unroll
    for (int j = 0; j < kMaxLists / 32; ++j) {
      const int list = lane + 32 * j;
      if (list >= n_lists || at[j] >= a.select) continue;
      const uint32_t b = list / a.pieces;
      const double to = base[b];
      Pair p;
      p.beam = b;
      if (a.finished && a.finished[seq * a.beams + b]) {
        if (at[j] > 0 || list % a.pieces) continue;
        p.value = to;
        p.token = (uint32_t)a.eos;
      } else {
        const u64 key = lists[list * a.select + at[j]];
        if (key == 0) continue;
        p.value = to + (double)unordered((uint32_t)(key >> 32));
        p.token = ~(uint32_t)key;
      }
      if (!(p.value > -INFINITY)) continue;            // (NaN: the beam has no pairs)
      if (from < 0 || before(p, best)) {
        best = p;
        from = j;
      }
    }
    Pair w = best;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      Pair x;
      x.value = __shfl_xor_sync(kAll, w.value, o);
      x.beam = __shfl_xor_sync(kAll, w.beam, o);
      x.token = __shfl_xor_sync(kAll, w.token, o);
      if (before(x, w)) w = x;
    }
#pragma unroll
    for (int j = 0; j < kMaxLists / 32; ++j)
      if (j == from && best.beam == w.beam && best.token == w.token) ++at[j];
    if (lane == 0) {
      const size_t o = (size_t)seq * a.select + k;
      a.out_score[o] = (float)w.value;                 // (rounded once; -inf where pairs ran out)
      a.out_beam[o] = (int32_t)w.beam;
      a.out_token[o] = (int32_t)w.token;
    }
  }
}

// Pieces of a row: enough CTAs to fill the machine twice over where there are few rows, none shorter
// than 2048 elements.
int pieces_of(const apar_beam_config* c, int32_t n_seq) {
  const int64_t rows = (int64_t)n_seq * c->num_beams;
  int64_t p = std::min<int64_t>({kMaxPieces, (2 * 148 + rows - 1) / rows, (c->vocab + 2047) / 2048,
                                 kMaxLists / c->num_beams});
  return (int)std::max<int64_t>(1, p);
}

bool valid(const apar_beam_config* c, int32_t n_seq) {
  return c && n_seq >= 0 && c->vocab > 0 && c->num_beams > 0 && c->num_beams <= kMaxBeams &&
         c->num_select > 0 && c->num_select <= kMaxSelect && c->logits_type >= APAR_LOGITS_BF16 &&
         c->logits_type <= APAR_LOGITS_F32 && c->eos >= -1 && c->eos < c->vocab &&
         c->vocab < (1 << 28) &&
         (int64_t)n_seq * c->num_beams * kMaxPieces < INT32_MAX / kMaxSelect;
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }

}  // namespace
}  // namespace apar

using namespace apar;

extern "C" size_t apar_beam_workspace_bytes(const apar_beam_config* cfg, int32_t n_seq) {
  if (!valid(cfg, n_seq)) return 0;
  if (n_seq == 0) return 256;
  const size_t lists = (size_t)n_seq * cfg->num_beams * pieces_of(cfg, n_seq);
  return align256(lists * cfg->num_select * sizeof(u64)) + align256(lists * sizeof(float2));
}

extern "C" apar_status apar_beam_select(const apar_beam_config* cfg, int32_t n_seq, const void* logits,
                                        int64_t seq_stride, int64_t beam_stride, const float* scores,
                                        const uint8_t* finished, float* out_score, int32_t* out_beam,
                                        int32_t* out_token, void* workspace, size_t workspace_bytes,
                                        void* cuda_stream) {
  if (!valid(cfg, n_seq)) return APAR_ERR_INVALID_ARG;
  if (n_seq == 0) return APAR_OK;
  if (!logits || !scores || !out_score || !out_beam || !out_token || !workspace)
    return APAR_ERR_INVALID_ARG;
  const uintptr_t size = cfg->logits_type == APAR_LOGITS_F32 ? 4 : 2;
  if (((uintptr_t)logits & (size - 1)) || ((uintptr_t)workspace & 255) ||
      (((uintptr_t)scores | (uintptr_t)out_score | (uintptr_t)out_beam | (uintptr_t)out_token) & 3))
    return APAR_ERR_INVALID_ARG;
  if (finished && cfg->eos < 0) return APAR_ERR_INVALID_ARG;
  if (workspace_bytes < apar_beam_workspace_bytes(cfg, n_seq)) return APAR_ERR_WORKSPACE_TOO_SMALL;
  BeamArgs a;
  a.logits = logits;
  a.seq_stride = seq_stride ? seq_stride : (int64_t)cfg->num_beams * cfg->vocab;
  a.beam_stride = beam_stride ? beam_stride : cfg->vocab;
  a.n_seq = n_seq;
  a.beams = cfg->num_beams;
  a.vocab = cfg->vocab;
  a.select = cfg->num_select;
  a.pieces = pieces_of(cfg, n_seq);
  a.scores = scores;
  a.finished = finished;
  a.eos = cfg->eos;
  const int lists = n_seq * a.beams * a.pieces;
  a.keys = (u64*)workspace;
  a.stats = (float2*)((char*)workspace + align256((size_t)lists * a.select * sizeof(u64)));
  a.out_score = out_score;
  a.out_beam = out_beam;
  a.out_token = out_token;
  const cudaStream_t st = (cudaStream_t)cuda_stream;
  auto scan = cfg->logits_type == APAR_LOGITS_F32   ? beam_scan_kernel<float>
              : cfg->logits_type == APAR_LOGITS_F16 ? beam_scan_kernel<__half>
                                                    : beam_scan_kernel<__nv_bfloat16>;
  const size_t smem = (size_t)a.beams * a.pieces * a.select * sizeof(u64);
  cudaError_t e = cudaSuccess;
  if (smem > 48 * 1024)
    e = cudaFuncSetAttribute(beam_pick_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             kMaxLists * kMaxSelect * (int)sizeof(u64));
  if (e == cudaSuccess) e = launch_kernel(scan, dim3(lists), dim3(kWarps * 32), 0, st, false, a);
  if (e == cudaSuccess) e = launch_kernel(beam_pick_kernel, dim3(n_seq), dim3(32), smem, st, true, a);
  if (e != cudaSuccess) {
    note_cuda_error(e);
    return APAR_ERR_CUDA;
  }
  return APAR_OK;
}
