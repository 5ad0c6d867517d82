// Beam search's selection: of all (beam, token) pairs of a sequence the num_select with the highest
// score[b] + x[b][v] - lse(x[b]), where lse is the log-sum-exp of the beam's row of logits.
//
// Within one row the order of the pairs is the order of the logits, so one pass over the logits is
// enough: it keeps, per piece of a row, the num_select largest logits and the piece's maximum and sum
// of exponentials, and a second small kernel puts the pieces of a sequence's rows together.
//
// beam_scan_kernel   one CTA per piece of a row.  A thread goes over its elements a step of 16 at a time,
//     sixteen bytes to a load where the row begins on such a boundary, the next step's on their way
//     meanwhile, and keeps the largest, a sum of 2^((x - a reference) log2 e) and, in shared memory, each step's
//     largest.  Which thread holds which element, and so the order of the sums, depends on the element
//     alone: equal rows tie exactly.  A threshold that at least num_select elements reach comes from the
//     threads' maxima: with j = num_select / 8 rounded up, the least of the eight warps' j-th largest.
//     The steps that reach it (some two to three times num_select; the exact num_select-th largest of the
//     maxima leaves fewer, but takes longer than it saves) are read again, the elements that do collected
//     and put in order by counting, for each, how many are larger.  A key is (ordered bits of the logit,
//     complement of the token): of equal logits the lower token is kept.  Where more than 512 elements
//     reach the threshold (many equal ones) the warps go over the piece again with buffers that they
//     sort and cut back as they fill.
// beam_rows_kernel   the same for many short rows, a warp each.
// beam_pick_kernel   one CTA per sequence: a threshold by halving (the beams' scores differ too much for
//     the one above), and the few pairs that reach it ordered by counting.  Values of different beams are
//     compared in 64 bits: their difference goes through two log-sum-exps, and 32 bits would round it.
//
// Bound: HBM, 4 bytes per f32 logit, and one special-function operation for each.  2048 rows of 32003 f32
// logits, a fifth of them finished (208 MB read): scan 48.5 us, 4.3 TB/s; 10 of them are the end of a piece
// (threshold, collecting, ordering), a chain of short steps that the SM's other CTAs cover in part.  128 rows
// of 131072 bf16 logits: 13.8 us, 2.4 TB/s.  4 rows of 32000: 4 us, then 5 for the pick; that of 64 pairs for
// 16 sequences of 64 beams takes 35.  (Tried: the next step's copies into shared memory meanwhile, and whole
// pieces in registers until the end: 73 and 55 us.)
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

constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr int kCand = 512;                    // elements that may reach a threshold
constexpr int kBuf = 128;                     // keys a warp holds where more do
constexpr int kMaxSelect = 64, kMaxBeams = 64;
constexpr int kMaxPieces = 16;                // of a row
constexpr int kMaxLists = 128;                // pieces of a sequence's rows
// SMs that rows are cut for.  A constant, as the scratch depends on it and its size may be asked for where there is no
// device; on a part of a B200 the pieces are as right, if more than they need be.
constexpr int kSms = 148;
constexpr float kLog2e = 1.4426950408889634f;
constexpr unsigned kAll = 0xffffffffu;
typedef unsigned long long u64;

__device__ __forceinline__ u64 pair_of(float a, float b) {
  return (u64)__float_as_uint(b) << 32 | __float_as_uint(a);
}
__device__ __forceinline__ float2 parts_of(u64 p) {
  return make_float2(__uint_as_float((uint32_t)p), __uint_as_float((uint32_t)(p >> 32)));
}
__device__ __forceinline__ u64 mul2(u64 a, u64 b) {
  u64 d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ u64 add2(u64 a, u64 b) {
  u64 d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}

__device__ __forceinline__ uint32_t ordered(float x) {   // (-0 counts as 0)
  const uint32_t b = __float_as_uint(x + 0.f);
  return b ^ (uint32_t)((int32_t)b >> 31 | 0x80000000);
}
__device__ __forceinline__ float unordered(uint32_t o) {   // (what is below -inf counts as that)
  if (o < 0x007fffffu) return -INFINITY;
  return __uint_as_float(o & 0x80000000u ? o ^ 0x80000000u : ~o);
}

// A row's elements in packs of sixteen bytes.  (f32: 2 packs a step and 6 CTAs of an SM 54 us, 3 and 5 54,
// 4 and 4 50; 16-bit: 1 and 6 20 us, 2 and 5 13.4, 4 and 3 15.)
__device__ __forceinline__ float number(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float number(__half x) { return __half2float(x); }
__device__ __forceinline__ float number(float x) { return x; }
template <typename T>
struct Packs;
template <>
struct Packs<float> {
  static constexpr int kPer = 4, kHeld = 4, kCtas = 4; // a pack's elements, packs of a step, CTAs of an SM
  static constexpr uint32_t kNone = 0xff800000u;       // -inf
  static __device__ __forceinline__ void numbers(uint4 w, float (&x)[4]) {
    x[0] = __uint_as_float(w.x);
    x[1] = __uint_as_float(w.y);
    x[2] = __uint_as_float(w.z);
    x[3] = __uint_as_float(w.w);
  }
};
template <>
struct Packs<__nv_bfloat16> {
  static constexpr int kPer = 8, kHeld = 2, kCtas = 5;
  static constexpr uint32_t kNone = 0xff80ff80u;
  static __device__ __forceinline__ void numbers(uint4 w, float (&x)[8]) {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xffff0000u);
    }
  }
};
template <>
struct Packs<__half> {
  static constexpr int kPer = 8, kHeld = 2, kCtas = 5;
  static constexpr uint32_t kNone = 0xfc00fc00u;
  static __device__ __forceinline__ void numbers(uint4 w, float (&x)[8]) {
    const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*(const __half2*)&v[i]);
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  }
};
__device__ __forceinline__ float max3(float a, float b, float c) {   // (a NaN counts as less than everything)
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
template <int N>
__device__ __forceinline__ float largest(float m, const float (&x)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 2) m = max3(m, x[i], x[i + 1]);
  return m;
}
// A whole pack from an address on a boundary of kAlign bytes.
template <int kAlign>
__device__ __forceinline__ uint4 load_pack(const void* p) {
  if constexpr (kAlign == 16) {
    return __ldg((const uint4*)p);
  } else {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      w[i] = kAlign == 4 ? __ldg((const uint32_t*)p + i)
                         : (uint32_t)__ldg((const uint16_t*)p + 2 * i) |
                               (uint32_t)__ldg((const uint16_t*)p + 2 * i + 1) << 16;
    return make_uint4(w[0], w[1], w[2], w[3]);
  }
}
// This thread's packs at0, at0 + kStride, ... of the n elements of a row; what lies past them is -inf.
template <typename T, int kAlign, int kStride, int kN>
__device__ __forceinline__ void load_packs(uint4 (&v)[kN], const T* row, int n, int at0) {
  constexpr int kPer = Packs<T>::kPer;
#pragma unroll
  for (int k = 0; k < kN; ++k) {
    const int at = at0 + k * kStride;
    v[k] = make_uint4(Packs<T>::kNone, Packs<T>::kNone, Packs<T>::kNone, Packs<T>::kNone);
    if ((at + 1) * kPer <= n) v[k] = load_pack<kAlign>(row + (int64_t)at * kPer);
  }
  const int last = n / kPer, k_last = (last - at0) / kStride;     // the pack that the row's end cuts
  if (n % kPer && last >= at0 && (last - at0) % kStride == 0) {
    alignas(16) T x[kPer];
    const uint32_t none = Packs<T>::kNone;
#pragma unroll
    for (int i = 0; i < kPer; ++i) x[i] = last * kPer + i < n ? row[last * kPer + i] : *(const T*)&none;
#pragma unroll
    for (int k = 0; k < kN; ++k)
      if (k == k_last) v[k] = *(const uint4*)x;
  }
}
// (whatever the row's alignment)
template <typename T, int kStride, int kN>
__device__ __forceinline__ void load_packs(uint4 (&v)[kN], const T* row, int n, int at0) {
  if (((uintptr_t)row & 15) == 0) load_packs<T, 16, kStride>(v, row, n, at0);
  else if (sizeof(T) == 4 || ((uintptr_t)row & 3) == 0) load_packs<T, 4, kStride>(v, row, n, at0);
  else load_packs<T, 2, kStride>(v, row, n, at0);
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

// A value that at least `select` of the CTA's threads' maxima (as ordered integers) reach: the least of
// the j-th largest of the first `full` warps, all of whose threads have something.  The least there is
// where those warps are too few.  *most receives the largest of all.  `sh`: 2 * kWarps words.
__device__ __forceinline__ uint32_t threshold(uint32_t mine, int select, int full, uint32_t* sh,
                                              uint32_t* most) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t rest = mine, top = __reduce_max_sync(kAll, mine);
  if (lane == 0) sh[warp] = top;
  full = min(full, kWarps);
  if (full * 32 < select) full = 0;
  for (int j = full ? (select + full - 1) / full : 0; j > 1; --j) {
    // (one of those that hold the largest steps back)
    if (lane == __ffs(__ballot_sync(kAll, rest == top)) - 1) rest = 0;
    top = __reduce_max_sync(kAll, rest);
  }
  if (lane == 0) sh[kWarps + warp] = top;
  __syncthreads();
  uint32_t least = 0xffffffffu, m = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    m = max(m, sh[w]);
    if (w < full) least = min(least, sh[kWarps + w]);
  }
  *most = m;
  return full ? least : 0;
}

// ------------------------------------------------------------------ pieces with many equal elements
__device__ __forceinline__ void warp_sort(u64 (&v)[kBuf / 32], int lane) {   // largest first
  constexpr int P = kBuf / 32;
#pragma unroll 1
  for (int size = 2; size <= kBuf; size *= 2) {
#pragma unroll 1
    for (int d = size / 2; d >= P; d /= 2) {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        const u64 o = __shfl_xor_sync(kAll, v[i], d / P);
        const int at = lane * P + i;
        const bool big = ((at & d) == 0) == ((at & size) == 0);   // keeps the larger of the two
        v[i] = (o > v[i]) == big ? o : v[i];
      }
    }
#pragma unroll
    for (int d = P / 2; d > 0; d /= 2) {
      if (d >= size) continue;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        if (i & d) continue;
        const bool down = ((lane * P + i) & size) == 0;
        const u64 a = v[i], b = v[i | d];
        const bool swap = (b > a) == down;
        v[i] = swap ? b : a;
        v[i | d] = swap ? a : b;
      }
    }
  }
}

// Cuts a warp's buffer of n keys back to its `select` largest, sorted; returns how many there are.
__device__ __noinline__ int cut_back(u64* buf, int n, int select) {
  const int lane = threadIdx.x & 31;
  u64 v[kBuf / 32];
#pragma unroll
  for (int i = 0; i < kBuf / 32; ++i) {
    const int at = lane * (kBuf / 32) + i;
    v[i] = at < n ? buf[at] : 0ull;
  }
  __syncwarp();
  warp_sort(v, lane);
#pragma unroll
  for (int i = 0; i < kBuf / 32; ++i) buf[lane * (kBuf / 32) + i] = v[i];
  __syncwarp();
  return min(n, select);
}

// The `select` largest of the elements [e0, e1) that reach tau, one warp; sorted into buf, their number
// returned.
template <typename T>
__device__ int scan_again(const T* row, int e0, int e1, float tau, int select, u64* buf) {
  const int lane = threadIdx.x & 31;
  int n = 0;
  u64 last = 0;                                // keys below this one are of no use
  for (int e = e0; e < e1; e += 32) {
    const float x = e + lane < e1 ? number(row[e + lane]) : -INFINITY;
    const u64 key = (u64)ordered(x) << 32 | (uint32_t)~(e + lane);
    const bool in = x >= tau && x > -INFINITY;             // (a NaN is not)
    unsigned who = __ballot_sync(kAll, in && key > last);
    if (who == 0) continue;
    if (n + 32 > kBuf) {                       // (more than num_select are held)
      n = cut_back(buf, n, select);
      last = buf[n - 1];
      who = __ballot_sync(kAll, in && key > last);
    }
    if (who >> lane & 1) buf[n + __popc(who & ((1u << lane) - 1))] = key;
    n += __popc(who);
    __syncwarp();
  }
  return cut_back(buf, n, select);
}

// ------------------------------------------------------------------ pieces of rows
constexpr int kSlots = 16;
union ScanKeys {
  u64 cand[kCand];
  u64 bufs[kWarps][kBuf];
};

template <typename T>
__global__ void __launch_bounds__(kThreads, Packs<T>::kCtas) beam_scan_kernel(const BeamArgs a) {
  using W = Packs<T>;
  constexpr int kPer = W::kPer, kHeld = W::kHeld, kChunk = kThreads * kHeld;   // packs of a round
  __shared__ ScanKeys sh;
  __shared__ uint32_t tops[2 * kWarps];
  __shared__ float sums[kWarps];
  __shared__ int counts[kWarps], n_cand, n_hit;
  __shared__ float peaks[kSlots][kThreads];    // largest of so many steps of a thread
  __shared__ uint16_t hit[kCand];              // (slot, thread) that has something that reaches the threshold
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int row = blockIdx.x / a.pieces, piece = blockIdx.x % a.pieces;
  const int seq = row / a.beams, beam = row % a.beams;
  const T* x = (const T*)a.logits + seq * a.seq_stride + beam * a.beam_stride;
  const int packs = (a.vocab + kPer - 1) / kPer, per_piece = (packs + a.pieces - 1) / a.pieces;
  const int begin = piece * per_piece, end = min(packs, begin + per_piece);
  const int n_in = min(a.vocab, end * kPer);   // elements before this one are the piece's
  u64* keys = a.keys + (size_t)blockIdx.x * a.select;
  if (begin >= end || (a.finished && a.finished[row])) {   // (has its one continuation, see the other kernel)
    if ((int)threadIdx.x < a.select) keys[threadIdx.x] = 0ull;
    if (threadIdx.x == 0) a.stats[blockIdx.x] = make_float2(-INFINITY, 0.f);
    return;
  }
  if (threadIdx.x == 0) n_cand = n_hit = 0;
  // ---- this thread's elements: the largest, and the sum of 2^((x - ref) log2 e).  (The difference first: no
  // logit is too large or, as the lowest number of its type, too small for it.)  The reference follows the
  // largest once that is 8 above it, so that a slowly rising row's sum is not scaled, and rounded, at every
  // step; 128 terms at most are added up in 32 bits, in two sums, and their totals in 64, however long the row.
  float mine = -INFINITY, ref = -INFINITY;
  u64 part = 0;                                // two sums
  double total = 0.0;
  const u64 scale = pair_of(kLog2e, kLog2e);
  auto load = [&](uint4 (&v)[kHeld], int c0) { load_packs<T, kThreads>(v, x, n_in, c0 + threadIdx.x); };
  const int steps = (end - begin + kChunk - 1) / kChunk, of_slot = (steps + kSlots - 1) / kSlots;
  int slot = 0, left = of_slot;
  float peak = -INFINITY;
  auto add = [&](const uint4 (&v)[kHeld]) {
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
      float e[kPer];
      W::numbers(v[k], e);
      peak = largest(peak, e);
    }
    mine = fmaxf(mine, peak);
    if (mine > ref + 8.f) {
      const float less = ref == -INFINITY ? 0.f : ex2((ref - mine) * kLog2e);
      part = mul2(part, pair_of(less, less));
      total *= less;
      ref = mine;
    }
    if (--left == 0) {
      peaks[slot++][threadIdx.x] = peak;
      peak = -INFINITY;
      left = of_slot;
    }
    const float from = ref == -INFINITY ? 0.f : ref;
    const u64 minus = pair_of(-from, -from);
#pragma unroll
    for (int k = 0; k < kHeld; ++k) {
      float e[kPer];
      W::numbers(v[k], e);
#pragma unroll
      for (int i = 0; i < kPer; i += 2) {
        const float2 p = parts_of(mul2(add2(pair_of(e[i], e[i + 1]), minus), scale));
        part = add2(part, pair_of(ex2(p.x), ex2(p.y)));
      }
    }
  };
  auto fold = [&]() {
    total += (double)parts_of(part).x + (double)parts_of(part).y;
    part = 0;
  };
  uint4 v0[kHeld], v1[kHeld];                  // one on its way while the other is added
  load(v0, begin);
#pragma unroll 1
  for (int c0 = begin; c0 < end; c0 += 2 * kChunk) {
    if (c0 + kChunk < end) load(v1, c0 + kChunk);
    add(v0);
    if (c0 + kChunk >= end) break;
    if (c0 + 2 * kChunk < end) load(v0, c0 + 2 * kChunk);
    add(v1);
    if (((c0 - begin) & 7 * kChunk) == 6 * kChunk) fold();   // (after eight steps)
  }
  if (left != of_slot) peaks[slot++][threadIdx.x] = peak;
  // ---- the threads together
  uint32_t most;
  const float tau = unordered(threshold(ordered(mine), a.select, (end - begin) / 32, tops, &most));
  if (mine >= tau && mine > -INFINITY)
    for (int k = 0; k < slot; ++k)
      if (peaks[k][threadIdx.x] >= tau && peaks[k][threadIdx.x] > -INFINITY) {
        const int at = atomicAdd(&n_hit, 1);
        if (at < kCand) hit[at] = (uint16_t)(k * kThreads + threadIdx.x);
      }
  const float top = unordered(most);
  fold();
  float sum = (float)total;
  if (ref != top) sum *= ex2((ref - top) * kLog2e);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kAll, sum, o);
  if (lane == 0) sums[warp] = sum;
  __syncthreads();
  if (threadIdx.x == 0) {
    float s = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) s += sums[w];
    a.stats[blockIdx.x] = make_float2(top, s);
  }
  // The few elements that reach the threshold: where there is one, the packs are read again, by a thread each.
  // (Looked for by the threads that hold them, they take longer than all the exponentials.)
  const int n_again = n_hit, of_hit = of_slot * kHeld;
  for (int i = threadIdx.x; i < n_again * of_hit && n_again <= kCand; i += kThreads) {
    const int t = i / of_hit, h = hit[t];
    const int at = begin + (h / kThreads * of_hit + i - t * of_hit) * kThreads + h % kThreads;
    if (at >= end) continue;
    float e[kPer];
    if (((uintptr_t)x & 15) == 0 && (at + 1) * kPer <= n_in) {
      W::numbers(load_pack<16>(x + (int64_t)at * kPer), e);
    } else {
#pragma unroll
      for (int k = 0; k < kPer; ++k) e[k] = at * kPer + k < n_in ? number(x[at * kPer + k]) : -INFINITY;
    }
    if (!(largest(-INFINITY, e) >= tau)) continue;
    int put = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) put += e[k] >= tau && e[k] > -INFINITY;
    put = atomicAdd(&n_cand, put);
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      if (!(e[k] >= tau && e[k] > -INFINITY)) continue;
      if (put < kCand) sh.cand[put] = (u64)ordered(e[k]) << 32 | (uint32_t)~(at * kPer + k);
      ++put;
    }
  }
  __syncthreads();
  const int n = n_cand;
  if (n <= kCand && n_again <= kCand) {
    // (four threads to each of them; their order in the list does not matter)
    for (int i0 = 0; i0 < n; i0 += kThreads / 4) {
      const int i = i0 + threadIdx.x / 4;
      const u64 key = i < n ? sh.cand[i] : 0ull;
      int rank = 0;
      for (int j = threadIdx.x & 3; j < n; j += 4) rank += sh.cand[j] > key;
      rank += __shfl_xor_sync(kAll, rank, 1);
      rank += __shfl_xor_sync(kAll, rank, 2);
      if (i < n && rank < a.select && (threadIdx.x & 3) == 0) keys[rank] = key;
    }
    if ((int)threadIdx.x >= n && (int)threadIdx.x < a.select) keys[threadIdx.x] = 0ull;
    return;
  }
  const int per_warp = ((end - begin + kWarps - 1) / kWarps) * kPer, first = begin * kPer + warp * per_warp;
  const int found = scan_again(x, min(n_in, first), min(n_in, first + per_warp), tau, a.select, sh.bufs[warp]);
  if (lane == 0) counts[warp] = found;
  __syncthreads();
  if (warp != 0) return;
  // the warps' sorted lists become one
  int at = 0, have = lane < kWarps ? counts[lane] : 0;
  for (int k = 0; k < a.select; ++k) {
    const u64 head = at < have ? sh.bufs[lane & (kWarps - 1)][at] : 0ull;
    u64 most_of = head;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) most_of = max(most_of, __shfl_xor_sync(kAll, most_of, o));
    if (head == most_of) ++at;
    if (lane == 0) keys[k] = most_of;
  }
}

// ------------------------------------------------------------------ short rows
// A warp to a row of up to 2048 elements, which it holds in registers.  The threshold by halving, counting
// elements: no waits between warps, and few candidates even where half of a row's elements is asked for.  Taken
// where there are more rows than CTAs of the other kernel run at a time (64000 rows of 1000, 32 pairs, f32: 195
// us and 542, 64 pairs, bf16: 259 and 855; 16000 of 1500: 45 and 121; 800 of 2048: 6.8 and 8.9; but 256 of
// 2000: 8.4 and 6.3, one: 8.9 and 6.5).  Bound by instruction issue.
constexpr int kShort = 2048, kShortRows = 4 * kSms;
template <typename T>
__global__ void __launch_bounds__(kThreads, 2) beam_rows_kernel(const BeamArgs a) {
  using W = Packs<T>;
  constexpr int kPer = W::kPer, kN = kShort / kPer / 32;
  __shared__ u64 bufs[kWarps][kBuf];
  pdl_launch_dependents();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, row = blockIdx.x * kWarps + warp;
  if (row >= a.n_seq * a.beams) return;
  const int seq = row / a.beams, beam = row % a.beams;
  u64* keys = a.keys + (size_t)row * a.select;
  if (a.finished && a.finished[row]) {
    for (int i = lane; i < a.select; i += 32) keys[i] = 0ull;
    if (lane == 0) a.stats[row] = make_float2(-INFINITY, 0.f);
    return;
  }
  const T* x = (const T*)a.logits + seq * a.seq_stride + beam * a.beam_stride;
  uint4 v[kN];
  load_packs<T, 32>(v, x, a.vocab, lane);
  const int used = (a.vocab + 32 * kPer - 1) / (32 * kPer);   // packs of a lane
  float mine = -INFINITY;
#pragma unroll
  for (int k = 0; k < kN; ++k) {
    float e[kPer];
    W::numbers(v[k], e);
    mine = largest(mine, e);
  }
  const float top = unordered(__reduce_max_sync(kAll, ordered(mine)));
  const float from = top == -INFINITY ? 0.f : top;
  const u64 minus = pair_of(-from, -from), scale = pair_of(kLog2e, kLog2e);
  u64 part = 0;
#pragma unroll
  for (int k = 0; k < kN; ++k) {
    if (k >= used) break;
    float e[kPer];
    W::numbers(v[k], e);
#pragma unroll
    for (int i = 0; i < kPer; i += 2) {
      const float2 p = parts_of(mul2(add2(pair_of(e[i], e[i + 1]), minus), scale));
      part = add2(part, pair_of(ex2(p.x), ex2(p.y)));
    }
  }
  float sum = parts_of(part).x + parts_of(part).y;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kAll, sum, o);
  if (lane == 0) a.stats[row] = make_float2(top, sum);
  // elements of this lane that reach t (and are above -inf)
  auto here = [&](float t) {
    int c = 0;
#pragma unroll
    for (int k = 0; k < kN; ++k) {
      if (k >= used) break;
      float e[kPer];
      W::numbers(v[k], e);
#pragma unroll
      for (int i = 0; i < kPer; ++i) c += e[i] >= t;
    }
    return c;
  };
  float tau = -INFINITY, above = top;
  int reach = 0;
  if (a.select <= 16) {
    // the num_select-th largest of the lanes' maxima: at least as many elements reach it (16000 rows of 1500, 16
    // pairs: 45 us, without this 52; but with 32 pairs of 64000 rows 209 and 184)
    uint32_t rest = ordered(mine), t = 0;
    for (int j = 0; j < a.select; ++j) {
      t = __reduce_max_sync(kAll, rest);
      if (lane == __ffs(__ballot_sync(kAll, rest == t)) - 1) rest = 0;
    }
    tau = unordered(t);
  }
  if (tau == -INFINITY) {                      // (or there are not so many: down from the largest)
    tau = top;
    for (float width = 1.f; reach < a.select && tau > -3e38f; width *= 4.f) {
      above = tau;
      tau = top - width;
      reach = __reduce_add_sync(kAll, here(tau));
    }
    if (reach < a.select) tau = -3.4028235e38f;
  }
  reach = __reduce_add_sync(kAll, here(tau));
  for (int i = 0; i < 24 && reach > min(kBuf, 2 * a.select + 16); ++i) {
    const float mid = 0.5f * tau + 0.5f * above;
    const int n = __reduce_add_sync(kAll, here(mid));
    if (n >= a.select) {
      tau = mid;
      reach = n;
    } else {
      above = mid;
    }
  }
  u64* buf = bufs[warp];
  if (reach > kBuf) {                          // many equal ones
    const int n = scan_again(x, 0, a.vocab, tau, a.select, buf);
    for (int i = lane; i < a.select; i += 32) keys[i] = i < n ? buf[i] : 0ull;
    return;
  }
  int at = here(tau);
  {
    const int c = at;
#pragma unroll
    for (int o = 1; o < 32; o *= 2) {
      const int up = __shfl_up_sync(kAll, at, o);
      if (lane >= o) at += up;
    }
    at -= c;
  }
#pragma unroll
  for (int k = 0; k < kN; ++k) {
    if (k >= used) break;
    float e[kPer];
    W::numbers(v[k], e);
    if (!(largest(-INFINITY, e) >= tau)) continue;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (e[i] >= tau) buf[at++] = (u64)ordered(e[i]) << 32 | (uint32_t)~((k * 32 + lane) * kPer + i);
  }
  __syncwarp();
  for (int i = lane; i < reach; i += 32) {
    const u64 key = buf[i];
    int rank = 0;
    for (int j = 0; j < reach; ++j) rank += buf[j] > key;
    if (rank < a.select) keys[rank] = key;
  }
  for (int i = reach + lane; i < a.select; i += 32) keys[i] = 0ull;
}

// ------------------------------------------------------------------ sequences
// A pair's place in the order: larger value first, then lower beam, then lower token.
struct Pair {
  double value;
  u64 at;                                      // beam << 32 | token
};
__device__ __forceinline__ bool before(const Pair& a, const Pair& b) {
  return a.value != b.value ? a.value > b.value : a.at < b.at;
}

__global__ void __launch_bounds__(kThreads) beam_pick_kernel(const BeamArgs a) {
  __shared__ Pair cand[kCand];
  __shared__ double base[kMaxBeams];           // score - (lse - largest logit); NaN: the beam has no pairs
  __shared__ float2 stats[kMaxLists], terms[kMaxLists];
  __shared__ uint8_t over[kMaxBeams];
  __shared__ float vals[kMaxLists * kMaxSelect];   // rounded; a thread's own
  __shared__ uint32_t tops[kWarps];
  __shared__ int counts[2][kWarps], n_cand;
  __shared__ Pair picks[kWarps];
  const int seq = blockIdx.x, n_lists = a.beams * a.pieces, n_all = n_lists * a.select;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  pdl_wait();                                  // (the scan has written its lists)
  // (everything that is needed first is asked for at once)
  const u64* keys = a.keys + (size_t)seq * n_all;
  constexpr int kAhead = 4;
  u64 ahead[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k) {
    const int i = threadIdx.x + k * kThreads;
    ahead[k] = i < n_all ? keys[i] : 0ull;
  }
  const int b = threadIdx.x, row = seq * a.beams + b;
  const float score = b < a.beams ? a.scores[row] : 0.f;
  const bool done = b < a.beams && a.finished && a.finished[row];
  if (threadIdx.x == 0) n_cand = 0;
  // (n_lists <= kMaxLists < kThreads)
  float2 mine_s = make_float2(-INFINITY, 0.f);
  if (b < n_lists) stats[b] = mine_s = a.stats[(size_t)seq * n_lists + b];
  __syncthreads();
  if (b < n_lists) {
    const int first = b / a.pieces * a.pieces;
    float M = -INFINITY;
    for (int p = first; p < first + a.pieces; ++p) M = fmaxf(M, stats[p].x);
    // the piece's sum relative to the row's maximum
    terms[b] = make_float2(M, mine_s.x == M || mine_s.x == -INFINITY ? mine_s.y
                                                                     : mine_s.y * ex2((mine_s.x - M) * kLog2e));
  }
  __syncthreads();
  if (b < a.beams) {
    over[b] = done;
    double to = NAN;
    if (score - score == 0.f) {                // finite
      if (done) {
        to = score;
      } else {
        double L = 0.0;
        for (int p = 0; p < a.pieces; ++p) L += terms[b * a.pieces + p].y;
        const double M = terms[b * a.pieces].x, rest = log(L);
        if (M - M == 0.0 && rest - rest == 0.0) to = (double)score - rest;
      }
    }
    base[b] = to;
  }
  __syncthreads();
  // pair i of the lists; a value that is not above -inf: none
  const float by_select = 1.f / a.select, by_pieces = 1.f / a.pieces;   // (i < 2^13: the quotients are exact)
  auto entry = [&](int i, u64 key) {
    const int list = (int)((i + 0.5f) * by_select), b = (int)((list + 0.5f) * by_pieces);
    if (over[b])
      return Pair{i == b * a.pieces * a.select ? base[b] : -INFINITY, (u64)b << 32 | (uint32_t)a.eos};
    const double less = (double)unordered((uint32_t)(key >> 32)) - (double)terms[b * a.pieces].x;
    return Pair{key ? base[b] + less : -INFINITY, (u64)b << 32 | (uint32_t)~(uint32_t)key};
  };
  float mine = -INFINITY;
  for (int i0 = threadIdx.x; i0 < n_all; i0 += kAhead * kThreads) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = i0 + k * kThreads;
      if (i >= n_all) break;
      const double x = entry(i, ahead[k]).value;
      const float r = x > -INFINITY ? __double2float_rn(x) : -INFINITY;   // (rounding keeps the order)
      vals[i] = r;
      mine = fmaxf(mine, r);
    }
    if (n_all <= kAhead * kThreads) break;     // (they stay where they are)
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = i0 + (k + kAhead) * kThreads;
      ahead[k] = i < n_all ? keys[i] : 0ull;
    }
  }
  // A threshold that at least num_select pairs reach, and hardly more: down from the largest in growing
  // steps, then halving the last one.  (Beams differ too much for what serves above.)
  const uint32_t most_here = __reduce_max_sync(kAll, ordered(mine));
  if (lane == 0) tops[warp] = most_here;
  __syncthreads();
  uint32_t most = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) most = max(most, tops[w]);
  int turn = 0;
  auto count = [&](float t) {                  // pairs that reach t
    if (n_all <= kThreads) return __syncthreads_count(mine >= t);
    int c = 0;
    for (int i = threadIdx.x; i < n_all; i += kThreads) c += vals[i] >= t;
    c = __reduce_add_sync(kAll, c);
    if (lane == 0) counts[turn][warp] = c;
    __syncthreads();
    c = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) c += counts[turn][w];
    turn ^= 1;
    return c;
  };
  float tau = unordered(most), above = tau, width = 1.f;
  int reach = 0;
  while (reach < a.select && tau > -3e38f) {
    above = tau;
    tau = unordered(most) - width;
    width *= 4.f;
    reach = count(tau);
  }
  if (reach < a.select) tau = -INFINITY;
  for (int i = 0; i < 16 && reach > 2 * a.select + 32; ++i) {
    const float mid = 0.5f * (tau + above);
    const int n = count(mid);
    if (n >= a.select) {
      tau = mid;
      reach = n;
    } else {
      above = mid;
    }
  }
  auto offer = [&](int i, u64 key) {
    const int at = atomicAdd(&n_cand, 1);
    if (at < kCand) cand[at] = entry(i, key);
  };
  if (n_all <= kAhead * kThreads) {
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = threadIdx.x + k * kThreads;
      if (i < n_all && vals[i] >= tau && vals[i] > -INFINITY) offer(i, ahead[k]);
    }
  } else {
    for (int i = threadIdx.x; i < n_all; i += kThreads)
      if (vals[i] >= tau && vals[i] > -INFINITY) offer(i, keys[i]);
  }
  __syncthreads();
  const int n = n_cand;
  float* out_score = a.out_score + (size_t)seq * a.select;
  int32_t* out_beam = a.out_beam + (size_t)seq * a.select;
  int32_t* out_token = a.out_token + (size_t)seq * a.select;
  auto put = [&](int k, const Pair& p) {       // (values are rounded once, here)
    out_score[k] = (float)p.value;
    out_beam[k] = (int32_t)(p.at >> 32);
    out_token[k] = (int32_t)p.at;
  };
  const Pair none{-INFINITY, ~0ull};
  if (n <= kCand) {
    for (int i = threadIdx.x; i < n; i += kThreads) {
      const Pair p = cand[i];
      int rank = 0;
      for (int j = 0; j < n; ++j) rank += before(cand[j], p);
      if (rank < a.select) put(rank, p);
    }
    if ((int)threadIdx.x >= n && (int)threadIdx.x < a.select) put(threadIdx.x, none);
    return;
  }
  // many equal values: one pair after the other, each the first behind the one before
  Pair last{INFINITY, 0};
  for (int k = 0; k < a.select; ++k) {
    Pair best = none;
    for (int i = threadIdx.x; i < n_all; i += kThreads) {
      if (!(vals[i] >= tau && vals[i] > -INFINITY)) continue;
      const Pair p = entry(i, keys[i]);
      if (before(last, p) && before(p, best)) best = p;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const Pair x{__shfl_xor_sync(kAll, best.value, o), __shfl_xor_sync(kAll, best.at, o)};
      if (before(x, best)) best = x;
    }
    if (lane == 0) picks[warp] = best;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWarps; ++w)
      if (before(picks[w], best)) best = picks[w];
    last = best;
    if (threadIdx.x == 0) put(k, best);
    __syncthreads();
  }
}

// Pieces of a row.  Few rows are cut to fill the machine twice over, no piece shorter than 2048 elements;
// more rows into pieces of no less than 8192 (f32) or 16384, as long as that gives no more than two rounds of
// CTAs: the end of a piece costs as much as some thousand elements (256 x 8 rows of 32003, f32, in 1, 2 and 4
// pieces: 50, 57 and 67 us).  Scan and pick, with pieces of half that size, of that and of twice as much: bf16, rows of
// 131072, 64 of them 18.4, 14.8 and 16.3 us, 128 26.5, 20.9 and 19.1, 256 34.0, 34.2 and 29.8; 600 rows of 32000 27.0,
// 22.3 and 20.0; f32, 128 rows of 131072 33.6, 33.1 and 27.6, 128 of 50000 22.5, 18.2 and 16.1.  With one round of
// CTAs, two and three: bf16, 128 rows of 131072 23.3, 20.9 and 20.7 us, 1200 of 32000 31.9, 35.8 and 35.9, 2048 of 32003
// 58.2, 58.0 and 63.4; f32, 128 of 131072 32.2, 33.1 and 36.5, 600 of 32000 32.3, 31.0 and 35.7.
int pieces_of(const apar_beam_config* c, int32_t n_seq) {
  const int64_t rows = (int64_t)n_seq * c->num_beams;
  const bool f32 = c->logits_type == APAR_LOGITS_F32;
  const int64_t held = f32 ? 8192 : 16384;
  const int64_t round = kSms * (f32 ? Packs<float>::kCtas : Packs<__half>::kCtas);
  const int64_t few = std::min<int64_t>((2 * kSms + rows - 1) / rows, (c->vocab + 2047) / 2048);
  const int64_t fit = std::min<int64_t>((2 * round + rows - 1) / rows, (c->vocab + held - 1) / held);
  return (int)std::min<int64_t>({std::max(few, fit), kMaxPieces, kMaxLists / c->num_beams});
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
  cudaError_t e;
  if (a.vocab <= kShort && lists > kShortRows) {   // (rows of one piece)
    auto rows = cfg->logits_type == APAR_LOGITS_F32   ? beam_rows_kernel<float>
                : cfg->logits_type == APAR_LOGITS_F16 ? beam_rows_kernel<__half>
                                                      : beam_rows_kernel<__nv_bfloat16>;
    e = launch_kernel(rows, dim3((lists + kWarps - 1) / kWarps), dim3(kThreads), 0, st, false, a);
  } else {
    e = launch_kernel(scan, dim3(lists), dim3(kThreads), 0, st, false, a);
  }
  if (e == cudaSuccess) e = launch_kernel(beam_pick_kernel, dim3(n_seq), dim3(kThreads), 0, st, true, a);
  if (e != cudaSuccess) {
    note_cuda_error(e);
    return APAR_ERR_CUDA;
  }
  return APAR_OK;
}
