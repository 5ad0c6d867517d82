// Accumulated attention weights of cached keys, and eviction by them.
//
// A float per (layer, block, kv head, row) lies beside the K and V pools, in the same order: how much
// weight the key has received so far, summed over queries and the heads of a group,
//     w[key] (+)= sum_{query, head} exp(scale <q, k> - lse[query, head]),
// where lse is the log of the softmax's denominator that the attention call has written.  So one pass
// over K is enough, V is not read, and no maximum or sum has to be found first.
#include <algorithm>

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "apar_internal.h"
#include "ptx.cuh"

namespace apar {
namespace {

constexpr unsigned kAll = 0xffffffffu;

// ------------------------------------------------------------------ rows that come and move
__global__ void __launch_bounds__(256) weights_clear_kernel(float* __restrict__ w, size_t layer_floats,
                                                            const int32_t* __restrict__ slots,
                                                            int n_rows, int num_kv_heads) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= (int64_t)n_rows * num_kv_heads) return;
  const int slot = slots[i / num_kv_heads], h = (int)(i % num_kv_heads);
  w[blockIdx.y * layer_floats + ((size_t)(slot >> 4) * num_kv_heads + h) * kBlock + (slot & 15)] = 0.f;
}

// A group is at most 64 rows whose sources and destinations may overlap: all are read, then written.
__global__ void __launch_bounds__(64) weights_move_kernel(float* __restrict__ w, size_t layer_floats,
                                                          const RowMove* __restrict__ moves,
                                                          const int32_t* __restrict__ group_begin,
                                                          int num_kv_heads) {
  const int m = group_begin[blockIdx.x] + threadIdx.x, h = blockIdx.y;
  float* p = w + blockIdx.z * layer_floats;
  const bool on = m < group_begin[blockIdx.x + 1];
  auto at = [&](int slot) {
    return ((size_t)(slot >> 4) * num_kv_heads + h) * kBlock + (slot & 15);
  };
  float v = 0.f;
  if (on) v = p[at(moves[m].src_slot)];
  __syncthreads();
  if (on) p[at(moves[m].dst_slot)] = v;
}

// ------------------------------------------------------------------ one query per thread
// A unit is a run of keys and the queries that see it; no key belongs to two units, so a unit adds
// to its keys' weights without atomics and in a fixed order.  One warp takes a unit and a kv head:
// sixteen keys at a time are the A operand of mma.m16n8k16, eight rows (query, head of the group) the
// B operand.  The contraction may take the dims in any order as long as both operands take the same:
// a lane loads sixteen consecutive bytes of its key's row, which hold its share of two products, so K
// comes straight from memory into registers.
// K is read once for up to 8 * NT rows, whose queries stay in registers; units of more than 32 go over their
// keys again, in the L2 cache.  Units of up to 8, 16 and more rows have a launch each (in one kernel
// the three share the widest one's registers; with one of 8 rows, K is read again for every 8: 64 prompts
// of 2400 keys and 3 forks each, 32 heads on 8, 117 us, now 68); a launch may start before the one before
// it is done.  kAhead blocks of keys are on their way while one is worked on: it takes some 48 KB an SM in
// flight to keep HBM busy.  (Of 32 rows with one block ahead and three CTAs, two and two, or 64 rows with one and
// two: 64 prompts of 1024 under 16 threads each 73, 77 and 72 us; 16 of 3000 under 8 34, 36 and 48.)
// Bound by HBM: those 64 x 2400 keys are 315 MB, 4.6 TB/s; 256 threads with 2400 keys of their own are 1.26 GB
// and take 215 us, 5.8 TB/s.
__device__ __forceinline__ uint4 ld_k(const uint4* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2,
                                         uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9},"
      " {%0,%1,%2,%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

constexpr int kKeyWarps = 4;                     // per CTA

// Rows r0 .. r0 + 8 NT - 1 of the unit against its keys [begin, end) of kv head h.
template <int NT, int kAhead>
__device__ __forceinline__ void key_rows(const KeyArgs& a, const KeyUnit& it, const KeyUser* users,
                                         const int32_t* table, int h, int end, int rows, int r0,
                                         bool replace) {
  const int lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int G = a.shape.group, HQ = a.shape.num_q_heads, HKV = a.shape.num_kv_heads;
  const int n_blk = (end - it.tok_begin + kBlock - 1) / kBlock;
  const int32_t* ids = table + it.tok_begin / kBlock;
  // block ids of 32 blocks at a time, lane b's being block b's
  int id = lane < n_blk ? ids[lane] : 0, id_next = 32 + lane < n_blk ? ids[32 + lane] : 0;
  const uint8_t* k_base = (const uint8_t*)a.k_pool + (size_t)h * kTileBytes + g * 256 + t * 16;
  uint4 k[kAhead][8];
  auto fetch = [&](uint4 (&dst)[8], int block) {
    const uint4* src = (const uint4*)(k_base + (size_t)block * HKV * kTileBytes);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      dst[w] = ld_k(src + 4 * w);
      dst[4 + w] = ld_k(src + 128 + 4 * w);
    }
  };
#pragma unroll
  for (int x = 0; x < kAhead; ++x)
    if (x < n_blk) fetch(k[x], __shfl_sync(kAll, id, x));
  // this lane's part of the rows: rows 8 i + g as operands, 8 i + 2 t and + 1 as results
  uint4 q[NT][4];
  float ref[NT][2];
  int see[NT][2];                                // keys before this one are seen
#pragma unroll
  for (int i = 0; i < NT; ++i) {
    const int r = r0 + 8 * i + g;
    if (r < rows) {
      const int query = users[it.user_begin + r / G].query;
      const uint4* src = (const uint4*)((const __nv_bfloat16*)a.q + ((size_t)query * HQ + h * G + r % G) * kDim);
#pragma unroll
      for (int w = 0; w < 4; ++w) q[i][w] = __ldg(src + 4 * w + t);
    } else {
#pragma unroll
      for (int w = 0; w < 4; ++w) q[i][w] = make_uint4(0u, 0u, 0u, 0u);
    }
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int rr = r0 + 8 * i + 2 * t + e;
      ref[i][e] = 0.f;
      see[i][e] = 0;
      if (rr < rows) {
        const KeyUser user = users[it.user_begin + rr / G];
        ref[i][e] = __ldg(a.lse + (size_t)user.query * HQ + h * G + rr % G) * 1.4426950408889634f;
        see[i][e] = min(user.lim, end);
      }
    }
  }
  for (int b0 = 0; b0 < n_blk; b0 += kAhead) {
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {           // (unrolled: each block in registers of its own)
      const int b = b0 + x;
      if (b >= n_blk) break;
      if (b > 0 && (b & 31) == 0) {
        id = id_next;
        id_next = b + 32 + lane < n_blk ? ids[b + 32 + lane] : 0;
      }
      const int block = __shfl_sync(kAll, id, b & 31);
      float d[NT][4];
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        d[i][0] = d[i][1] = d[i][2] = d[i][3] = 0.f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          mma16816(d[i], k[x][w].x, k[x][4 + w].x, k[x][w].y, k[x][4 + w].y, q[i][w].x, q[i][w].y);
          mma16816(d[i], k[x][w].z, k[x][4 + w].z, k[x][w].w, k[x][4 + w].w, q[i][w].z, q[i][w].w);
        }
      }
      const int nb = b + kAhead;
      if (nb < n_blk) {
        const int from = (nb & 31) < (b & 31) ? id_next : id;   // (already of the next 32?)
        fetch(k[x], __shfl_sync(kAll, from, nb & 31));
      }
      // keys tok + g (d[0], d[1]) and tok + g + 8 (d[2], d[3]); a key that a row does not see may
      // hold any bits
      const int tok = it.tok_begin + b * kBlock;
      float lo = 0.f, hi = 0.f;
#pragma unroll
      for (int i = 0; i < NT; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          if (tok + g < see[i][e]) lo += ex2(fmaf(d[i][e], a.scale_log2e, -ref[i][e]));
          if (tok + g + 8 < see[i][e]) hi += ex2(fmaf(d[i][2 + e], a.scale_log2e, -ref[i][e]));
        }
      lo += __shfl_xor_sync(kAll, lo, 1);
      hi += __shfl_xor_sync(kAll, hi, 1);
      lo += __shfl_xor_sync(kAll, lo, 2);
      hi += __shfl_xor_sync(kAll, hi, 2);
      if (t < 2) {
        const int row = g + 8 * t;
        float* w = a.weights + ((size_t)block * HKV + h) * kBlock + row;
        const float add = t ? hi : lo;
        if (tok + row < end) *w = replace ? add : *w + add;
      }
    }
  }
}

template <int NT, int kAhead, int kCtas>
__global__ void __launch_bounds__(kKeyWarps * 32, kCtas) key_weights_kernel(const KeyArgs a) {
  constexpr int kClass = NT == 1 ? 0 : NT == 2 ? 1 : 2;
  const int G = a.shape.group, HKV = a.shape.num_kv_heads;
  const int64_t stride = (int64_t)gridDim.x * kKeyWarps;
  pdl_launch_dependents();
  const KeyUnit* units = a.plan->units();
  const KeyUser* users = a.plan->users();
#pragma unroll
  for (int c = 2; c > kClass; --c) units += a.plan->n_units[c];
  const int64_t total = (int64_t)a.plan->n_units[kClass] * HKV;
  for (int64_t u = (int64_t)blockIdx.x * kKeyWarps + (threadIdx.x >> 5); u < total; u += stride) {
    const KeyUnit it = units[u / HKV];
    const int h = (int)(u % HKV);
    const int32_t* table = a.d_tables + (size_t)it.table_row * a.shape.table_stride;
    const int end = it.tok_end < 0 ? a.d_lens[it.table_row] : it.tok_end;
    const int rows = it.n_users * G;
    if (it.tok_begin >= end) continue;
    for (int r0 = 0; r0 < rows; r0 += 8 * NT)
      key_rows<NT, kAhead>(a, it, users, table, h, end, rows, r0, a.replace && r0 == 0);
  }
  pdl_wait();                                    // (done means that the launches before it are, too)
}

// ------------------------------------------------------------------ read back
// One warp per block: its weights are one contiguous piece of the pool, and so are its rows of the output.
__global__ void __launch_bounds__(256) weights_read_kernel(const float* __restrict__ w,
                                                           const int32_t* __restrict__ tables, int stride,
                                                           const __grid_constant__ RowRanges few,
                                                           const RowRange* __restrict__ many,
                                                           int num_kv_heads, float* __restrict__ out) {
  const RowRange r = many ? many[blockIdx.y] : few.r[blockIdx.y];
  const int lane = threadIdx.x & 31, last = (r.begin + r.count - 1) / kBlock;
  for (int b = r.begin / kBlock + blockIdx.x * 8 + (threadIdx.x >> 5); b <= last; b += gridDim.x * 8) {
    const float* src = w + (size_t)tables[(size_t)r.table_row * stride + b] * num_kv_heads * kBlock;
    const int p0 = max(r.begin, b * kBlock), p1 = min(r.begin + r.count, b * kBlock + kBlock);
    float* dst = out + (r.first + p0 - r.begin) * num_kv_heads;
    for (int i = lane; i < (p1 - p0) * num_kv_heads; i += 32)
      dst[i] = src[(i % num_kv_heads) * kBlock + (p0 & 15) + i / num_kv_heads];
  }
}

// ------------------------------------------------------------------ eviction: which rows
// A cluster of one to eight CTAs per (stretch, layer, kv head), each with a contiguous part of the rows,
// whose weights it reads once and keeps in registers as ordered integers.  The keep-th largest is
// found eleven bits at a time (three rounds): every CTA counts its part in shared memory and reads the
// others' counts there.  Rows above it are kept, and of the rows equal to it the first few.  Ranks (which
// of the equal rows, which of the rows that move, which of the places they move to) come from counts per
// warp and row of a thread, added up once over the CTA and once over the cluster.
// Bound by its steps one after the other, some 20 barriers: 32 x 8 stretches of 2048 rows (2 MB) take 13 us,
// 8 of 131072 rows (4 MB) 38; one CTA that reads the weights for every round took 605 for those.
__device__ __forceinline__ uint32_t weight_key(float x) {      // larger weight, larger key; a NaN on top
  const uint32_t b = __float_as_uint(x + 0.f);
  return x != x ? 0xffffffffu : b ^ (uint32_t)((int32_t)b >> 31 | 0x80000000);
}

// Threads of a CTA and rows a thread holds.  Eight warps where that is enough and there are more stretches
// than SMs, or little to do (every warp adds up counts of its own: 32 x 8 stretches of 2048 rows 13 us, with
// 32 warps 16; but 8 of them 10.5 and 7.6), else 32 warps.  More than 8192 rows are cut in two, four or eight
// while SMs are idle (8 stretches of 16384 rows 23.5 us in one CTA, 19.4 in two; of 8192 rows 13.9 and 15.3;
// 128 of 16384 rows 27 and 43), and more than a CTA's registers hold always.
constexpr int kPickFew = 256, kPickFewKeys = 8;
constexpr int kPickMany = 1024, kPickManyKeys = 16;
constexpr int kPickRows = kPickMany * kPickManyKeys;           // a CTA holds at most
constexpr int kPickCluster = 8;
constexpr int kBins = 2048;

template <int kThreads, int kKeys>
struct __align__(16) PickShared {
  static constexpr int kWarps = kThreads / 32;
  uint32_t hist[kBins];
  uint32_t warp_sum[32];
  uint32_t prefix, left;
  int before[3][kKeys * kWarps];           // rows of a kind before those of (key, warp), in the CTA
  int total[3];                            // in the CTA
};

// Sum of the values of the threads before this one; *all: of all threads.
template <int kThreads>
__device__ __forceinline__ uint32_t sum_before(uint32_t mine, uint32_t* warp_sum, uint32_t* all) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  uint32_t upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const uint32_t x = __shfl_up_sync(kAll, upto, o);
    if (lane >= o) upto += x;
  }
  if (lane == 31) warp_sum[warp] = upto;
  __syncthreads();
  const uint32_t w = lane < kThreads / 32 ? warp_sum[lane] : 0;
  *all = __reduce_add_sync(kAll, w);
  return __reduce_add_sync(kAll, lane < warp ? w : 0) + upto - mine;
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {               // (all CTAs of a cluster run at the same time)
  asm volatile("barrier.cluster.arrive.aligned;\nbarrier.cluster.wait.aligned;" ::: "memory");
}
// What lies at `p` in the shared memory of CTA `rank`.
__device__ __forceinline__ uint32_t ld_peer(const void* p, uint32_t rank) {
  uint32_t a, v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(s32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 ld_peer2(const void* p, uint32_t rank) {
  uint32_t a;
  uint2 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(s32(p)), "r"(rank));
  asm volatile("ld.shared::cluster.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}

// sh.before[kind][..] holds counts per (key, warp) and becomes how many rows of that kind come earlier
// in the stretch; returns the number of all of them.
template <int kThreads, int kKeys>
__device__ int ranks_of(PickShared<kThreads, kKeys>& sh, int kind, int used, uint32_t n_cta, uint32_t me) {
  constexpr int kWarps = kThreads / 32;
  static_assert(kKeys * kWarps <= kThreads, "a thread for each count");
  const int lane = threadIdx.x & 31;
  const bool on = (int)threadIdx.x < used * kWarps;
  uint32_t all;
  uint32_t base = sum_before<kThreads>(on ? sh.before[kind][threadIdx.x] : 0, sh.warp_sum, &all);
  if (n_cta > 1) {
    if (threadIdx.x == 0) sh.total[kind] = (int)all;
    cluster_sync();
    const uint32_t t = (uint32_t)lane < n_cta ? ld_peer(&sh.total[kind], lane) : 0;   // (a lane per CTA)
    base += __reduce_add_sync(kAll, (uint32_t)lane < me ? t : 0);
    all = __reduce_add_sync(kAll, t);
  }
  if (on) sh.before[kind][threadIdx.x] = (int)base;
  __syncthreads();
  return (int)all;
}

template <int kThreads, int kKeys>
__global__ void __launch_bounds__(kThreads, kThreads <= 256 ? 6 : 1)
evict_pick_kernel(const EvictArgs a, const __grid_constant__ EvictFew few, int n_cta) {
  constexpr int kWarps = kThreads / 32, kPerThread = kBins / kThreads;
  __shared__ PickShared<kThreads, kKeys> sh;
  pdl_launch_dependents();
  const uint32_t me = n_cta > 1 ? cluster_rank() : 0;
  const int entry = blockIdx.x / n_cta;
  const EvictEntry en = a.entries ? a.entries[entry] : few.entries[entry];
  const int heads = a.num_kv_heads, lh = blockIdx.y, l = lh / heads, h = lh % heads;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float* w = a.weights + (size_t)l * a.layer_floats;
  const int32_t* table = a.d_tables + (size_t)en.table_row * a.table_stride + en.begin / kBlock;
  int2* list = a.moves + en.list_begin + (size_t)lh * en.list_rows;
  // this CTA's rows, r0 .. r0 + n - 1; thread t holds rows t, t + kThreads, ... of them
  const int per = (en.n + n_cta * kThreads - 1) / (n_cta * kThreads) * kThreads;
  const int r0 = min(en.n, (int)me * per), n = min(en.n - r0, per);
  const int used = (n + kThreads - 1) / kThreads;
  uint32_t key[kKeys];
#pragma unroll
  for (int k = 0; k < kKeys; ++k) {
    key[k] = 0;
    const int i = r0 + k * kThreads + threadIdx.x;
    if (k < used && i < r0 + n)
      key[k] = weight_key(w[((size_t)table[i >> 4] * heads + h) * kBlock + (i & 15)]);
  }
  uint32_t prefix = 0, left = en.keep;           // the left-th largest of the keys that start with prefix
  for (int round = 0; round < 3; ++round) {
    const int shift = round == 0 ? 21 : round == 1 ? 10 : 0, bits = round == 2 ? 10 : 11;
    for (int i = threadIdx.x; i < kBins; i += kThreads) sh.hist[i] = 0;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kKeys; ++k) {
      if (k >= used) break;
      if (k * kThreads + (int)threadIdx.x < n && (round == 0 || key[k] >> (shift + bits) == prefix))
        atomicAdd(&sh.hist[key[k] >> shift & ((1u << bits) - 1)], 1u);
    }
    __syncthreads();
    if (n_cta > 1) cluster_sync();
    // a thread looks after a few neighbouring bins, the first one after the highest
    const int top = kBins - 1 - kPerThread * threadIdx.x;
    uint32_t c[kPerThread], sum = 0;               // c[0]: the highest
    if (n_cta == 1) {
#pragma unroll
      for (int j = 0; j < kPerThread; ++j) c[j] = sh.hist[top - j];
    } else {
      uint2 part[kPickCluster];
#pragma unroll
      for (int j = 0; j < kPerThread; j += 2) {
#pragma unroll
        for (int r = 0; r < kPickCluster; ++r)     // (all on their way at once)
          part[r] = r < n_cta ? ld_peer2(&sh.hist[top - j - 1], r) : make_uint2(0u, 0u);
        c[j] = c[j + 1] = 0;
#pragma unroll
        for (int r = 0; r < kPickCluster; ++r) {
          c[j] += part[r].y;
          c[j + 1] += part[r].x;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < kPerThread; ++j) sum += c[j];
    uint32_t all;
    uint32_t above = sum_before<kThreads>(sum, sh.warp_sum, &all);
    if (above < left && left <= above + sum) {
#pragma unroll
      for (int j = 0; j < kPerThread; ++j) {
        if (above < left && left <= above + c[j]) {
          sh.prefix = prefix << bits | (uint32_t)(top - j);
          sh.left = left - above;
        }
        above += c[j];
      }
    }
    __syncthreads();
    prefix = sh.prefix;
    left = sh.left;
    if (n_cta > 1) cluster_sync();               // (the counts have been read: they may be cleared)
  }
  // ---- which rows are kept, and where they go
#pragma unroll
  for (int k = 0; k < kKeys; ++k) {
    if (k >= used) break;
    const unsigned who = __ballot_sync(kAll, k * kThreads + (int)threadIdx.x < n && key[k] == prefix);
    if (lane == 0) sh.before[0][k * kWarps + warp] = __popc(who);
  }
  __syncthreads();
  ranks_of(sh, 0, used, n_cta, me);
  uint32_t kept = 0;                             // bit k: row k of this thread
#pragma unroll
  for (int k = 0; k < kKeys; ++k) {
    if (k >= used) break;
    const int at = k * kThreads + threadIdx.x, i = r0 + at;
    const bool equal = at < n && key[k] == prefix;
    const unsigned who = __ballot_sync(kAll, equal);
    const int rank = sh.before[0][k * kWarps + warp] + __popc(who & ((1u << lane) - 1));
    const bool keep = at < n && (key[k] > prefix || (equal && rank < (int)left));
    if (keep) kept |= 1u << k;
    const unsigned move = __ballot_sync(kAll, keep && i >= en.keep);
    const unsigned hole = __ballot_sync(kAll, at < n && !keep && i < en.keep);
    if (lane == 0) {
      sh.before[1][k * kWarps + warp] = __popc(move);
      sh.before[2][k * kWarps + warp] = __popc(hole);
    }
  }
  __syncthreads();
  const int n_move = ranks_of(sh, 1, used, n_cta, me);
  ranks_of(sh, 2, used, n_cta, me);
#pragma unroll
  for (int k = 0; k < kKeys; ++k) {
    if (k >= used) break;
    const int at = k * kThreads + threadIdx.x, i = r0 + at;
    const bool keep = kept >> k & 1, move = keep && i >= en.keep;
    const bool hole = at < n && !keep && i < en.keep;
    const unsigned wm = __ballot_sync(kAll, move), wh = __ballot_sync(kAll, hole);
    const unsigned lower = (1u << lane) - 1;
    const int holes = sh.before[2][k * kWarps + warp] + __popc(wh & lower);
    if (move) list[sh.before[1][k * kWarps + warp] + __popc(wm & lower)].x = i;
    if (hole) list[holes].y = i;
    // out of place the rows that stay are copied as well, behind those that move: the row's place
    // less the free places before it
    if (!en.in_place && keep && !move) list[n_move + i - holes] = make_int2(i, i);
  }
  if (threadIdx.x == 0 && me == 0)
    a.counts[(size_t)entry * gridDim.y + lh] = en.in_place ? n_move : en.keep;
  if (n_cta > 1) cluster_sync();                 // (nobody leaves while its counts are being read)
}

// The same for stretches that the registers of a cluster do not hold: one CTA, eight bits at a time,
// the weights read again for every round and for the ranks.
constexpr int kPickThreads = 512;
__global__ void __launch_bounds__(kPickThreads) evict_pick_long_kernel(const EvictArgs a,
                                                                       const __grid_constant__ EvictFew few) {
  __shared__ uint32_t hist[256];
  __shared__ uint32_t s_prefix, s_left;
  __shared__ int s_scan[3][kPickThreads / 32];
  pdl_launch_dependents();
  const EvictEntry en = a.entries ? a.entries[blockIdx.x] : few.entries[blockIdx.x];
  const int heads = a.num_kv_heads, lh = blockIdx.y, l = lh / heads, h = lh % heads;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const float* w = a.weights + (size_t)l * a.layer_floats;
  const int32_t* table = a.d_tables + (size_t)en.table_row * a.table_stride + en.begin / kBlock;
  int2* list = a.moves + en.list_begin + (size_t)lh * en.list_rows;
  auto key_at = [&](int i) {
    return weight_key(w[((size_t)table[i >> 4] * heads + h) * kBlock + (i & 15)]);
  };
  uint32_t prefix = 0, left = en.keep;           // the left-th largest key that starts with prefix
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = threadIdx.x; i < 256; i += kPickThreads) hist[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < en.n; i += kPickThreads) {
      const uint32_t k = key_at(i);
      if (shift == 24 || k >> (shift + 8) == prefix) atomicAdd(&hist[k >> shift & 255], 1u);
    }
    __syncthreads();
    if (warp == 0) {
      // lane i looks after bins 255 - 8 i downwards
      uint32_t sum = 0;
      for (int j = 0; j < 8; ++j) sum += hist[255 - 8 * lane - j];
      uint32_t upto = sum;
#pragma unroll
      for (int o = 1; o < 32; o *= 2) {
        const uint32_t x = __shfl_up_sync(kAll, upto, o);
        if (lane >= o) upto += x;
      }
      uint32_t above = upto - sum;
      if (above < left && left <= upto) {
        int bin = 255 - 8 * lane;
        while (above + hist[bin] < left) above += hist[bin--];
        s_prefix = prefix << 8 | bin;
        s_left = left - above;
      }
    }
    __syncthreads();
    prefix = s_prefix;
    left = s_left;
  }
  // rows above `prefix` are kept, and the first `left` rows equal to it
  int n_equal = 0, n_move = 0, n_hole = 0;
  for (int i0 = 0; i0 < en.n; i0 += kPickThreads) {
    const int i = i0 + threadIdx.x;
    const uint32_t k = i < en.n ? key_at(i) : 0;
    const bool equal = i < en.n && k == prefix;
    unsigned who = __ballot_sync(kAll, equal);
    if (lane == 0) s_scan[0][warp] = __popc(who);
    __syncthreads();
    int before = n_equal + __popc(who & ((1u << lane) - 1)), total = 0;
    for (int x = 0; x < kPickThreads / 32; ++x) {
      if (x < warp) before += s_scan[0][x];
      total += s_scan[0][x];
    }
    n_equal += total;
    const bool kept = i < en.n && (k > prefix || (equal && before < (int)left));
    const bool move = kept && i >= en.keep, hole = !kept && i < en.keep;
    const unsigned wm = __ballot_sync(kAll, move), wh = __ballot_sync(kAll, hole);
    if (lane == 0) {
      s_scan[1][warp] = __popc(wm);
      s_scan[2][warp] = __popc(wh);
    }
    __syncthreads();
    int m = n_move + __popc(wm & ((1u << lane) - 1)), o = n_hole + __popc(wh & ((1u << lane) - 1));
    for (int x = 0; x < kPickThreads / 32; ++x) {
      if (x < warp) {
        m += s_scan[1][x];
        o += s_scan[2][x];
      }
      n_move += s_scan[1][x];
      n_hole += s_scan[2][x];
    }
    if (move) list[m].x = i;
    if (hole) list[o].y = i;
    __syncthreads();
  }
  // out of place the rows that stay are copied as well, behind those that move
  if (!en.in_place) {
    int n_stay = n_move;
    n_equal = 0;
    for (int i0 = 0; i0 < en.keep; i0 += kPickThreads) {
      const int i = i0 + threadIdx.x;
      const uint32_t k = i < en.n ? key_at(i) : 0;
      const bool equal = i < en.n && k == prefix;
      const unsigned who = __ballot_sync(kAll, equal);
      if (lane == 0) s_scan[0][warp] = __popc(who);
      __syncthreads();
      int before = n_equal + __popc(who & ((1u << lane) - 1));
      for (int x = 0; x < kPickThreads / 32; ++x) {
        if (x < warp) before += s_scan[0][x];
        n_equal += s_scan[0][x];
      }
      const bool stay = i < en.keep && i < en.n && (k > prefix || (equal && before < (int)left));
      const unsigned ws = __ballot_sync(kAll, stay);
      if (lane == 0) s_scan[1][warp] = __popc(ws);
      __syncthreads();
      int m = n_stay + __popc(ws & ((1u << lane) - 1));
      for (int x = 0; x < kPickThreads / 32; ++x) {
        if (x < warp) m += s_scan[1][x];
        n_stay += s_scan[1][x];
      }
      if (stay) list[m] = make_int2(i, i);
      __syncthreads();
    }
    n_move = n_stay;
  }
  if (threadIdx.x == 0) a.counts[(size_t)blockIdx.x * gridDim.y + lh] = n_move;
}

// ------------------------------------------------------------------ eviction: the rows move
// Half a warp per row, four rows at a time: 256 bytes of K, 256 of V, and the weight.  Sources lie behind
// `keep` and destinations before it, or in other blocks: no move reads what another writes.
// Bound by HBM: 32 x 900 rows of 16 (layer, head) pairs, 472 MB read and written, 81 us, 5.8 TB/s.
constexpr int kMoveRows = 4;
__global__ void __launch_bounds__(256) evict_move_kernel(const EvictArgs a, const __grid_constant__ EvictFew few) {
  const EvictEntry en = a.entries ? a.entries[blockIdx.z] : few.entries[blockIdx.z];
  const int heads = a.num_kv_heads, lh = blockIdx.y, l = lh / heads, h = lh % heads;
  const int2* list = a.moves + en.list_begin + (size_t)lh * en.list_rows;
  const int32_t* from = a.d_tables + (size_t)en.table_row * a.table_stride + en.begin / kBlock;
  const int32_t* to = en.in_place ? from : (a.entries ? a.dst_blocks : few.dst_blocks) + en.dst_begin;
  uint4* k = (uint4*)((char*)a.k_pool + (size_t)l * a.layer_bytes);
  uint4* v = (uint4*)((char*)a.v_pool + (size_t)l * a.layer_bytes);
  float* w = a.weights + (size_t)l * a.layer_floats;
  pdl_wait();                                  // (the list is written)
  const int n = a.counts[(size_t)blockIdx.z * gridDim.y + lh], c = threadIdx.x & 15;
  for (int m0 = blockIdx.x * 16 * kMoveRows + (threadIdx.x >> 4); m0 < n; m0 += gridDim.x * 16 * kMoveRows) {
    size_t src[kMoveRows], dst[kMoveRows];
    uint4 x[kMoveRows], y[kMoveRows];
    float z[kMoveRows];
#pragma unroll
    for (int r = 0; r < kMoveRows; ++r) {
      const int2 mv = list[min(m0 + 16 * r, n - 1)];
      src[r] = ((size_t)from[mv.x >> 4] * heads + h) * kBlock + (mv.x & 15);
      dst[r] = ((size_t)to[mv.y >> 4] * heads + h) * kBlock + (mv.y & 15);
    }
#pragma unroll
    for (int r = 0; r < kMoveRows; ++r) {
      x[r] = k[src[r] * 16 + c];
      y[r] = v[src[r] * 16 + c];
      if (c == 0) z[r] = w[src[r]];
    }
#pragma unroll
    for (int r = 0; r < kMoveRows; ++r) {
      if (m0 + 16 * r >= n) break;
      k[dst[r] * 16 + c] = x[r];
      v[dst[r] * 16 + c] = y[r];
      if (c == 0) w[dst[r]] = z[r];
    }
  }
}

}  // namespace

cudaError_t launch_weights_clear(float* w, size_t layer_floats, int num_layers, const int32_t* d_slots,
                                 int n_rows, int num_kv_heads, cudaStream_t st) {
  if (n_rows <= 0) return cudaSuccess;
  const unsigned grid = (unsigned)(((int64_t)n_rows * num_kv_heads + 255) / 256);
  return launch_kernel(weights_clear_kernel, dim3(grid, num_layers), dim3(256), 0, st, false, w,
                       layer_floats, d_slots, n_rows, num_kv_heads);
}

cudaError_t launch_weights_move(float* w, size_t layer_floats, int num_layers, const RowMove* d_moves,
                                const int32_t* d_group_begin, int n_groups, int num_kv_heads,
                                cudaStream_t st) {
  if (n_groups <= 0) return cudaSuccess;
  return launch_kernel(weights_move_kernel, dim3(n_groups, num_kv_heads, num_layers), dim3(64), 0, st,
                       false, w, layer_floats, d_moves, d_group_begin, num_kv_heads);
}

cudaError_t launch_key_weights(const KeyArgs& a, const int32_t (&n_units)[3], bool all, cudaStream_t st) {
  cudaError_t e = cudaSuccess;
  bool first = true;
  auto launch = [&](auto kernel, int n, int ctas) {
    if ((n <= 0 && !all) || e != cudaSuccess) return;
    const int64_t ctas_full = (int64_t)ctas * a.num_sms, warps = (int64_t)n * a.shape.num_kv_heads;
    const int grid = (int)(all ? ctas_full : std::min<int64_t>((warps + kKeyWarps - 1) / kKeyWarps, ctas_full));
    e = launch_kernel(kernel, dim3(grid), dim3(kKeyWarps * 32), 0, st, !first, a);
    first = false;
  };
  launch(key_weights_kernel<4, 1, 3>, n_units[2], 3);
  launch(key_weights_kernel<2, 2, 3>, n_units[1], 3);
  launch(key_weights_kernel<1, 2, 4>, n_units[0], 4);
  return e;
}

cudaError_t launch_weights_read(const float* w, const int32_t* d_tables, int table_stride,
                                const RowRanges& few, const RowRange* many, int n, int max_count,
                                int num_kv_heads, float* out, cudaStream_t st) {
  if (n <= 0 || max_count <= 0) return cudaSuccess;
  const unsigned grid = (unsigned)std::min(max_count / (kBlock * 8) + 1, 1024);
  for (int i = 0; i < n; i += 65535) {                 // (the grid's limit)
    const cudaError_t e = launch_kernel(weights_read_kernel, dim3(grid, std::min(n - i, 65535)), dim3(256),
                                        0, st, false, w, d_tables, table_stride, few,
                                        many ? many + i : nullptr, num_kv_heads, out);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

cudaError_t launch_evict(const EvictArgs& a, const EvictFew& few, int n, int num_layers, int max_len,
                         int max_rows, int num_sms, cudaStream_t st) {
  if (n <= 0) return cudaSuccess;
  const int lh = num_layers * a.num_kv_heads;
  cudaError_t e;
  const int64_t stretches = (int64_t)n * lh;
  if (max_len <= kPickFew * (stretches > num_sms ? kPickFewKeys : 2)) {
    e = launch_kernel(evict_pick_kernel<kPickFew, kPickFewKeys>, dim3(n, lh), dim3(kPickFew), 0, st, false, a,
                      few, 1);
  } else if (max_len <= kPickCluster * kPickRows) {
    int n_cta = 1;                               // of a stretch
    while (n_cta < kPickCluster &&
           (max_len > n_cta * kPickRows || (max_len > n_cta * 8192 && 2 * n_cta * stretches <= num_sms)))
      n_cta *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(n * n_cta, lh);
    cfg.blockDim = dim3(kPickMany);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = n_cta;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = n_cta > 1 ? 1 : 0;
    e = cudaLaunchKernelEx(&cfg, evict_pick_kernel<kPickMany, kPickManyKeys>, a, few, n_cta);
  } else {
    e = launch_kernel(evict_pick_long_kernel, dim3(n, lh), dim3(kPickThreads), 0, st, false, a, few);
  }
  if (e != cudaSuccess || max_rows <= 0) return e;
  const unsigned grid = (unsigned)std::min((max_rows + 16 * kMoveRows - 1) / (16 * kMoveRows), 1024);
  EvictArgs part = a;
  for (int i = 0; i < n && e == cudaSuccess; i += 65535) {   // (the grid's limit)
    if (a.entries) part.entries = a.entries + i;
    part.counts = a.counts + (size_t)i * lh;
    e = launch_kernel(evict_move_kernel, dim3(grid, lh, std::min(n - i, 65535)), dim3(256), 0, st, i == 0,
                      part, few);
  }
  return e;
}

}  // namespace apar
