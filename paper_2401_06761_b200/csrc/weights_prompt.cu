// Accumulated weights of keys (see weights.cu) for runs of consecutive queries, each of which sees the
// keys up to its own position: whole prompts, or a window of queries behind a long context.
//
// A unit is up to 256 keys of one kv head; the products are S^T = K Q^T, keys in the rows.  So a thread
// owns a key (its TMEM lane), goes over the queries in the columns and adds up
//     exp2(c s - log2 e * lse[column])
// in a register: no shuffles, no atomics, nothing but one number per key leaves the SM.
//   warps 0-3, 4-7  own keys 0..127 and 128..255 of the unit, each with two S buffers of 128 columns.
//   warp 8          reads the unit list, copies K tiles (double-buffered, 64 KiB a unit) and query
//                   tiles (128 / group tokens times the group's heads; three in flight) by TMA, and puts
//                   each query tile's log-sum-exps and a description beside it.
//   warp 9          issues the products (lane 0): per query tile and half of the keys M 128, N 128, K 128.
// 256 keys to a unit, so that a query tile is read from L2 once for twice the keys.  Units are dealt out
// longest first, forwards and backwards in turn.  All waits are bounded, as in the attention kernels.
#include <algorithm>

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include "apar_internal.h"
#include "ptx.cuh"
#include "tcgen05.cuh"

namespace apar {
namespace {

constexpr int kKeys = 128;                       // of a half
constexpr int kHalf = kKeys * 128;               // bytes of 64 dims of 128 rows
constexpr int kTileB = 2 * kHalf;                // 32 KiB: 128 rows of K, or of queries
constexpr int kUnitB = 2 * kTileB;
constexpr int kQStages = 3;
constexpr int kOffQ = 2 * kUnitB;
constexpr int kOffLse = kOffQ + kQStages * kTileB;
constexpr int kOffDesc = kOffLse + kQStages * kKeys * 4;
constexpr int kOffBar = kOffDesc + kQStages * 32;
constexpr int kSmem = kOffBar + 256 + 1024;
static_assert(kSmem <= 227 * 1024, "shared memory");

struct TileDesc {
  int32_t n_tok;                 // queries' tokens of the tile; 0: no more tiles
  int32_t pos;                   // position of the first
  int32_t tok_begin, end;        // the unit's keys
  int32_t table_row, kvh;
  int32_t flags;                 // 1: the unit's first tile, 2: its last
  int32_t pad;
};
static_assert(sizeof(TileDesc) == 32, "description");

enum { B_KFULL = 0, B_KEMPTY = 2, B_QFULL = 4, B_QEMPTY = B_QFULL + kQStages,
       B_SFULL = B_QEMPTY + kQStages,            // [half][buffer]
       B_SEMPTY = B_SFULL + 4, B_TOTAL = B_SEMPTY + 4 };
static_assert(8 * B_TOTAL + 16 <= 256, "barrier area");

// Units in the order they are dealt out: CTA b's i-th.
__device__ __forceinline__ int64_t dealt(int64_t i) {
  return i * gridDim.x + (i & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
}

__global__ void __launch_bounds__(320, 1)
prompt_weights_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_q,
                      const KeyArgs a, int n_units) {
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (s32(smem_raw) + 1023u) & ~1023u;
  uint8_t* bp = smem_raw + (base - s32(smem_raw));
  auto bar = [&](int i) { return base + kOffBar + 8u * i; };
  volatile int* cta_abort = (volatile int*)(bp + kOffBar + 8 * B_TOTAL);
  volatile uint32_t* tmem_slot = (volatile uint32_t*)(bp + kOffBar + 8 * B_TOTAL + 8);
  TileDesc* descs = (TileDesc*)(bp + kOffDesc);
  float* lses = (float*)(bp + kOffLse);
  const int G = a.shape.group, HQ = a.shape.num_q_heads, HKV = a.shape.num_kv_heads;
  const int T = kKeys / G;                       // tokens of a query tile
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr unsigned kAll = 0xffffffffu;

  if (threadIdx.x == 0) {
    *cta_abort = *(volatile int*)a.d_error;      // an earlier kernel gave up: do not pile up
    asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)&tm_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)&tm_q) : "memory");
    for (int b = 0; b < 2; ++b) {
      bar_init(bar(B_KFULL + b), 1);
      bar_init(bar(B_KEMPTY + b), 1);
    }
    for (int s = 0; s < kQStages; ++s) {
      bar_init(bar(B_QFULL + s), 1);
      bar_init(bar(B_QEMPTY + s), 9);            // the products' end, and eight warps
    }
    for (int s = 0; s < 4; ++s) {
      bar_init(bar(B_SFULL + s), 1);
      bar_init(bar(B_SEMPTY + s), 4);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // rows of a query tile that the copies do not reach (where the group does not divide 128) are zero
  for (int i = threadIdx.x; i < kQStages * kTileB / 16; i += blockDim.x)
    *(uint4*)(bp + kOffQ + 16 * i) = make_uint4(0u, 0u, 0u, 0u);
  fence_async_smem();
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(s32((const void*)tmem_slot)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;              // columns of (half w, buffer b): 256 w + 128 b
  const bool dead = *cta_abort != 0;
  const int64_t total = (int64_t)n_units * HKV;

  if (dead) {
  } else if (warp == 8) {
    // ---------------------------------------------------------------- copies
    int off[4];                                  // this lane's rows of a tile, in the lse array
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = lane + 32 * i;
      off[i] = r < T * G ? r / G * HQ + r % G : -1;
    }
    int g = 0, ku = 0;                           // query tiles and units so far
    bool ok = true;
    for (int64_t i = 0; ok && i * gridDim.x < total; ++i) {
      const int64_t u = dealt(i);
      if (u >= total) continue;
      const KeyUnit it = a.units[u / HKV];
      const int h = (int)(u % HKV), n_blk = (it.tok_end - it.tok_begin + kBlock - 1) / kBlock;
      const int32_t* table = a.d_tables + (size_t)it.table_row * a.shape.table_stride + it.tok_begin / kBlock;
      const int bid = (lane >> 1) < n_blk ? table[lane >> 1] : 0;
      bool first = true;
      for (int x = 0; ok && x < it.n_users; ++x) {
        const KeyUser user = a.users[it.user_begin + x];
        for (int j = max(0, it.tok_begin - user.lim); j < user.count; j += T, ++g) {
          const int st = g % kQStages, n_tok = min(T, user.count - j), q0 = user.query + j;
          float l[4];                            // (on its way while the stage is waited for)
#pragma unroll
          for (int k = 0; k < 4; ++k)
            l[k] = off[k] >= 0 && lane + 32 * k < n_tok * G ? __ldg(a.lse + (int64_t)q0 * HQ + h * G + off[k])
                                                            : INFINITY;
          if (g >= kQStages)
            ok = bar_wait(bar(B_QEMPTY + st), (g / kQStages - 1) & 1, cta_abort, a.d_error, 22000);
          if (first && ku >= 2)
            ok = ok && bar_wait(bar(B_KEMPTY + (ku & 1)), ((ku >> 1) - 1) & 1, cta_abort, a.d_error, 22100);
          ok = __all_sync(kAll, ok);
          if (!ok) break;
          if (first) {
            if (lane == 0) bar_expect_tx(bar(B_KFULL + (ku & 1)), (uint32_t)n_blk * kTileBytes);
            __syncwarp();
            // block b of the unit: 16 rows of its half of the keys, in two pieces of 64 dims
            const uint32_t dst = base + (ku & 1) * kUnitB + (lane & 1) * kHalf;
            const int b = lane >> 1;
            if (b < n_blk)
              tma_2d(dst + (b >> 3) * kTileB + (b & 7) * (kBlock * 128), &tm_k, (lane & 1) * 64,
                     (bid * HKV + h) * kBlock, bar(B_KFULL + (ku & 1)));
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) lses[st * kKeys + lane + 32 * k] = l[k] * 1.4426950408889634f;
          if (lane == 0) {
            const bool last = x == it.n_users - 1 && j + T >= user.count;
            descs[st] = TileDesc{n_tok, user.lim + j, it.tok_begin, it.tok_end, it.table_row, h,
                                 (first ? 1 : 0) | (last ? 2 : 0), 0};
          }
          __syncwarp();
          if (lane == 0) bar_expect_tx(bar(B_QFULL + st), 2u * T * G * 128u);
          __syncwarp();
          if (lane < 2)
            tma_3d(base + kOffQ + st * kTileB + lane * kHalf, &tm_q, lane * 64, h * G, q0, bar(B_QFULL + st));
          first = false;
        }
      }
      if (!first) ++ku;
    }
    if (ok && g >= kQStages)
      ok = __all_sync(kAll, bar_wait(bar(B_QEMPTY + g % kQStages), (g / kQStages - 1) & 1, cta_abort,
                                     a.d_error, 22200));
    if (ok && lane == 0) {
      descs[g % kQStages].n_tok = 0;
      bar_arrive(bar(B_QFULL + g % kQStages));
    }
    // after a wait that gave up: the copies in flight are waited for (with a limit of their own)
    if (*cta_abort && lane == 0) {
      for (int x = max(0, g - kQStages); x < g; ++x)
        for (uint32_t i = 0; i < kSpin && !bar_try(bar(B_QFULL + x % kQStages), (x / kQStages) & 1); ++i) {}
      for (int x = max(0, ku - 1); x <= ku; ++x)
        for (uint32_t i = 0; i < kSpin && !bar_try(bar(B_KFULL + (x & 1)), (x >> 1) & 1); ++i) {}
    }
  } else if (warp == 9) {
    // ---------------------------------------------------------------- products
    constexpr uint32_t kIdesc = instr_desc(128, false, 128);
    int ku = 0, cnt[2] = {0, 0};
    for (int g = 0;; ++g) {
      const int st = g % kQStages;
      if (!__all_sync(kAll, bar_wait(bar(B_QFULL + st), (g / kQStages) & 1, cta_abort, a.d_error, 23000)))
        break;
      const TileDesc d = descs[st];
      if (d.n_tok == 0) break;
      bool ok = true;
      if (d.flags & 1)
        ok = bar_wait(bar(B_KFULL + (ku & 1)), (ku >> 1) & 1, cta_abort, a.d_error, 23100);
      const int halves = d.end - d.tok_begin > kKeys ? 2 : 1;
      for (int w = 0; w < halves && ok; ++w) {
        const int sb = cnt[w] & 1;
        if (cnt[w] >= 2)
          ok = bar_wait(bar(B_SEMPTY + 2 * w + sb), ((cnt[w] >> 1) - 1) & 1, cta_abort, a.d_error, 23200);
        ok = __all_sync(kAll, ok);
        if (!ok) break;
        tc_fence_after();
        if (lane == 0) {
          const uint64_t kd = smem_desc(base + (ku & 1) * kUnitB + w * kTileB, 16, 1024);
          const uint64_t qd = smem_desc(base + kOffQ + st * kTileB, 16, 1024);
#pragma unroll
          for (int ks = 0; ks < 8; ++ks) {
            const uint64_t at = (uint64_t)(((ks >> 2) * kHalf + (ks & 3) * 32) >> 4);
            umma_bf16(tmem + 256u * w + 128u * sb, kd + at, qd + at, kIdesc, ks > 0);
          }
          umma_commit(bar(B_SFULL + 2 * w + sb));
        }
        ++cnt[w];
      }
      if (!__all_sync(kAll, ok)) break;
      if (lane == 0) {
        umma_commit(bar(B_QEMPTY + st));
        if (d.flags & 2) umma_commit(bar(B_KEMPTY + (ku & 1)));
      }
      if (d.flags & 2) ++ku;
      __syncwarp();
    }
  } else {
    // ---------------------------------------------------------------- sums
    const int w = warp >> 2, row = (warp & 3) * 32 + lane;     // the key's row of its half: its TMEM lane
    const uint32_t lane_sel = (uint32_t)((warp & 3) * 32) << 16;
    const float c = a.scale_log2e;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    int cnt = 0;
    for (int g = 0;; ++g) {
      const int st = g % kQStages;
      if (!__all_sync(kAll, bar_wait(bar(B_QFULL + st), (g / kQStages) & 1, cta_abort, a.d_error, 24000)))
        break;
      const TileDesc d = descs[st];
      if (d.n_tok == 0) break;
      const int key = d.tok_begin + kKeys * w + row;
      if (d.tok_begin + kKeys * w < d.end) {     // (the unit reaches into this half)
        const int sb = cnt & 1;
        if (!__all_sync(kAll, bar_wait(bar(B_SFULL + 2 * w + sb), (cnt >> 1) & 1, cta_abort, a.d_error,
                                       24100)))
          break;
        ++cnt;
        tc_fence_after();
        const uint32_t ts = (tmem + 256u * w + 128u * sb) | lane_sel;
        const float* lse = lses + st * kKeys;
        // the key is seen by columns lo .. hi - 1: by the tokens from its own position on
        const int lo = max(0, key - d.pos) * G, hi = d.n_tok * G;
        const bool all = __all_sync(kAll, lo == 0 && d.n_tok == T);
        for (int q4 = 0; q4 < 4; ++q4) {
          uint32_t s[32];
          TMEM_LD_32(ts + 32u * q4, s, 0);
          tmem_wait_ld();
          if (q4 == 3) {                         // all of it is in registers
            tc_fence_before();
            __syncwarp();
            if (lane == 0) bar_arrive(bar(B_SEMPTY + 2 * w + sb));
          }
          if (all) {
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
              const float4 l = *(const float4*)(lse + 32 * q4 + j);
              acc[0] += ex2(fmaf(__uint_as_float(s[j]), c, -l.x));
              acc[1] += ex2(fmaf(__uint_as_float(s[j + 1]), c, -l.y));
              acc[2] += ex2(fmaf(__uint_as_float(s[j + 2]), c, -l.z));
              acc[3] += ex2(fmaf(__uint_as_float(s[j + 3]), c, -l.w));
            }
          } else {
#pragma unroll
            for (int j = 0; j < 32; ++j) {
              const int col = 32 * q4 + j;
              const float p = ex2(fmaf(__uint_as_float(s[j]), c, -lse[col]));
              if (col >= lo && col < hi) acc[j & 3] += p;
            }
          }
        }
      }
      __syncwarp();
      if (lane == 0) bar_arrive(bar(B_QEMPTY + st));
      if (d.flags & 2) {
        if (key < d.end) {
          const int block = a.d_tables[(size_t)d.table_row * a.shape.table_stride + (key >> 4)];
          float* out = a.weights + ((size_t)block * HKV + d.kvh) * kBlock + (key & 15);
          const float sum = (acc[0] + acc[1]) + (acc[2] + acc[3]);
          *out = a.replace ? sum : *out + sum;
        }
        acc[0] = acc[1] = acc[2] = acc[3] = 0.f;
      }
    }
  }
  // ---- common exit: every role arrives here, then the allocating warp frees TMEM
  tc_fence_before();
  __syncthreads();
  if (warp == 9) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

}  // namespace

cudaError_t launch_prompt_weights(const KeyArgs& a, const CUtensorMap* tm_k, const CUtensorMap* tm_q,
                                  int n_units, cudaStream_t st) {
  if (n_units <= 0) return cudaSuccess;
  const cudaError_t e = cudaFuncSetAttribute(prompt_weights_kernel,
                                             cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  if (e != cudaSuccess) return e;
  const int grid = (int)std::min<int64_t>((int64_t)n_units * a.shape.num_kv_heads, a.num_sms);
  return launch_kernel(prompt_weights_kernel, dim3(grid), dim3(320), kSmem, st, false, *tm_k, *tm_q, a, n_units);
}

}  // namespace apar
