// Accumulated weights of keys (see weights.cu) for runs of consecutive queries, each of which sees the
// keys up to its own position: whole prompts, or a window of queries behind a long context.
//
// A unit is up to 256 keys of one kv head; the products are S^T = K Q^T, keys in the rows.  So a thread
// owns a key (its TMEM lane), goes over the queries in the columns and adds up
//     exp2(c s - log2 e * lse[column])
// in a register: no shuffles, no atomics, nothing but one number per key leaves the SM.
//   warps 0-15      eight to a half of the unit's keys, which has two S buffers of 128 columns: four take the
//                   even query tiles and four the odd ones, all columns of a tile.  So the barriers and the
//                   first scores' way from TMEM (1400 cycles a tile) pass while the other four have the
//                   special-function unit (1000 cycles a tile and half).  At a unit's end those that
//                   had its first tile write their sums and the others add theirs.
//   warp 16         copies, by TMA, K tiles (double-buffered, 64 KiB a unit) and query tiles (128 / group
//                   tokens times the group's heads; three in flight).
//   warp 17         puts each query tile's log-sum-exps and a description into a ring of five.
//   warps 18, 19    issue the products (lane 0), one for each half of the keys: M 128, N 128, K 128 per query
//                   tile.
// Each of these four does one small thing per tile: next to warps that keep the SM busy a single warp gets an
// instruction in every ten cycles or so and a look at a barrier takes it 250, and a tile's sums take 2000.
// (One warp that copied and described, and one that issued both products, took 3200 a tile.)
// 256 keys to a unit, so that a query tile is read from L2 once for twice the keys.  Units are dealt out
// longest first, forwards and backwards in turn.  All waits are bounded, as in the attention kernels.
// Bound by the special-function unit, one exponential a score: 8 prompts of 2048 tokens, 32 heads, 150 us, two
// thirds of its rate (86 us for the exponentials alone, 60 for the products); windows of 32 queries behind long
// prompts 86 us, 240 MB.  (Some of the exponentials as polynomials on the multipliers took longer: 4 of 16 156
// us, 7 of 16 167, as did scores asked for a tile ahead, 185.)
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
constexpr int kLStages = 5;
constexpr int kOffDesc = kOffLse + kLStages * kKeys * 4;
constexpr int kOffFlags = kOffDesc + kLStages * 32;
constexpr int kOffBar = kOffFlags + 16;
constexpr int kSmem = kOffBar + 320;
constexpr int kSumWarps = 16;
constexpr int kWarps = kSumWarps + 4;
static_assert(kSmem <= 227 * 1024, "shared memory");

struct TileDesc {
  int32_t n_tok;                 // queries' tokens of the tile; 0: no more tiles
  int32_t pos;                   // position of the first
  int32_t tok_begin, end;        // the unit's keys
  int32_t table_row, kvh;
  int32_t t, n_tiles;            // tile of the unit, and how many it has
};
static_assert(sizeof(TileDesc) == 32, "description");
// What the issuers need of it: a word beside each stage of the ring of query tiles.
enum { F_FIRST = 1, F_LAST = 2,  // tile of the unit
       F_BOTH = 4,               // the unit reaches into both halves of the keys
       F_END = 8 };

enum { B_KFULL = 0, B_KEMPTY = 2, B_QFULL = 4, B_QEMPTY = B_QFULL + kQStages,
       B_LFULL = B_QEMPTY + kQStages, B_LEMPTY = B_LFULL + kLStages,   // log-sum-exps and description
       B_SFULL = B_LEMPTY + kLStages,            // [half][buffer]
       B_SEMPTY = B_SFULL + 4,
       B_WFULL = B_SEMPTY + 4, B_WEMPTY = B_WFULL + 4,   // [half][turn of the first tile's warps]: they have
       B_TOTAL = B_WEMPTY + 4 };                         // written; the others have seen that
static_assert(8 * B_TOTAL + 16 <= 320, "barrier area");

// ---- two numbers at a time
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float lo, float hi) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpair(f32x2 v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// Waits for the loads from TMEM into r.  Naming the registers keeps what is done with them behind the wait:
// to the compiler they have their values from the load on.
__device__ __forceinline__ void wait_scores(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]),
                 "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]),
                 "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]),
                 "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]),
                 "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]),
                 "+r"(r[31])
               :: "memory");
}

// Of `issued` copies through a ring of so many stages, the oldest that may still be in flight: a stage is only
// filled again once its copy has been consumed.
__host__ __device__ constexpr int oldest_in_flight(int issued, int stages) {
  return issued > stages ? issued - stages : 0;
}
// Checked when this is compiled: whichever of those copies have not landed yet, waits for the parities of copies
// oldest_in_flight .. issued - 1, in order, wait for each of them, and none waits for a copy nobody asked for.
constexpr bool drain_waits_for_all(int stages) {
  for (int issued = 0; issued < 4 * stages; ++issued)
    for (unsigned missing = 0; missing < 1u << stages; ++missing) {   // bit of a stage: its last copy is on its way
      unsigned left = missing;
      for (int x = oldest_in_flight(issued, stages); x < issued; ++x) {
        const int s = x % stages, filled = (issued - 1 - s) / stages + 1;
        const int phase = filled - (left >> s & 1);                   // phases that the barrier has completed
        const bool through = phase > 0 ? (phase - 1) % 2 == x / stages % 2 : x / stages % 2 == 1;
        if (!through && !(left >> s & 1)) return false;               // (would run into its limit)
        if (!through) left &= ~(1u << s);
      }
      if (left & ((1u << (issued < stages ? issued : stages)) - 1)) return false;
    }
  return true;
}
static_assert(drain_waits_for_all(2) && drain_waits_for_all(kQStages), "copies in flight at a give-up");

// Units in the order they are dealt out: CTA b's i-th.
__device__ __forceinline__ int64_t dealt(int64_t i) {
  return i * gridDim.x + (i & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x);
}

// The units of a CTA in their order.  Descriptions are asked for two units ahead, a unit's first user and
// its block ids (lane b: of block b / 2) one unit ahead.
struct UnitWalk {
  const KeyArgs& a;
  const int64_t total;
  const int b;
  const KeyUnit* units;
  const KeyUser* users;
  int64_t i = 0;                                 // units looked at so far
  KeyUnit it, it1, it2;                          // the current one, the next, the one after that
  KeyUser user, user1;
  int h, h1, h2, bid, bid1;
  bool more, more1, more2;

  __device__ UnitWalk(const KeyArgs& args, int64_t n, int lane)
      : a(args), total(n), b(lane >> 1), units(args.plan->units()), users(args.plan->users()) {
    look();
    fetch();
    look();
    step();
  }
  __device__ void look() {
    more2 = false;
    while (i * gridDim.x < total && !more2) {
      const int64_t u = dealt(i++);
      if (u >= total) continue;
      it2 = units[u / a.shape.num_kv_heads];
      h2 = (int)(u % a.shape.num_kv_heads);
      more2 = true;
    }
  }
  __device__ void fetch() {
    more1 = more2;
    if (!more1) return;
    it1 = it2;
    h1 = h2;
    user1 = users[it1.user_begin];
    bid1 = b < (it1.tok_end - it1.tok_begin + kBlock - 1) / kBlock
               ? a.d_tables[(size_t)it1.table_row * a.shape.table_stride + it1.tok_begin / kBlock + b] : 0;
  }
  __device__ void step() {
    more = more1;
    if (!more) return;
    it = it1;
    user = user1;
    h = h1;
    bid = bid1;
    fetch();
    look();
  }
};

__global__ void __launch_bounds__(kWarps * 32, 1)
prompt_weights_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_q,
                      const KeyArgs a, int n_units) {
  extern __shared__ __align__(1024) uint8_t bp[];
  const uint32_t base = s32(bp);
  auto bar = [&](int i) { return base + kOffBar + 8u * i; };
  volatile int* cta_abort = (volatile int*)(bp + kOffBar + 8 * B_TOTAL);
  volatile uint32_t* tmem_slot = (volatile uint32_t*)(bp + kOffBar + 8 * B_TOTAL + 8);
  TileDesc* descs = (TileDesc*)(bp + kOffDesc);
  float* lses = (float*)(bp + kOffLse);
  volatile int* q_flags = (volatile int*)(bp + kOffFlags);
  const int G = a.shape.group, HQ = a.shape.num_q_heads, HKV = a.shape.num_kv_heads;
  const int T = kKeys / G;                       // tokens of a query tile
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  constexpr unsigned kAll = 0xffffffffu;

  if (threadIdx.x == 0) {
    *cta_abort = *(volatile int*)a.d_error;      // an earlier kernel gave up: do not pile up
    if (base & 1023) {                           // (the swizzle counts from 1024-byte boundaries)
      *cta_abort = 1;
      atomicCAS(a.d_error, 0, 25000);
    }
    asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)&tm_k) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"((uint64_t)&tm_q) : "memory");
    for (int b = 0; b < 2; ++b) {
      bar_init(bar(B_KFULL + b), 1);
      bar_init(bar(B_KEMPTY + b), 2);            // both issuers
    }
    for (int b = 0; b < 4; ++b) {
      bar_init(bar(B_WFULL + b), 4);
      bar_init(bar(B_WEMPTY + b), 4);
    }
    for (int s = 0; s < kQStages; ++s) {
      bar_init(bar(B_QFULL + s), 1);
      bar_init(bar(B_QEMPTY + s), 2);
    }
    for (int s = 0; s < kLStages; ++s) {
      bar_init(bar(B_LFULL + s), 1);
      bar_init(bar(B_LEMPTY + s), kSumWarps / 2);
    }
    for (int s = 0; s < 4; ++s) {
      bar_init(bar(B_SFULL + s), 1);
      bar_init(bar(B_SEMPTY + s), kSumWarps / 4);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  // rows of a query tile that the copies do not reach (where the group does not divide 128) are zero
  for (int i = threadIdx.x; i < kQStages * kTileB / 16; i += blockDim.x)
    *(uint4*)(bp + kOffQ + 16 * i) = make_uint4(0u, 0u, 0u, 0u);
  fence_async_smem();
  if (warp == kSumWarps + 2) {
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
  } else if (warp == kSumWarps) {
    // ---------------------------------------------------------------- copies
    int g = 0, ku = 0;                           // query tiles and units so far
    bool ok = true;
    const uint32_t q_bytes = 2u * T * G * 128u;
    for (UnitWalk u(a, total, lane); ok && u.more; u.step(), ++ku) {
      const int n_blk = (u.it.tok_end - u.it.tok_begin + kBlock - 1) / kBlock, kf = bar(B_KFULL + (ku & 1));
      if (ku >= 2)
        ok = __all_sync(kAll, bar_wait(bar(B_KEMPTY + (ku & 1)), ((ku >> 1) - 1) & 1, cta_abort, a.d_error,
                                       22100));
      if (!ok) break;
      if (lane == 0) bar_expect_tx(kf, (uint32_t)n_blk * kTileBytes);
      __syncwarp();
      // block b of the unit: 16 rows of its half of the keys, in two pieces of 64 dims
      if (u.b < n_blk)
        tma_2d(base + (ku & 1) * kUnitB + (u.b >> 3) * kTileB + (lane & 1) * kHalf + (u.b & 7) * (kBlock * 128),
               &tm_k, (lane & 1) * 64, (u.bid * HKV + u.h) * kBlock, kf);
      int flags = F_FIRST | (n_blk * kBlock > kKeys ? F_BOTH : 0);
      KeyUser user = u.user;
      for (int x = 0; ok; user = u.users[u.it.user_begin + x]) {
        const int end = user.query + user.count;
        ++x;
        for (int q0 = user.query + max(0, u.it.tok_begin - user.lim); q0 < end; q0 += T, ++g) {
          const int st = g % kQStages;
          if (g >= kQStages &&
              !__all_sync(kAll, bar_wait(bar(B_QEMPTY + st), (g / kQStages - 1) & 1, cta_abort, a.d_error,
                                         22000))) {
            ok = false;
            break;
          }
          if (x == u.it.n_users && q0 + T >= end) flags |= F_LAST;
          if (lane == 0) {
            q_flags[st] = flags;
            bar_expect_tx(bar(B_QFULL + st), q_bytes);
          }
          flags &= ~F_FIRST;
          __syncwarp();
          if (lane < 2)
            tma_3d(base + kOffQ + st * kTileB + lane * kHalf, &tm_q, lane * 64, u.h * G, q0, bar(B_QFULL + st));
        }
        if (x == u.it.n_users) break;
      }
    }
    const int st = g % kQStages;
    if (ok && g >= kQStages)
      ok = __all_sync(kAll, bar_wait(bar(B_QEMPTY + st), (g / kQStages - 1) & 1, cta_abort, a.d_error, 22400));
    if (ok && lane == 0) {
      q_flags[st] = F_END;
      bar_arrive(bar(B_QFULL + st));
    }
    // After a wait that gave up: the copies in flight are waited for (with a limit of their own).  On every way
    // here query tiles 0 .. g - 1 and units 0 .. ku - 1 have been asked for, and no others; the end's word (ok)
    // takes a stage as a tile does.
    if (*cta_abort && lane == 0) {
      for (int x = oldest_in_flight(ok ? g + 1 : g, kQStages); x < g; ++x)
        for (uint32_t i = 0; i < kSpin && !bar_try(bar(B_QFULL + x % kQStages), (x / kQStages) & 1); ++i) {}
      for (int x = oldest_in_flight(ku, 2); x < ku; ++x)
        for (uint32_t i = 0; i < kSpin && !bar_try(bar(B_KFULL + (x & 1)), (x >> 1) & 1); ++i) {}
    }
  } else if (warp == kSumWarps + 1) {
    // ---------------------------------------------------------------- log-sum-exps, descriptions
    const float* src[4];                         // this lane's rows of a tile that begins with query 0, head 0
    int row_of[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = lane + 32 * i;
      row_of[i] = r < T * G ? r : 1 << 30;
      src[i] = a.lse + (r < T * G ? r / G * HQ + r % G : 0);
    }
    int g = 0;
    bool ok = true;
    for (UnitWalk u(a, total, lane); ok && u.more; u.step()) {
      KeyUser user = u.user;
      int t = 0;
      for (int x = 0; ok; user = u.users[u.it.user_begin + x]) {
        ++x;
        int j = max(0, u.it.tok_begin - user.lim);
        int64_t at = (int64_t)(user.query + j) * HQ + u.h * G;
        float l[4];
        auto ask = [&](int n) {                  // a tile of n tokens
#pragma unroll
          for (int k = 0; k < 4; ++k) l[k] = row_of[k] < n * G ? __ldg(src[k] + at) : INFINITY;
        };
        ask(min(T, user.count - j));
        for (; j < user.count; j += T, ++g) {
          const int ls = g % kLStages;
          if (g >= kLStages &&
              !__all_sync(kAll, bar_wait(bar(B_LEMPTY + ls), (g / kLStages - 1) & 1, cta_abort, a.d_error,
                                         22300))) {
            ok = false;
            break;
          }
#pragma unroll
          for (int k = 0; k < 4; ++k) lses[ls * kKeys + lane + 32 * k] = l[k] * -1.4426950408889634f;
          if (lane == 0)
            descs[ls] = TileDesc{min(T, user.count - j), user.lim + j, u.it.tok_begin, u.it.tok_end,
                                 u.it.table_row, u.h, t, u.it.n_tiles};
          ++t;
          __syncwarp();
          if (lane == 0) bar_arrive(bar(B_LFULL + ls));
          at += (int64_t)T * HQ;
          ask(min(T, user.count - j - T));       // (of no tokens behind the last tile)
        }
        if (x == u.it.n_users) break;
      }
    }
    for (int x = 0; x < 2 && ok; ++x, ++g) {     // (one for each of the two that take turns)
      const int ls = g % kLStages;
      if (g >= kLStages)
        ok = __all_sync(kAll, bar_wait(bar(B_LEMPTY + ls), (g / kLStages - 1) & 1, cta_abort, a.d_error, 22200));
      if (ok && lane == 0) {
        descs[ls].n_tok = 0;
        bar_arrive(bar(B_LFULL + ls));
      }
    }
  } else if (warp > kSumWarps + 1) {
    // ---------------------------------------------------------------- products
    constexpr uint32_t kIdesc = instr_desc(128, false, 128);
    const int w = warp - kSumWarps - 2;
    int ku = 0, cnt[2] = {0, 0};                 // units; products of each buffer
    bool seen = false;                           // the tile was there at the last look
    for (int g = 0;; ++g) {
      const int st = g % kQStages, sb = g & 1;
      if (!__all_sync(kAll, seen) &&
          !__all_sync(kAll, bar_wait(bar(B_QFULL + st), (g / kQStages) & 1, cta_abort, a.d_error, 23000)))
        break;
      const int flags = q_flags[st];
      if (flags & F_END) break;
      if (w == 0 || (flags & F_BOTH)) {
        bool ok = true;
        if (flags & F_FIRST)
          ok = bar_wait(bar(B_KFULL + (ku & 1)), (ku >> 1) & 1, cta_abort, a.d_error, 23100);
        const int n = sb ? cnt[1]++ : cnt[0]++;
        if (n > 0)
          ok = ok && bar_wait(bar(B_SEMPTY + 2 * w + sb), (n - 1) & 1, cta_abort, a.d_error, 23200);
        if (!__all_sync(kAll, ok)) break;
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
          umma_commit(bar(B_QEMPTY + st));
          if (flags & F_LAST) umma_commit(bar(B_KEMPTY + (ku & 1)));
        }
      } else if (lane == 0) {                    // (nothing of this half in the unit)
        bar_arrive(bar(B_QEMPTY + st));
        if (flags & F_LAST) bar_arrive(bar(B_KEMPTY + (ku & 1)));
      }
      if (flags & F_LAST) ++ku;
      __syncwarp();
      seen = bar_test(bar(B_QFULL + (g + 1) % kQStages), ((g + 1) / kQStages) & 1);
    }
  } else {
    // ---------------------------------------------------------------- sums
    const int w = warp >> 3, turn = warp >> 2 & 1;   // half of the keys; even or odd tiles
    const int row = (warp & 3) * 32 + lane;        // the key's row of its half: its TMEM lane
    const uint32_t ts = (tmem + 256u * w + 128u * turn) | (uint32_t)((warp & 3) * 32) << 16;
    const float c = a.scale_log2e;
    const f32x2 c2 = pair(c, c);
    f32x2 acc[2] = {0ull, 0ull};
    int cnt = 0;                                   // times scores were taken
    // units of more than a tile whose first these warps had, or had not.  (Each has barriers of its own: a
    // warp may not wait for a phase before the one before it, which it has not seen, is complete.)
    int firsts = 0, seconds = 0;
    // Adds up 32 columns, of which lo .. hi - 1 see the key.
    auto add = [&](const uint32_t (&s)[32], const float* lse, int lo, int hi) {
      if (__all_sync(kAll, lo <= 0 && hi >= 32)) {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const f32x2 l = *(const f32x2*)(lse + 2 * j);                // (times - log2 e)
          const f32x2 x = fma2(pair(__uint_as_float(s[2 * j]), __uint_as_float(s[2 * j + 1])), c2, l);
          float e0, e1;
          unpair(x, e0, e1);
          acc[j & 1] = add2(acc[j & 1], pair(ex2(e0), ex2(e1)));
        }
      } else if (!__all_sync(kAll, lo >= 32 || hi <= 0)) {
        float part[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          const float p = ex2(fmaf(__uint_as_float(s[j]), c, lse[j]));
          if (j >= lo && j < hi) part[j & 1] += p;
        }
        acc[1] = add2(acc[1], pair(part[0], part[1]));
      }
    };
    for (int g = turn;; g += 2) {
      const int ls = g % kLStages;
      if (!__all_sync(kAll, bar_wait(bar(B_LFULL + ls), (g / kLStages) & 1, cta_abort, a.d_error, 24000)))
        break;
      const TileDesc d = descs[ls];
      if (d.n_tok == 0) break;
      const int key = d.tok_begin + kKeys * w + row;
      const bool used = d.tok_begin + kKeys * w < d.end;       // (the unit reaches into this half)
      if (used) {
        if (!__all_sync(kAll, bar_wait(bar(B_SFULL + 2 * w + turn), cnt & 1, cta_abort, a.d_error, 24100)))
          break;
        ++cnt;
        tc_fence_after();
        uint32_t s0[32], s1[32];
        TMEM_LD_32(ts, s0, 0);
        // by the tokens from the key's own position on; a whole tile but for zero rows behind its last
        // token, whose log-sum-exp is infinite
        const int lo = max(0, key - d.pos) * G, hi = d.n_tok == T ? kKeys : d.n_tok * G;
        const float* lse = lses + ls * kKeys;
        wait_scores(s0);
        TMEM_LD_32(ts + 32u, s1, 0);
        add(s0, lse, lo, hi);
        wait_scores(s1);
        TMEM_LD_32(ts + 64u, s0, 0);
        add(s1, lse + 32, lo - 32, hi - 32);
        wait_scores(s0);
        TMEM_LD_32(ts + 96u, s1, 0);
        add(s0, lse + 64, lo - 64, hi - 64);
        wait_scores(s1);
        tc_fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(bar(B_SEMPTY + 2 * w + turn));
        add(s1, lse + 96, lo - 96, hi - 96);
      }
      __syncwarp();
      if (lane == 0) bar_arrive(bar(B_LEMPTY + ls));
      if (used && d.t + 2 >= d.n_tiles) {          // the last one of the unit for these warps
        float sum, more;
        unpair(add2(acc[0], acc[1]), sum, more);
        sum += more;
        float* out = nullptr;
        if (key < d.end) {
          const int block = a.d_tables[(size_t)d.table_row * a.shape.table_stride + (key >> 4)];
          out = a.weights + ((size_t)block * HKV + d.kvh) * kBlock + (key & 15);
        }
        if (!(d.t & 1)) {
          const int full = B_WFULL + 2 * w + turn, empty = B_WEMPTY + 2 * w + turn;
          if (out) *out = a.replace ? sum : *out + sum;
          if (d.n_tiles > 1) {
            if (firsts > 0 &&
                !__all_sync(kAll, bar_wait(bar(empty), (firsts - 1) & 1, cta_abort, a.d_error, 24200)))
              break;
            __syncwarp();
            if (lane == 0) bar_arrive(bar(full));
            ++firsts;
          }
        } else {
          const int full = B_WFULL + 2 * w + (turn ^ 1), empty = B_WEMPTY + 2 * w + (turn ^ 1);
          if (!__all_sync(kAll, bar_wait(bar(full), seconds & 1, cta_abort, a.d_error, 24300))) break;
          if (lane == 0) bar_arrive(bar(empty));
          if (out) *out += sum;
          ++seconds;
        }
        acc[0] = acc[1] = 0ull;
      }
    }
  }
  // ---- common exit: every role arrives here, then the allocating warp frees TMEM
  tc_fence_before();
  __syncthreads();
  if (warp == kSumWarps + 2) {
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
  return launch_kernel(prompt_weights_kernel, dim3(grid), dim3(kWarps * 32), kSmem, st, false, *tm_k, *tm_q, a, n_units);
}

}  // namespace apar
