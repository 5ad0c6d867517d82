// Tree attention over a KV pool held in 4 bits for work items with more than eight query rows
// (prompts shared by siblings, candidates of a verification, GQA groups above eight), on the
// Blackwell tensor cores (tcgen05).
//
// mma.sync has to turn the codes of a block into operand registers once per eight rows, which for
// 64 rows costs eight times the arithmetic of one; here a block is turned into f16 operand tiles in
// shared memory once for all of an item's rows.  A unit is one item and kv head (at most 64 rows),
// walked in tiles of 64 tokens; two persistent CTAs per SM take units in the planner's order, forwards
// and backwards in turn, and every role runs on from one unit into the next (a CTA per unit spent
// some 6 us on each: 92 of 178 us of a case whose roles did nothing else):
//   warps 4-7  one block of the tile each: its 4-bit K and V tiles arrive by cp.async while the tile
//              before is converted, and leave as f16 operands.
//              K' = s (c - 8) 2^-e, e from the token's largest scale: eight bits of s times at
//              most three of c - 8, so exact for scales down to 2^-12 of that one, and beyond it
//              good to 2^-20 of it.  A code enters as the subnormal number c * 2^-20, brought to
//              the second nibble of its 16 bits; one fused multiply-add per pair of values.
//              What is left of a key, lo + 8 s of each group, meets the query's sum over the group
//              in one more product: lo and 8 s in f16 (exact too) against that sum as two f16
//              numbers, which makes a k of 16.  Scores are then as good as 32-bit sums, whatever
//              the keys have in common.  (Keys rounded to 11 bits with their offsets inside, under one
//              exponent per block, made errors of the exponent: 2.6 times the output's rounding
//              where two channels had offsets of 16, seventy times at 200.)
//              V' = V 2^(13 - F), F the exponent of the token's largest value, rounded to 11 bits:
//              normal numbers down to 2^-27 of that.  (Scaled to 2^-8, as the codes as they
//              lie in the word would have it, a group 2^10 below the row's largest lost its digits.)
//              Here a code enters as 1024 + c, or 1024 + 16 c a nibble up, less the constant.
//              At a unit's first tile they also stage its query rows, 16 each.  One fence and one
//              arrival per tile cover all of it (separate ones for K', V' and Q: 148 us instead of
//              139).
//   warp 8     issues S = Q K'^T (M 64, N 64, K 128 + 16) and, one tile behind, O += P V' (M 64, N 128,
//              K 64).
//   warps 0-3  16 rows each, a row's scores spread over a quad: x = S u 2^e + F - 13,
//              P = 2^(x - ref) in f16, its sum less the token's factor in 32 bits, P to shared memory
//              as an operand.  The reference follows score and size of V together and moves
//              lazily, as in attn_q4.cu.  (With a thread per row - M 128, P in tensor memory -
//              every thread reads every token's constants, a quarter of the shared-memory cycles.)
// K', V' and S are double-buffered; P is not, for want of shared memory.  Weights and V' are rounded
// to 11 bits, against eight of the output.
// All waits are bounded; a wait that gives up raises the error word and every role unwinds to the
// common exit where TMEM is released.
//
// Measured: 64 prompts of 2048 tokens, 64 rows on each of 8 kv heads (34 GFLOP, 168 MB): 155 us;
// 2496 candidates of 96 threads, 40 or 64 rows, 32 heads over 8: 193 us.  With keys rounded to 11 bits
// and V scaled to 2^-8 it was 139 and 172: V's codes by way of 1024 + c cost 8 us of each, the exact
// keys the rest.  (Then a tile took a CTA some 3600 cycles, of which a converter warp was busy 2500,
// a softmax warp 2300 and the MMA warp 1500; the converters' share is what grew.)  No single unit
// is full: the roles wait for one another, and 18 warps of different code miss the instruction
// cache (a sixth of the stalls).
#include <algorithm>
#include <climits>

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include "apar_internal.h"
#include "kv4.cuh"
#include "ptx.cuh"
#include "tcgen05.cuh"

namespace apar {
namespace {

constexpr int kTok = 64;                             // tokens of a tile
constexpr int kConv = 4, kSoftmax = 4;               // warps
constexpr int kThreads = 32 * (kSoftmax + kConv + 1);
constexpr int kBlk = 2 * kQ4TileBytes;               // K and V of one block, as stored
constexpr int kHalfOp = 64 * 128;                    // 64 rows x 64 dims f16, 128-byte swizzle
constexpr int kOpBytes = 2 * kHalfOp;                // K' or V' of a tile, or Q
constexpr int kOffK = kOpBytes;
constexpr int kOffVw = kOffK + 2 * kOpBytes;
constexpr int kOffP = kOffVw + 2 * kOpBytes;         // P: 64 rows x 64 tokens f16
constexpr int kCoreBytes = 64 * 16;                  // 64 rows x 8 f16, no swizzle: 8 rows to 128 bytes
constexpr int kMidBytes = 2 * kCoreBytes;            // lo, 8 s of a tile's tokens, or the rows' sums
constexpr int kOffQmid = kOffP + kHalfOp;
constexpr int kOffKmid = kOffQmid + kMidBytes;
constexpr int kOffRaw = kOffKmid + 2 * kMidBytes;
constexpr int kOffTok = kOffRaw + kConv * kBlk;      // [2] F - 13, 2^(13 - F), 2^(e - 8) of 64 tokens
constexpr int kTokc = 3 * kTok;
constexpr int kOffRow = kOffTok + 2 * kTokc * 4;              // [4 units][64] the rows' factors
constexpr int kOffBarW = kOffRow + 4 * 64 * 4;
enum { BW_FULL = 0, BW_KEMPTY = 2, BW_VEMPTY = 4, BW_SFULL = 6, BW_PFULL = 8, BW_PVDONE = 9,
       BW_ODONE = 10, BW_TOTAL = 11 };
constexpr int kSmemWide = kOffBarW + 8 * BW_TOTAL + 16;
static_assert(2 * (kSmemWide + 1024) <= 228 * 1024, "two CTAs per SM");
constexpr int kTmemColsW = 256;                      // S at 0 and 64, O at 128
constexpr float kHeadroomW = 6.f, kSlackW = 15.5f;   // as in attn_q4.cu, but set to 2^6: V' has taken the
                                                     // sizes of the groups on itself, and moving O
                                                     // costs more here (with 2^12 the candidates
                                                     // took 201 us instead of 190)
constexpr float kNoRefW = -3e38f;
constexpr int kLiftV = 13;                           // exponent of the largest values of V'
constexpr int kDropK = 5;                            // e less the exponent of the largest scale: that one
                                                     // times 2^20 (for the codes) is then below 2^16
constexpr int kLiftMid = 7;                          // lo and 8 s stand that much above K', sums below
constexpr int kStepK = 8;                            // of e, carried by the rows' factors (range)
constexpr uint32_t kEvenW = 0x000f000fu, kOddW = 0x00f000f0u;
constexpr uint32_t kSixteenth = 0x2c002c00u;         // f16 1/16 twice
constexpr int kMinExpV = -60;                        // V rows below 2^-60 count as of that size

// D fp32, A and B f16, both K-major.
__host__ __device__ constexpr uint32_t instr_desc_f16(int n, int m) {
  return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ uint32_t f16x2(float lo, float hi) {
  __half2 h = __floats2half2_rn(lo, hi);
  return *(uint32_t*)&h;
}
__device__ __forceinline__ uint32_t hfma2(uint32_t a, uint32_t b, uint32_t c) {
  __half2 r = __hfma2(*(__half2*)&a, *(__half2*)&b, *(__half2*)&c);
  return *(uint32_t*)&r;
}
__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b) {
  __half2 r = __hmul2(*(__half2*)&a, *(__half2*)&b);
  return *(uint32_t*)&r;
}
__device__ __forceinline__ uint32_t hadd2(uint32_t a, uint32_t b) {
  __half2 r = __hadd2(*(__half2*)&a, *(__half2*)&b);
  return *(uint32_t*)&r;
}
// The f16 pairs c of nibbles 0 and 4 of a word, and of nibbles 1 and 5; exact.
__device__ __forceinline__ uint32_t codes_even(uint32_t w) {
  return hadd2((w & kEvenW) | 0x64006400u, 0xe400e400u);               // less 1024
}
__device__ __forceinline__ uint32_t codes_odd(uint32_t w) {
  return hfma2((w & kOddW) | 0x64006400u, kSixteenth, 0xd400d400u);    // a sixteenth, less 64
}
__device__ __forceinline__ float pow2(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
// exponent of a non-negative number, kept away from the low end of the range
__device__ __forceinline__ int exponent_of(float x, int lowest) {
  return min(127, max(lowest, (int)(__float_as_uint(x) >> 23) - 127));
}
// Descriptor of a K-major operand without swizzle whose second eight k lie kCoreBytes on.
__device__ __forceinline__ uint64_t core_desc(uint32_t addr) {
  return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(kCoreBytes >> 4) << 16) |
         ((uint64_t)(128 >> 4) << 32) | (1ull << 46);
}
// largest magnitude a group can stand for
__device__ __forceinline__ float group_top(uint32_t sl) {
  const float s = bf16_lo(sl), lo = bf16_hi(sl);
  return fmaxf(fabsf(lo), fabsf(fmaf(15.f, s, lo)));   // (a NaN group counts as 0)
}
// Orders chosen so that the converters' shared-memory accesses fall into different banks.  Token of
// a block that takes row (K', and column of V') pos of it: bits 2 and 3 change places.  Row of V'
// that holds dim 32 G + 4 g + e: 32 G + 4 g + (e ^ G).
__device__ __forceinline__ int token_at(int pos) {
  return (pos & 3) | ((pos & 4) << 1) | ((pos & 8) >> 1);
}
#define TMEM_LD_16(taddr, r)                                                                     \
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 "                                         \
               "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"                  \
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]),         \
                 "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),       \
                 "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])                              \
               : "r"(taddr))
#define TMEM_ST_16(taddr, r)                                                                     \
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "                                   \
               "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"                        \
               ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]),   \
                 "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), \
                 "r"(r[13]), "r"(r[14]), "r"(r[15])                                              \
               : "memory")
#define TMEM_LD_16x256_32(taddr, r)                                                              \
  asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 "                                         \
               "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"                  \
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]),         \
                 "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),       \
                 "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])                              \
               : "r"(taddr))
__device__ __forceinline__ void cp16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

__global__ void __launch_bounds__(kThreads, 2)
attn_q4_wide_kernel(const AttnArgs a, int n_units) {
  extern __shared__ __align__(1024) uint8_t bp[];    // (swizzled operands want 1024)
  const uint32_t base = s32(bp);
  if (base & 1023u) {                                // no room to round it up: refuse
    if (threadIdx.x == 0) atomicCAS(a.d_error, 0, 25000);
    return;
  }
  auto bar = [&](int i) { return base + kOffBarW + 8u * i; };
  volatile int* cta_abort = (volatile int*)(bp + kOffBarW + 8 * BW_TOTAL);
  volatile uint32_t* tmem_slot = (volatile uint32_t*)(bp + kOffBarW + 8 * BW_TOTAL + 8);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int G = a.shape.group, HQ = a.shape.num_q_heads, HKV = a.shape.num_kv_heads;
  pdl_launch_dependents();

  if (threadIdx.x == 0) {
    *cta_abort = *(volatile int*)a.d_error;          // an earlier kernel gave up: do not pile up
    for (int b = 0; b < 2; ++b) {
      bar_init(bar(BW_FULL + b), kConv);
      bar_init(bar(BW_KEMPTY + b), 1);
      bar_init(bar(BW_VEMPTY + b), 1);
      bar_init(bar(BW_SFULL + b), 1);
    }
    bar_init(bar(BW_PFULL), kSoftmax);
    bar_init(bar(BW_PVDONE), 1);
    bar_init(bar(BW_ODONE), kSoftmax);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;"
                 ::"r"(s32((const void*)tmem_slot)), "r"(kTmemColsW) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  // this CTA's units: number `pass` of the list, or -1
  const int W = gridDim.x;
  auto unit_of = [&](int pass) {
    const int u = pass * W + ((pass & 1) ? W - 1 - (int)blockIdx.x : (int)blockIdx.x);
    return u < n_units ? u : -1;
  };
  const int n_passes = (n_units + W - 1) / W;        // (the last one may have no unit for this CTA)
  const int my_units = n_passes - (unit_of(n_passes - 1) < 0 ? 1 : 0);
  struct Unit {
    int row, begin, n_tok, n_tiles, kvh;
  };
  auto describe = [&](int pass) {
    const int u = unit_of(pass);
    const WorkItem& it = a.d_items[u / HKV];
    Unit d;
    d.row = it.table_row;
    d.begin = it.tok_begin;
    d.n_tok = (it.tok_end < 0 ? a.d_lens[d.row] : it.tok_end) - d.begin;
    d.n_tiles = (d.n_tok + kTok - 1) / kTok;
    d.kvh = u % HKV;
    return d;
  };
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;

  if (*cta_abort) {
    // nothing is started
  } else if (warp >= kSoftmax && warp < kSoftmax + kConv) {
    // ---------------------------------------------------------------- converters
    const int cw = warp - kSoftmax;
    const uint32_t raw = base + kOffRaw + cw * kBlk;
    // the loads run a tile ahead, into the next units too: a tile's block is asked for once the
    // one before is in registers, and has all of its conversion to arrive in
    Unit lu = {0, 0, 0, 0, 0}, nu = my_units ? describe(0) : lu;   // the loads' unit; the one after it
    int l_pass = -1, l_t = 0, l_bid = 0;
    const int32_t* l_tab = nullptr;
    auto load_tile = [&]() {                         // this warp's block of the next tile, if any
      if (l_t == lu.n_tiles && l_pass + 1 < my_units) {
        lu = nu;
        ++l_pass;
        l_t = 0;
        l_tab = a.d_tables + (size_t)lu.row * a.shape.table_stride + lu.begin / kBlock;
        l_bid = cw * kBlock < lu.n_tok ? l_tab[cw] : 0;
        if (l_pass + 1 < my_units) nu = describe(l_pass + 1);
      }
      if (l_t < lu.n_tiles) {
        if ((l_t * kConv + cw) * kBlock < lu.n_tok) {
          const size_t tile = ((size_t)l_bid * HKV + lu.kvh) * kQ4TileBytes + lane * 16;
          const uint8_t* kt = (const uint8_t*)a.k_pool + tile;
          const uint8_t* vt = (const uint8_t*)a.v_pool + tile - kQ4TileBytes;
          const uint32_t dst = raw + lane * 16;
          cp16(dst, kt);
          cp16(dst + 512, kt + 512);
          cp16(dst + 1024, (lane < 16 ? kt : vt) + 1024);
          cp16(dst + 1536, vt + 1536);
          cp16(dst + 2048, vt + 2048);
        }
        ++l_t;
        const int nb = l_t * kConv + cw;
        if (nb * kBlock < lu.n_tok) l_bid = l_tab[nb];         // (arrives while a tile is converted)
      }
    };
    load_tile();
    int T = 0;                                       // tiles of all units
    // The query rows of the unit whose first tile is T into the operand, in f16 under a power of two
    // of their own: this warp's 16, a lane four pieces of rows lane / 4 and lane / 4 + 8.  (By these
    // warps, which have the time: the softmax warps spent 6000 cycles on it between two units.)
    auto stage_rows = [&](int pass) -> bool {
      const int un = unit_of(pass), g8 = lane >> 2, qd = lane & 3;
      const WorkItem& it = a.d_items[un / HKV];
      const int count = it.n_users * G, head0 = un % HKV * G, first = it.user_begin;
      uint4 v[2][4];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = cw * 16 + g8 + 8 * e, u = r / G;
        const bool on = r < count;
        const int query = on ? a.d_users[first + u].query : 0;
        const uint4* src = (const uint4*)a.q + ((size_t)query * HQ + head0 + (r - u * G)) * 16 + qd;
#pragma unroll
        for (int j = 0; j < 4; ++j) v[e][j] = on ? __ldg(src + 4 * j) : make_uint4(0u, 0u, 0u, 0u);
      }
      // the products of the unit before with its rows are complete
      if (T > 0 && !__all_sync(0xffffffffu, bar_wait(bar(BW_KEMPTY + ((T - 1) & 1)), ((T - 1) >> 1) & 1,
                                                     cta_abort, a.d_error, 23400)))
        return false;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = cw * 16 + g8 + 8 * e;
        uint32_t top = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          top = __vmaxu2(top, __vmaxu2(__vmaxu2(v[e][j].x & 0x7fff7fffu, v[e][j].y & 0x7fff7fffu),
                                       __vmaxu2(v[e][j].z & 0x7fff7fffu, v[e][j].w & 0x7fff7fffu)));
        top = max(top & 0xffffu, top >> 16);
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const int lift = min(126, 14 + 127 - (int)(top >> 7));
        const float f = pow2(lift);
        float sum[4];                                // over dims 32 j .. 32 j + 31
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int c = qd + 4 * j;
          const uint32_t w[4] = {v[e][j].x, v[e][j].y, v[e][j].z, v[e][j].w};
          uint32_t h[4];
          sum[j] = 0.f;
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            const float e0 = bf16_lo(w[p]) * f, e1 = bf16_hi(w[p]) * f;
            sum[j] += e0 + e1;
            h[p] = f16x2(e0, e1);
          }
          sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 1);
          sum[j] += __shfl_xor_sync(0xffffffffu, sum[j], 2);
          sum[j] *= 1.f / (1 << kLiftMid);
          *(uint4*)(bp + (c >> 3) * kHalfOp + r * 128 + (((c & 7) ^ (r & 7)) << 4)) =
              make_uint4(h[0], h[1], h[2], h[3]);
        }
        if (qd < 2) {                                // the sums to 11 bits, and what that leaves
          float part[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float first = __half2float(__float2half_rn(sum[j]));
            part[j] = qd ? sum[j] - first : first;
          }
          const uint32_t p01 = f16x2(part[0], part[1]), p23 = f16x2(part[2], part[3]);
          *(uint4*)(bp + kOffQmid + qd * kCoreBytes + r * 16) = make_uint4(p01, p23, p01, p23);
        }
        // (the softmax warps read them at the unit's first tile: four units on they have)
        if (qd == 0) ((float*)(bp + kOffRow))[(pass & 3) * 64 + r] = a.scale_log2e * pow2(kStepK - lift);
      }
      return true;
    };
    bool ok = true;
#pragma unroll 1
    for (int pass = 0; pass < my_units && ok; ++pass) {
      const Unit cu = describe(pass);                // (in the L1 cache by now)
#pragma unroll 1
    for (int t = 0; t < cu.n_tiles; ++t, ++T) {
      const int b = T & 1;
      asm volatile("cp.async.wait_all;" ::: "memory");
      __syncwarp();
      const uint8_t* kt = bp + (raw - base);
      const uint8_t* vt = kt + kQ4TileBytes;
      const int nv = cu.n_tok - (t * kConv + cw) * kBlock;   // tokens of the block that count

      // ---- what the tile holds, and the factors (both chains of shuffles at once)
      // K: lane = (operand row, half of its 16-byte pieces).  V: lane = (pair, group) for the
      // factors; then its group is that of its words, lane % 4, in both rounds, and its pairs are
      // those of operand columns 8 pg .. 8 pg + 7.
      const int pos = lane & 15, h = lane >> 4, tok = token_at(pos);
      const int pair = lane >> 2, g4 = lane & 3, pg = lane >> 4, GG = lane & 3;
      uint4 sc = *(const uint4*)(kt + tok * kQ4RowBytes + kQ4CodeBytes);
      const uint8_t* vsc = vt + pair * kQ4PairBytes + 2 * kQ4CodeBytes + 4 * g4;
      uint32_t se = *(const uint32_t*)vsc, so = *(const uint32_t*)(vsc + 16);
      const uint4 c0 = *(const uint4*)(kt + tok * kQ4RowBytes + 32 * h);
      const uint4 c1 = *(const uint4*)(kt + tok * kQ4RowBytes + 32 * h + 16);
      uint32_t w[2][4];
#pragma unroll
      for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int i = 0; i < 2; ++i)                          // word 4 g + G
          w[i][p] = *(const uint32_t*)(vt + (2 * pg) * kQ4PairBytes + 4 * (lane & 15) +
                                       ((p & 1) + 2 * (p & 2)) * kQ4PairBytes + 64 * i);
      if (tok >= nv) sc = make_uint4(0u, 0u, 0u, 0u);        // (unspecified bits: the row is zeros)
      if (2 * pair >= nv) se = 0u;
      if (2 * pair + 1 >= nv) so = 0u;
      const uint32_t sl[4] = {sc.x, sc.y, sc.z, sc.w};
      float te = group_top(se), to = group_top(so);
#pragma unroll
      for (int d = 1; d <= 2; d <<= 1) {
        te = fmaxf(te, __shfl_xor_sync(0xffffffffu, te, d));
        to = fmaxf(to, __shfl_xor_sync(0xffffffffu, to, d));
      }
      // the token's largest scale; and lo has to stay below 2^16 where all groups are flat
      const float s_top = fmaxf(fmaxf(bf16_lo(sl[0]), bf16_lo(sl[1])),
                                fmaxf(bf16_lo(sl[2]), bf16_lo(sl[3])));
      const float lo_top = fmaxf(fmaxf(fabsf(bf16_hi(sl[0])), fabsf(bf16_hi(sl[1]))),
                                 fmaxf(fabsf(bf16_hi(sl[2])), fabsf(bf16_hi(sl[3]))));
      const int ek = max(min(exponent_of(s_top, -100), 124) + kDropK, exponent_of(lo_top, -100) + kLiftMid - 14);
      const int ee = exponent_of(te, kMinExpV) - kLiftV, eo = exponent_of(to, kMinExpV) - kLiftV;
      const float de = pow2(-ee), dn = pow2(-eo);
      const uint32_t x1 = f16x2(bf16_lo(se) * de, bf16_lo(so) * dn);
      const uint32_t xl = f16x2(bf16_hi(se) * de, bf16_hi(so) * dn);
      // ---- K
      {
        const float up = pow2(20 - ek);
        if (T >= 2 && !__all_sync(0xffffffffu, bar_wait(bar(BW_KEMPTY + b), ((T >> 1) - 1) & 1, cta_abort,
                                                        a.d_error, 23000))) {
          ok = false;
          break;
        }
        const uint32_t w0[4] = {c0.x, c0.y, c0.z, c0.w}, w1[4] = {c1.x, c1.y, c1.z, c1.w};
        const int r = cw * kBlock + pos;
        // 16-byte piece c of the row lies at c ^ (r % 8) of its half; c = 4 j + 2 h + x
        uint8_t* const dst = bp + kOffK + b * kOpBytes + r * 128;
        const uint32_t piece = (uint32_t)((2 * h) ^ (r & 7)) << 4;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float s = bf16_lo(sl[j]) * up;
          const uint32_t s1 = f16x2(s, s), m8 = hmul2(s1, 0x80808080u);   // (-8 * 2^-20 as an f16 number)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const uint32_t kw = x ? w1[j] : w0[j];
            *(uint4*)(dst + (j >> 1) * kHalfOp + (piece ^ ((4 * (j & 1) + x) << 4))) =
                make_uint4(hfma2((kw << 4) & kOddW, s1, m8), hfma2(kw & kOddW, s1, m8),
                           hfma2((kw >> 4) & kOddW, s1, m8), hfma2((kw >> 8) & kOddW, s1, m8));
          }
        }
        // lo and 8 s of the four groups, for either half of the query's sums
        const float dm = pow2(kLiftMid - ek), d8 = pow2(kLiftMid + 3 - ek);
        *(uint4*)(bp + kOffKmid + b * kMidBytes + h * kCoreBytes + r * 16) =
            make_uint4(f16x2(bf16_hi(sl[0]) * dm, bf16_hi(sl[1]) * dm),
                       f16x2(bf16_hi(sl[2]) * dm, bf16_hi(sl[3]) * dm),
                       f16x2(bf16_lo(sl[0]) * d8, bf16_lo(sl[1]) * d8),
                       f16x2(bf16_lo(sl[2]) * d8, bf16_lo(sl[3]) * d8));
      }
      if (t == 0 && !stage_rows(pass)) {
        ok = false;
        break;
      }
      __syncwarp();                                          // (the raw tile has been read by all)
      load_tile();
      // ---- V
      {
        uint32_t v1[4], vl[4];                               // of the four pairs, from the lanes
#pragma unroll                                               // that made them
        for (int p = 0; p < 4; ++p) {
          const int from = 8 * pg + GG + 4 * ((p & 1) + 2 * (p & 2));    // pair token_at(8 pg + 2 p) / 2
          v1[p] = __shfl_sync(0xffffffffu, x1, from);
          vl[p] = __shfl_sync(0xffffffffu, xl, from);
        }
        if (T >= 2 && !__all_sync(0xffffffffu, bar_wait(bar(BW_VEMPTY + b), ((T >> 1) - 1) & 1,
                                                        cta_abort, a.d_error, 23200))) {
          ok = false;
          break;
        }
        if (g4 == 0) {                                       // (a pair stays together)
          float* tokc = (float*)(bp + kOffTok) + b * kTokc + cw * kBlock + token_at(2 * pair);
          const bool e_on = 2 * pair < nv, o_on = 2 * pair + 1 < nv;
          *(float2*)tokc = make_float2(e_on ? (float)ee : -INFINITY, o_on ? (float)eo : -INFINITY);
          *(float2*)(tokc + kTok) = make_float2(e_on ? pow2(-ee) : 0.f, o_on ? pow2(-eo) : 0.f);
        }
        if (h == 0)
          ((float*)(bp + kOffTok))[b * kTokc + 2 * kTok + cw * kBlock + pos] = pow2(ek - kStepK);
        // operand row of word 4 g + G, dim e: d = 32 G + 4 g + (e ^ G), piece 2 cw + pg at its
        // place xor d % 8
        const int d0 = 32 * GG + 4 * ((lane & 15) >> 2), at = (2 * cw + pg) ^ (d0 & 4);
        uint8_t* const dst = bp + kOffVw + b * kOpBytes + d0 * 128;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t out[4][4];                                // [dim][pair]
#pragma unroll
          for (int p = 0; p < 4; ++p) {
            const uint32_t x = w[i][p], xh = x >> 8;
            out[0][p] = hfma2(codes_even(x), v1[p], vl[p]);
            out[1][p] = hfma2(codes_odd(x), v1[p], vl[p]);
            out[2][p] = hfma2(codes_even(xh), v1[p], vl[p]);
            out[3][p] = hfma2(codes_odd(xh), v1[p], vl[p]);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int u = e ^ GG;
            *(uint4*)(dst + u * 128 + ((at ^ u) << 4) + i * 16 * 128) =
                make_uint4(out[e][0], out[e][1], out[e][2], out[e][3]);
          }
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) bar_arrive(bar(BW_FULL + b));
      }
    }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  } else if (warp == 8) {
    // ---------------------------------------------------------------- MMA issuer
    constexpr uint32_t kIdescQK = instr_desc_f16(kTok, 64), kIdescPV = instr_desc_f16(kDim, 64);
    constexpr unsigned kAll = 0xffffffffu;
    // (addresses stay below 2^18: adding to the address field, in 16 bytes, carries nowhere)
    const uint64_t desc_q = smem_desc(base, 16, 1024), desc_p = smem_desc(base + kOffP, 16, 1024);
    const uint64_t desc_qm = core_desc(base + kOffQmid);
    int T = 0, due = -1;                             // tiles so far; the tile whose P V is due
    bool due_first = false, ok = true;
    int due_pass = 0;
    auto product_pv = [&]() -> bool {
      const int b = due & 1;
      bool w8 = bar_wait(bar(BW_PFULL), due & 1, cta_abort, a.d_error, 24100);
      if (due_first && due_pass > 0)                 // the unit before has read its O out
        w8 = w8 && bar_wait(bar(BW_ODONE), (due_pass - 1) & 1, cta_abort, a.d_error, 24300);
      if (!__all_sync(kAll, w8)) return false;
      tc_fence_after();
      if (lane == 0) {
        const uint64_t desc_v = smem_desc(base + kOffVw + b * kOpBytes, 16, 1024);
#pragma unroll
        for (int kk = 0; kk < kTok / 16; ++kk)
          umma_bf16(tmem + 128u, desc_p + 2 * kk, desc_v + 2 * kk, kIdescPV, !due_first || kk > 0);
        umma_commit(bar(BW_VEMPTY + b));
        umma_commit(bar(BW_PVDONE));
      }
      __syncwarp();
      due = -1;
      return true;
    };
    for (int pass = 0; pass < my_units && ok; ++pass) {
      const int n_tiles = describe(pass).n_tiles;
      for (int t = 0; t < n_tiles; ++t, ++T) {
        const int b = T & 1;
        // between units the last P V goes first: the rows of the next unit come after it
        if (t == 0 && due >= 0 && !product_pv()) {
          ok = false;
          break;
        }
        bool w8 = bar_wait(bar(BW_FULL + b), (T >> 1) & 1, cta_abort, a.d_error, 24000);
        if (!__all_sync(kAll, w8)) {
          ok = false;
          break;
        }
        tc_fence_after();
        if (lane == 0) {
          const uint64_t desc_k = smem_desc(base + kOffK + b * kOpBytes, 16, 1024);
#pragma unroll
          for (int ks = 0; ks < 8; ++ks) {
            const uint32_t off = (ks >> 2) * kHalfOp + (ks & 3) * 32;
            umma_bf16(tmem + 64u * b, desc_q + (off >> 4), desc_k + (off >> 4), kIdescQK, ks > 0);
          }
          umma_bf16(tmem + 64u * b, desc_qm, core_desc(base + kOffKmid + b * kMidBytes), kIdescQK, 1);
          umma_commit(bar(BW_SFULL + b));
          umma_commit(bar(BW_KEMPTY + b));
        }
        __syncwarp();
        if (due >= 0 && !product_pv()) {
          ok = false;
          break;
        }
        due = T;
        due_first = t == 0;
        due_pass = pass;
      }
    }
    if (ok && due >= 0) product_pv();
  } else {
    // ---------------------------------------------------------------- softmax
    // Warp w owns rows 16 w .. 16 w + 15 (an M 64 accumulator keeps them in the first 16 lanes of
    // its quarter of tensor memory); a lane works on rows g8 and g8 + 8 of them and the tokens
    // 8 k + 2 qd, 8 k + 2 qd + 1.
    const int g8 = lane >> 2, qd = lane & 3;
    const uint32_t lane_sel = (uint32_t)(warp * 32) << 16, tm_o = tmem + 128u;
    float u_lo = 0.f, u_hi = 0.f;                    // scale * log2(e) / the rows' factors
    // The unit's item and the users of the lane's two rows are read ahead.
    struct Rows {
      int count, begin, add, head0;
      UserRef user[2];
    } cur, nxt;
    auto read_item = [&](int pass, Rows& r) {
      const int un = unit_of(pass);
      const WorkItem& it = a.d_items[un / HKV];
      r.count = it.n_users * G;
      r.begin = it.user_begin;
      r.add = it.slot_add;
      r.head0 = un % HKV * G;
    };
    auto read_users = [&](Rows& r) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int row = warp * 16 + g8 + 8 * e;
        r.user[e] = UserRef{0, -1};
        if (row < r.count) r.user[e] = a.d_users[r.begin + row / G];
      }
    };
    int T = 0;
    bool alive = true;
    if (my_units) {
      read_item(0, nxt);
      read_users(nxt);
    }
#pragma unroll 1
    for (int pass = 0; pass < my_units; ++pass) {
      cur = nxt;
      const int R = cur.count;
      const bool more = pass + 1 < my_units;
      if (more) read_item(pass + 1, nxt);
      const int n_tiles = describe(pass).n_tiles;
      const bool idle = warp * 16 >= R;              // (no rows here: only keeps the phases)
      float ref_lo = kNoRefW, ref_hi = kNoRefW, l_lo = 0.f, l_hi = 0.f;
#pragma unroll 1
      for (int t = 0; t < n_tiles; ++t, ++T) {
        const int b = T & 1;
        bool ok = bar_wait(bar(BW_SFULL + b), (T >> 1) & 1, cta_abort, a.d_error, 22000);
        ok = ok && bar_wait(bar(BW_FULL + b), (T >> 1) & 1, cta_abort, a.d_error, 22100);
        if (!__all_sync(0xffffffffu, ok)) {
          alive = false;
          break;
        }
        tc_fence_after();
        if (t == 0) {
          const float* factor = (const float*)(bp + kOffRow) + (pass & 3) * 64 + warp * 16 + g8;
          u_lo = factor[0];
          u_hi = factor[8];
        }
        uint32_t pk_lo[8], pk_hi[8];
        if (!idle) {
          uint32_t sr[32];
          TMEM_LD_16x256((tmem + 64u * b) | lane_sel, sr);
          const float* tokc = (const float*)(bp + kOffTok) + b * kTokc + 2 * qd;
          float2 f[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) f[k] = *(const float2*)(tokc + 8 * k);
          tmem_wait_ld();
          float m_lo = -INFINITY, m_hi = -INFINITY;
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float2 e = *(const float2*)(tokc + 2 * kTok + 8 * k);
            const float x0 = fmaf(__uint_as_float(sr[4 * k]), u_lo * e.x, f[k].x);
            const float x1 = fmaf(__uint_as_float(sr[4 * k + 1]), u_lo * e.y, f[k].y);
            const float x2 = fmaf(__uint_as_float(sr[4 * k + 2]), u_hi * e.x, f[k].x);
            const float x3 = fmaf(__uint_as_float(sr[4 * k + 3]), u_hi * e.y, f[k].y);
            m_lo = fmaxf(m_lo, fmaxf(x0, x1));
            m_hi = fmaxf(m_hi, fmaxf(x2, x3));
            sr[4 * k] = __float_as_uint(x0);
            sr[4 * k + 1] = __float_as_uint(x1);
            sr[4 * k + 2] = __float_as_uint(x2);
            sr[4 * k + 3] = __float_as_uint(x3);
          }
          if (__any_sync(0xffffffffu, m_lo > ref_lo + kSlackW || m_hi > ref_hi + kSlackW)) {
#pragma unroll
            for (int d = 1; d <= 2; d <<= 1) {
              m_lo = fmaxf(m_lo, __shfl_xor_sync(0xffffffffu, m_lo, d));
              m_hi = fmaxf(m_hi, __shfl_xor_sync(0xffffffffu, m_hi, d));
            }
            m_lo = fmaxf(m_lo - kHeadroomW, ref_lo);
            m_hi = fmaxf(m_hi - kHeadroomW, ref_hi);
            const float f_lo = ex2(ref_lo - m_lo), f_hi = ex2(ref_hi - m_hi);
            ref_lo = m_lo;
            ref_hi = m_hi;
            l_lo *= f_lo;
            l_hi *= f_hi;
            if (t > 0) {                             // (P V of the tile before has to be complete)
              if (!__all_sync(0xffffffffu, bar_wait(bar(BW_PVDONE), (T - 1) & 1, cta_abort, a.d_error,
                                                    22200))) {
                alive = false;
                break;
              }
              tc_fence_after();
              const float fa = __shfl_sync(0xffffffffu, f_lo, 4 * (lane & 7));
              const float fb = __shfl_sync(0xffffffffu, f_hi, 4 * (lane & 7));
              const float fr = (lane & 8) ? fb : fa; // of row lane % 16
#pragma unroll
              for (int c = 0; c < 8; ++c) {
                uint32_t orow[16];
                TMEM_LD_16((tm_o + 16u * c) | lane_sel, orow);
                tmem_wait_ld();
#pragma unroll
                for (int j = 0; j < 16; ++j) orow[j] = __float_as_uint(__uint_as_float(orow[j]) * fr);
                TMEM_ST_16((tm_o + 16u * c) | lane_sel, orow);
              }
              tmem_wait_st();
              tc_fence_before();
            }
          }
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const float2 n = *(const float2*)(tokc + kTok + 8 * k);
            const float p0 = ex2(__uint_as_float(sr[4 * k]) - ref_lo);
            const float p1 = ex2(__uint_as_float(sr[4 * k + 1]) - ref_lo);
            const float p2 = ex2(__uint_as_float(sr[4 * k + 2]) - ref_hi);
            const float p3 = ex2(__uint_as_float(sr[4 * k + 3]) - ref_hi);
            l_lo = fmaf(p0, n.x, fmaf(p1, n.y, l_lo));
            l_hi = fmaf(p2, n.x, fmaf(p3, n.y, l_hi));
            pk_lo[k] = f16x2(p0, p1);
            pk_hi[k] = f16x2(p2, p3);
          }
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) pk_lo[k] = pk_hi[k] = 0u;
        }
        // P takes the place of the tile before's, once that has been used
        if (T > 0 && !__all_sync(0xffffffffu, bar_wait(bar(BW_PVDONE), (T - 1) & 1, cta_abort, a.d_error,
                                                       22250))) {
          alive = false;
          break;
        }
        if (!idle) {
          const int r = warp * 16 + g8;              // (rows r and r + 8: the same swizzle)
          uint8_t* const p = bp + kOffP + r * 128;
          const uint32_t piece = (uint32_t)((r & 7) << 4 | 4 * qd);
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            *(uint32_t*)(p + (piece ^ (k << 4))) = pk_lo[k];
            *(uint32_t*)(p + (piece ^ (k << 4)) + 8 * 128) = pk_hi[k];
          }
          fence_async_smem();
        }
        tc_fence_before();
        __syncwarp();
        if (lane == 0) bar_arrive(bar(BW_PFULL));
        if (t == 0 && more) read_users(nxt);
      }
      if (!alive) break;
      if (!__all_sync(0xffffffffu, bar_wait(bar(BW_PVDONE), (T - 1) & 1, cta_abort, a.d_error, 22300)))
        break;
      tc_fence_after();
      if (!idle) {
#pragma unroll
        for (int d = 1; d <= 2; d <<= 1) {
          l_lo += __shfl_xor_sync(0xffffffffu, l_lo, d);
          l_hi += __shfl_xor_sync(0xffffffffu, l_hi, d);
        }
        // O in the layout of the scores: rows g8 and g8 + 8, columns 8 k + 2 qd and the next, i.e.
        // the dims of the same numbers with their last two bits xor'ed with the group's number
        uint8_t* dst[2];
        bool on[2], last[2];
        float inv[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int row = warp * 16 + g8 + 8 * e, slot = cur.user[e].slot;
          const int head = cur.head0 + row % G;
          on[e] = row < R;
          last[e] = slot < 0;
          inv[e] = last[e] ? 1.f / (e ? l_hi : l_lo) : 1.f;
          const size_t prow = (size_t)((last[e] ? 0 : slot) + cur.add) * HQ + head;
          dst[e] = last[e] ? (uint8_t*)a.out + ((size_t)cur.user[e].query * HQ + head) * (kDim * 2)
                           : (uint8_t*)(a.part_o + prow * kDim);
          if (on[e] && !last[e] && qd == 0)
            a.part_ml[prow] = e ? make_float2(ref_hi, l_hi) : make_float2(ref_lo, l_lo);
        }
#pragma unroll
        for (int GG = 0; GG < 4; ++GG) {             // columns n, n + 1 hold dims n ^ GG, (n + 1) ^ GG
          uint32_t o[16];
          TMEM_LD_16x256_32((tm_o + 32u * GG) | lane_sel, o);
          tmem_wait_ld();
#pragma unroll
          for (int e = 0; e < 2; ++e)
            if (on[e]) {
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                const int n = 32 * GG + 8 * k + ((2 * qd) ^ (GG & 2));
                const float x = __uint_as_float(o[4 * k + 2 * e + (GG & 1)]) * inv[e];
                const float y = __uint_as_float(o[4 * k + 2 * e + 1 - (GG & 1)]) * inv[e];
                if (last[e]) *(uint32_t*)(dst[e] + 2 * n) = pack2(x, y);
                else *(float2*)(dst[e] + 4 * n) = make_float2(x, y);
              }
            }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive(bar(BW_ODONE));
    }
  }
  // ---- common exit: every role arrives here, then the allocating warp frees TMEM
  tc_fence_before();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem),
                 "r"(kTmemColsW) : "memory");
  }
}

}  // namespace

cudaError_t launch_attention_q4_wide(const AttnArgs& a, int n_items, cudaStream_t st) {
  if (n_items <= 0) return cudaSuccess;
  const int64_t units = (int64_t)n_items * a.shape.num_kv_heads;
  if (units > INT32_MAX - (1 << 20)) return cudaErrorInvalidValue;
  static bool configured[64] = {};
  int dev = 0;
  cudaGetDevice(&dev);
  if (dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
  if (!configured[dev]) {
    cudaError_t e = cudaFuncSetAttribute(attn_q4_wide_kernel,
                                         cudaFuncAttributeMaxDynamicSharedMemorySize, kSmemWide);
    if (e != cudaSuccess) return e;
    configured[dev] = true;
  }
  const int ctas = (int)std::min<int64_t>(units, 2 * a.num_sms);
  attn_q4_wide_kernel<<<ctas, kThreads, kSmemWide, st>>>(a, (int)units);
  return cudaGetLastError();
}

}  // namespace apar
