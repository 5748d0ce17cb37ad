// The products of the losses over a large vocabulary, sm_103a: TMA tiles (128-byte swizzle) -> tcgen05.mma -> epilogues that
// reduce or transform the accumulator before it leaves the SM. Persistent and warp-specialised like the engine's products: warp
// 0 issues the copies, warp 1 the products (one thread), eight warps drain the accumulators (two TMEM buffers, so that a
// tile's epilogue runs under the next one's products); large products run on CTA pairs (256-row tiles, each CTA half of B).
// Three things differ from the engine's kernel: the tile width is chosen at run time, so that the tiles fill whole waves of SMs
// (the vocabulary rarely is a multiple of anything); an fp32 operand takes part as three bf16 terms, the products of the
// terms being further k blocks (or, DIRECT, further products of a k block whose B is cut in the kernel); and epilogues gather a row's
// share in registers first. Every wait is bounded; where one gives up, what is not formed is NaN.
// Bound by the tensor cores, few rows by the reading of B. Measured: 2048 x 4096 x 32000 bf16 287 to 296 us (the burst peak's 284), 4096 x
// 768 x 50257 198 us reduced to log-sum-exps (84%), 86 us a piece of 16768 columns as dz (65%), 8 x 768 x 50257 18 us (4.3 TB/s); 203 x
// 768 x 50257 fp32 straight from W 112 us, its cutting warps waiting for their loads (the three DIRECT kernels have 96 registers a thread and
// spill 60 to 148 bytes of stores; the others none).
#include <algorithm>

#include "common.cuh"
#include "ops.h"
#include "per_device.h"
#include "tc_host.h"
#include "tcgen05.cuh"
#include "vocab.cuh"
#include "vocab_gemm.cuh"

namespace zl {
namespace vocab {
namespace {

using namespace zl::tc;

constexpr int BM = 128, BK = 64;
// Warpgroup 0 (copies, products, two idle warps) hands registers to the two epilogue warpgroups, whose threads hold half a row of a
// tile: of the launch's 384 x 168 they get 224 each (at 168 every epilogue spilled 40 to 236 bytes).
constexpr int kEpiWarps = 8, kThreads = 128 + 32 * kEpiWarps;
constexpr int kRegsLow = 56, kRegsEpi = 224;
static_assert(128 * kRegsLow + 32 * kEpiWarps * kRegsEpi <= kThreads * 168, "register split above the pool");
constexpr int kStageSpace = 6 * 32768;            // operand stages: as many as fit
constexpr int kOutBytes = kEpiWarps * 32 * 128;   // one box of 32 rows x 128 bytes a warp
constexpr int kSmem = kStageSpace + kOutBytes + 1024 + 256;
constexpr int kMaxStages = 12;
static_assert(kSmem <= 232448, "shared memory per CTA");
// Products straight from an fp32 B (DIRECT): eight more warps read it, cut it into its terms and write them as the copies would. 128
// columns, one CTA a tile; a stage holds three terms of both operands, whose six products go to two accumulators.
constexpr int kCutWarps = 8, kThreadsDirect = kThreads + 32 * kCutWarps, kDirectN = 128;
constexpr int kRegsEpiDirect = 120, kRegsCut = 88;
static_assert(128 * kRegsLow + 32 * kEpiWarps * kRegsEpiDirect + 32 * kCutWarps * kRegsCut <= kThreadsDirect * 96, "register split above the pool");

// The pairs of terms (a, b) of an fp32 product, two bits each, smallest products first: (l, h) (h, l) (m, m) (m, h) (h, m) (h, h).
constexpr uint32_t pair_table(bool b) {
  const int a[kPairs] = {2, 0, 1, 1, 0, 0}, bb[kPairs] = {0, 2, 1, 0, 1, 0};
  uint32_t t = 0;
  for (int i = 0; i < kPairs; ++i) t |= (uint32_t)(b ? bb[i] : a[i]) << (2 * i);
  return t;
}

struct Args {
  const float* Bf;                   // DIRECT: B [b_rows, ldb]
  int b_rows, ldb;
  int M, N, nk1, nk;                 // rows, columns; k blocks of one pair of terms and of all
  int bn, stages, a_bytes, b_bytes;  // tile width, stages, bytes of a stage's parts (of one CTA)
  int tiles_m, tiles_n, group_m;
  int splits, kb_per_split, kb_per_seg, kb_small;   // kb_small: k blocks of the smaller pairs of terms
  uint32_t pair_a, pair_b;           // pair tables
  int a_term, b_term, b_first;       // rows between terms, first row of B
  // kLse
  const int32_t* labels;
  float2* part;
  float* zl;
  unsigned* counter;
  // kGradZ
  const float* lse;
  int first, V, rows_p, ldz, terms;
  // kOut16, kOut32
  void* C;
  int add;
  const float *omega, *dloss;        // C times loss_weight() (omega NULL: 1)
};

// The end of the accumulation that begins with k block kb. The smaller pairs of terms share one: their sums, and what is cut off
// them, are 2^-8 of the others'.
__device__ __forceinline__ int seg_end(const Args& g, int kb, int kbe) {
  return min(kbe, kb < g.kb_small ? g.kb_small : kb + g.kb_per_seg);
}

// A tile row group sweeps the tile columns (tiles of B are read once, A stays in L2).
__device__ __forceinline__ void unit_tile(const Args& g, int unit, int num_tiles, bool pair, uint32_t crank, int& tm, int& tn) {
  const int tiles_m = pair ? (g.tiles_m + 1) / 2 : g.tiles_m;
  const int tile = unit % num_tiles, per_group = g.group_m * g.tiles_n;
  const int gid = tile / per_group, first = gid * g.group_m;
  const int gm = min(tiles_m - first, g.group_m), r = tile % per_group;
  tm = first + r % gm;
  tn = r / gm;
  if (pair) tm = 2 * tm + (int)crank;
}

template <bool A_MN, bool B_MN, int KIND, bool PAIR, bool DIRECT>
__global__ void __launch_bounds__(DIRECT ? kThreadsDirect : kThreads, 1)
    vocab_gemm_k(const __grid_constant__ CUtensorMap ta, const __grid_constant__ CUtensorMap tb,
                 const __grid_constant__ CUtensorMap tcm, const Args g) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  uint8_t* outbuf = smem + kStageSpace;
  uint64_t* full = (uint64_t*)(outbuf + kOutBytes);
  uint64_t* empty = full + kMaxStages;
  uint64_t* tfull = empty + kMaxStages;
  uint64_t* tempty = tfull + 2;
  uint64_t* fin = tempty + 2;
  uint32_t* tbase = (uint32_t*)(fin + 1);
  volatile int* abort_flag = (volatile int*)(tbase + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  static_assert(!DIRECT || (!PAIR && !A_MN), "direct products: one CTA, A as rows");
  const int a_all = (DIRECT ? kTerms : 1) * g.a_bytes, stage_bytes = a_all + g.b_bytes;
  if (threadIdx.x == 0) {
    for (int s = 0; s < g.stages; ++s) { mbar_init(&full[s], 1 + (DIRECT ? kCutWarps : 0)); mbar_init(&empty[s], 1); }
    for (int a = 0; a < 2; ++a) { mbar_init(&tfull[a], 1); mbar_init(&tempty[a], kEpiWarps * (PAIR ? 2 : 1)); }
    mbar_init(fin, 1);
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 2 && lane < 3) prefetch_map(lane == 0 ? &ta : lane == 1 ? &tb : &tcm);
  if (warp == 1) {
    if constexpr (PAIR) {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(su32(tbase)), "r"(512u) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    } else {
      asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(su32(tbase)), "r"(512u) : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
  }
  fence_before();
  __syncthreads();
  fence_after();
  if (PAIR) cluster_sync();   // both CTAs' barriers exist before anything is issued
  const uint32_t crank = PAIR ? cluster_rank() : 0u;
  const int unit0 = PAIR ? (int)(blockIdx.x >> 1) : (int)blockIdx.x;
  const int ustride = PAIR ? (int)(gridDim.x >> 1) : (int)gridDim.x;
  const uint32_t tmem = *tbase;
  const uint32_t tempty_addr = PAIR ? cluster_addr(tempty, 0) : 0u;
  pdl_wait();
  pdl_trigger();
  const int num_tiles = (PAIR ? (g.tiles_m + 1) / 2 : g.tiles_m) * g.tiles_n;
  const int num_units = num_tiles * g.splits;

  if (warp < 4) {
    regs_dec<kRegsLow>();
    if (warp == 0) {
      // ---------------- copies ----------------
      const bool leader = elect_one();
      const int bw = PAIR ? g.bn / 2 : g.bn, boxes = (bw + 63) / 64;
      int stage = 0;
      uint32_t phase = 0, used = 0, last = 0;   // bit s: stage s was filled; the parity of its last fill
      bool ok = true;
      for (int unit = unit0; ok && unit < num_units; unit += ustride) {
        int tm, tn;
        unit_tile(g, unit, num_tiles, PAIR, crank, tm, tn);
        const int kb0 = (unit / num_tiles) * g.kb_per_split, kb1 = min(g.nk, kb0 + g.kb_per_split);
        int pr = kb0 / g.nk1, kk = kb0 - pr * g.nk1;
        const int n0 = tn * g.bn + (PAIR ? (int)crank * bw : 0);
        for (int kb = kb0; kb < kb1; ++kb) {
          if (!uwait(&empty[stage], phase ^ 1u, abort_flag, nullptr)) { ok = false; break; }
          used |= 1u << stage;
          last = (last & ~(1u << stage)) | phase << stage;
          if (leader) {
            uint8_t* sa = smem + stage * stage_bytes;
            uint8_t* sb = sa + a_all;
            const int k0 = kk * BK;
            const int ra = (int)(g.pair_a >> (2 * pr) & 3u) * g.a_term, rb = (int)(g.pair_b >> (2 * pr) & 3u) * g.b_term + g.b_first;
            if constexpr (PAIR) {   // on the first CTA's barrier
              if (crank == 0) mbar_expect_tx(&full[stage], 2 * stage_bytes);
              const uint32_t bar = cluster_addr(&full[stage], 0);
              if (!A_MN) {
                tma2d_pair(sa, &ta, bar, k0, ra + tm * BM);
              } else {
                tma2d_pair(sa, &ta, bar, tm * BM, ra + k0);
                tma2d_pair(sa + 8192, &ta, bar, tm * BM + 64, ra + k0);
              }
              if (!B_MN) tma2d_pair(sb, &tb, bar, k0, rb + n0);
              else
                for (int j = 0; j < boxes; ++j) tma2d_pair(sb + j * 8192, &tb, bar, n0 + 64 * j, rb + k0);
            } else if constexpr (DIRECT) {
              mbar_expect_tx(&full[stage], a_all);
              for (int t = 0; t < kTerms; ++t) tma2d(sa + t * g.a_bytes, &ta, &full[stage], k0, t * g.a_term + tm * BM);
            } else {
              mbar_expect_tx(&full[stage], stage_bytes);
              if (!A_MN) {
                tma2d(sa, &ta, &full[stage], k0, ra + tm * BM);
              } else {
                tma2d(sa, &ta, &full[stage], tm * BM, ra + k0);
                tma2d(sa + 8192, &ta, &full[stage], tm * BM + 64, ra + k0);
              }
              if (!B_MN) tma2d(sb, &tb, &full[stage], k0, rb + n0);
              else
                for (int j = 0; j < boxes; ++j) tma2d(sb + j * 8192, &tb, &full[stage], n0 + 64 * j, rb + k0);
            }
          }
          __syncwarp();
          if (++stage == g.stages) { stage = 0; phase ^= 1u; }
          if (++kk == g.nk1) { kk = 0; ++pr; }
        }
      }
      if (PAIR && ok) {   // no copy and no arrival is still on its way when the CTAs exit
        for (int s = 0; s < g.stages; ++s)
          if ((used >> s & 1u) && !uwait(&empty[s], last >> s & 1u, abort_flag, nullptr)) break;
      }
      if (!ok && lane == 0) {   // unwinding: the copies in flight land first
        for (int s = 0; s < g.stages; ++s) {
          if (!(used >> s & 1u)) continue;
          const unsigned long long t0 = gtimer();   // (a pair's second CTA has no barrier of its own to test: 10 ms)
          while ((PAIR && crank != 0) ? gtimer() - t0 < 10000000ull
                                      : (!mbar_test(&full[s], last >> s & 1u) && gtimer() - t0 < 100000000ull)) {
          }
        }
      }
    } else if (warp == 1) {
      // ---------------- products (of a pair: the first CTA's thread, for both) ----------------
      const uint32_t id = idesc_f16(PAIR ? 2 * BM : BM, 0, A_MN, B_MN) | (uint32_t)(g.bn >> 3) << 17;
      const bool leader = elect_one();
      int stage = 0, it = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int unit = unit0; (!PAIR || crank == 0) && ok && unit < num_units; unit += ustride) {
        int kb0 = (unit / num_tiles) * g.kb_per_split;
        const int kbe = min(g.nk, kb0 + g.kb_per_split);
        for (; ok && kb0 < kbe; ++it) {   // one accumulation after another
          const int kb1 = seg_end(g, kb0, kbe);
          const int acc = it & 1;
          if (!uwait(&tempty[acc], ((uint32_t)(it >> 1) & 1u) ^ 1u, abort_flag, nullptr)) { ok = false; break; }
          fence_after();
          const uint32_t d = tmem + (uint32_t)(acc * 256);
          for (int kb = kb0; kb < kb1; ++kb) {
            if (!uwait(&full[stage], phase, abort_flag, nullptr)) { ok = false; break; }
            fence_after();
            if (leader) {
              const uint32_t a0 = su32(smem + stage * stage_bytes), b0 = a0 + a_all;
            if constexpr (DIRECT) {   // the largest pair of terms into d, the others into d + kDirectN
#pragma unroll 1
              for (int p = 0; p < kPairs; ++p) {
                const uint32_t at = a0 + (pair_table(false) >> (2 * p) & 3u) * g.a_bytes, bt = b0 + (pair_table(true) >> (2 * p) & 3u) * 16384u;
                const bool top = p == kPairs - 1;
#pragma unroll
                for (int kk = 0; kk < BK / 16; ++kk) {
                  const uint64_t bd = B_MN ? sdesc(bt + kk * 2048, 8192, 1024) : sdesc(bt + kk * 32, 16, 1024);
                  const uint32_t on = kb > kb0 || kk > 0 || (p > 0 && !top) ? 1u : 0u;
                  mma_bf16(top ? d : d + kDirectN, sdesc(at + kk * 32, 16, 1024), bd, id, on);
                }
              }
            } else {
#pragma unroll
              for (int kk = 0; kk < BK / 16; ++kk) {
                const uint64_t ad = A_MN ? sdesc(a0 + kk * 2048, 8192, 1024) : sdesc(a0 + kk * 32, 16, 1024);
                const uint64_t bd = B_MN ? sdesc(b0 + kk * 2048, 8192, 1024) : sdesc(b0 + kk * 32, 16, 1024);
                const uint32_t on = (kb > kb0 || kk > 0) ? 1u : 0u;
                if (PAIR) mma_bf16_pair(d, ad, bd, id, on);
                else mma_bf16(d, ad, bd, id, on);
              }
            }
              if (PAIR) mma_commit_pair(&empty[stage]);
              else mma_commit(&empty[stage]);
            }
            __syncwarp();
            if (++stage == g.stages) { stage = 0; phase ^= 1u; }
          }
          if (ok && leader) {
            if (PAIR) mma_commit_pair(&tfull[acc]);
            else mma_commit(&tfull[acc]);
          }
          __syncwarp();
          kb0 = kb1;
        }
      }
      if (leader) {   // completes before TMEM is released
        if (!PAIR) mma_commit(fin);
        else if (crank == 0) mma_commit_pair(fin);
      }
      __syncwarp();
    }
  } else if (DIRECT && warp >= 4 + kEpiWarps) {
    // ---------------- terms of B: line l of a tile is 64 values of a row (B_MN: of row l % 64, columns 64 (l / 64) on) ----------------
    // Sixteen threads a line, eight lines a thread; two k blocks' values are under way.
    regs_dec<kRegsCut>();
    const int t = threadIdx.x - (128 + 32 * kEpiWarps), c4 = t & 15, l0 = t >> 4;
    struct At {
      int unit, kb, kbe, n0;
    };
    auto begin = [&](At& a) {   // the first k block of its unit, or of the next that has one
      for (; a.unit < num_units; a.unit += ustride) {
        int tm;
        unit_tile(g, a.unit, num_tiles, false, 0u, tm, a.n0);
        a.n0 *= g.bn;
        a.kb = (a.unit / num_tiles) * g.kb_per_split;
        a.kbe = min(g.nk, a.kb + g.kb_per_split);
        if (a.kb < a.kbe) return;
      }
    };
    auto next = [&](At& a) {
      if (++a.kb < a.kbe) return;
      a.unit += ustride;
      begin(a);
    };
    auto load = [&](const At& a, float4 (&r)[8]) {
      if (a.unit >= num_units) return;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int l = l0 + 16 * i;
        const int row = g.b_first + (B_MN ? a.kb * BK + (l & 63) : a.n0 + l);
        const int col = (B_MN ? a.n0 + (l & 64) : a.kb * BK) + 4 * c4;
        r[i] = row < g.b_rows && col < g.ldb ? __ldg(reinterpret_cast<const float4*>(g.Bf + (size_t)row * g.ldb + col)) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
    };
    int stage = 0;
    uint32_t phase = 0;
    auto cut = [&](float4 (&r)[8]) {
      if (!uwait(&empty[stage], phase ^ 1u, abort_flag, nullptr)) return false;
      uint8_t* const sb = smem + stage * stage_bytes + a_all;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int l = l0 + 16 * i;
        uint8_t* const at = sb + l * 128 + (((c4 >> 1) ^ (l & 7)) << 4) + (c4 & 1) * 8;
        float x[4] = {r[i].x, r[i].y, r[i].z, r[i].w};
#pragma unroll
        for (int k = 0; k < kTerms; ++k) {
          uint32_t h[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            h[e] = __float_as_uint(x[e]) & 0xffff0000u;
            x[e] -= __uint_as_float(h[e]);   // (an infinity becomes NaN)
          }
          *reinterpret_cast<uint2*>(at + k * 16384) = make_uint2(h[0] >> 16 | h[1], h[2] >> 16 | h[3]);
        }
      }
      fence_async_smem();
      __syncwarp();
      if (lane == 0) mbar_arrive(&full[stage]);
      if (++stage == g.stages) { stage = 0; phase ^= 1u; }
      return true;
    };
    At a{unit0, 0, 0, 0};
    begin(a);
    float4 r0[8], r1[8];
    At b = a;
    load(a, r0);
    if (b.unit < num_units) next(b);
    load(b, r1);
    while (a.unit < num_units) {
      if (!cut(r0)) break;
      a = b;
      if (a.unit >= num_units) break;
      next(a);
      load(a, r0);
      if (!cut(r1)) break;
      b = a;
      if (b.unit >= num_units) break;
      next(b);
      load(b, r1);
    }
  } else {
    if constexpr (DIRECT) regs_inc<kRegsEpiDirect>();
    else regs_inc<kRegsEpi>();
    // ---------------- epilogues: one accumulator row a thread, the two warps of a lane quadrant take chunks in turn ----------------
    // A thread first gathers its share of the tile's row in registers, summing the accumulations in fp32 (rounded to nearest: the
    // tensor cores cut off what does not fit as they add), and hands TMEM back before it works on the values.
    constexpr int NV = DIRECT ? 64 : 128;   // columns of a thread
    constexpr int CH = KIND == kLse || KIND == kOut32 ? 32 : 64, NJ = NV / CH;   // columns of a chunk, chunks of a warp
    const int q = warp & 3, half = (warp - 4) >> 2;
    uint8_t* const sbuf = outbuf + (warp - 4) * (32 * 128);
    uint8_t* const srow = sbuf + lane * 128;
    const float nan = __uint_as_float(0x7FC00000u);
    int it = 0, unit = unit0;
    bool ok = true;
    float v[NV];
    auto gather = [&](int kb0, int kbe) {
      for (int kb = kb0; kb < kbe; kb = seg_end(g, kb, kbe), ++it) {
        int w = 1;
        if (lane == 0) w = mbar_wait(&tfull[it & 1], (uint32_t)(it >> 1) & 1u, abort_flag, nullptr) ? 1 : 0;
        if (!__shfl_sync(0xffffffffu, w, 0)) return false;
        fence_after();
        const uint32_t trow = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)((it & 1) * 256);
#pragma unroll
        for (int j = 0; j < NV / 32; ++j) {
          const int c = CH == 32 ? 32 * (half + 2 * j) : 64 * (half + 2 * (j >> 1)) + 32 * (j & 1);
          if (c < g.bn) {
            if constexpr (DIRECT) {   // the largest pair of terms, then the smaller ones, 16 columns at a time (registers)
#pragma unroll
              for (int h = 0; h < 4; ++h) {
                float t[16];
                tmem_ld16(trow + (uint32_t)((h & 1) * kDirectN + c + 16 * (h >> 1)), t);
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                  float& x = v[32 * j + 16 * (h >> 1) + e];
                  x = (h & 1) == 0 && kb == kb0 ? t[e] : x + t[e];
                }
              }
            } else if (kb == kb0) {
              tmem_ld32(trow + (uint32_t)c, v + 32 * j);
            } else {
              float t[32];
              tmem_ld32(trow + (uint32_t)c, t);
#pragma unroll
              for (int e = 0; e < 32; ++e) v[32 * j + e] += t[e];
            }
          }
        }
        fence_before();
        __syncwarp();
        if (lane == 0) {
          if (PAIR) mbar_arrive_cluster(tempty_addr + 8u * (uint32_t)(it & 1));
          else mbar_arrive(&tempty[it & 1]);
        }
      }
      return true;
    };
    if constexpr (KIND == kLse) {
      if (blockIdx.x == 0 && threadIdx.x == 128) *g.counter = 0u;
      for (; unit < num_units; unit += ustride) {
        int tm, tn;
        unit_tile(g, unit, num_tiles, PAIR, crank, tm, tn);
        const int m = tm * BM + q * 32 + lane, n0 = tn * g.bn;
        const int y = m < g.M ? g.labels[m] : -1;
        if (!(ok = gather(0, g.nk))) break;
        Lse A = lse_empty();
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const int c = 32 * (half + 2 * j);
          const int nv = min(g.bn - c, g.N - n0 - c);   // columns of the tile and of the vocabulary
          if (nv <= 0) continue;
          float (&x)[32] = *reinterpret_cast<float (*)[32]>(&v[32 * j]);
          if (nv < 32) {
#pragma unroll
            for (int e = 0; e < 32; ++e) x[e] = e < nv ? x[e] : -INFINITY;
          }
          const int e0 = y - n0 - c;
          if (e0 >= 0 && e0 < nv && e0 < 32) {
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (e == e0) g.zl[m] = x[e];
          }
          float mx = x[0];
#pragma unroll
          for (int e = 1; e < 32; ++e) mx = fmaxf(mx, x[e]);
          lse_add(A, x, mx, kL2e);
        }
        if (m < g.M) g.part[(size_t)m * (2 * g.tiles_n) + 2 * tn + half] = make_float2(A.m, A.s);
      }
#pragma unroll 1
      for (; !ok && unit < num_units; unit += ustride) {
        int tm, tn;
        unit_tile(g, unit, num_tiles, PAIR, crank, tm, tn);
        const int m = tm * BM + q * 32 + lane;
        if (m < g.M) g.part[(size_t)m * (2 * g.tiles_n) + 2 * tn + half] = make_float2(nan, nan);
      }
    } else {
      const float weight = KIND != kGradZ && g.omega ? loss_weight(g.omega, g.dloss) : 1.f;
      const int rows = KIND == kGradZ ? g.rows_p : g.M, cols = KIND == kGradZ ? g.ldz : g.N;   // of the output
      for (; unit < num_units; unit += ustride) {
        int tm, tn;
        unit_tile(g, unit, num_tiles, PAIR, crank, tm, tn);
        const int split = unit / num_tiles, row0 = tm * BM + q * 32, m = row0 + lane, n0 = tn * g.bn;
        const int kb0 = split * g.kb_per_split, kbe = min(g.nk, kb0 + g.kb_per_split);
        if (kb0 >= kbe) continue;   // (a shorter last piece of the vocabulary)
        int y = -1;
        float l = 0.f;
        if (KIND == kGradZ && m < g.M) {   // under way while the accumulator is waited for
          y = g.labels[m];
          l = g.lse[m];
        }
        if (!(ok = gather(kb0, kbe))) break;
        const bool on = y >= 0 && y < g.V;
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const int c = CH * (half + 2 * j);
          if (c >= g.bn) continue;
          float* const x = v + CH * j;
          if constexpr (KIND == kGradZ) {
            const int nv = g.V - g.first - n0 - c, e0 = y - g.first - n0 - c;
            const uint64_t l2 = f2(-l, -l), k2 = f2(kL2e, kL2e);
#pragma unroll
            for (int e = 0; e < CH; e += 2) {   // (the difference first: it is exact where p is near 1)
              const float2 d = uf2(mul2(add2(f2(x[e], x[e + 1]), l2), k2));
              x[e] = ex2(d.x);
              x[e + 1] = ex2(d.y);
            }
            if (e0 >= 0 && e0 < CH) {
#pragma unroll
              for (int e = 0; e < CH; ++e) x[e] -= e == e0 ? 1.f : 0.f;
            }
            if (nv < CH || __any_sync(0xffffffffu, !on)) {   // columns past the vocabulary, rows outside Omega
#pragma unroll
              for (int e = 0; e < CH; ++e) x[e] = on && e < nv ? x[e] : 0.f;
            }
          }
          if (KIND != kGradZ && g.omega) {
#pragma unroll
            for (int e = 0; e < CH; ++e) x[e] *= weight;
          }
          if constexpr (KIND == kGradZ) {
            // straight to memory, 32 bytes (a whole sector) at a time: staged for a bulk copy, the fences between the proxies and the
            // waits for the buffer made the epilogue longer than the products of K = 768 (58 us a piece of 12608 x 4096)
            if (m >= rows || n0 + c >= cols) continue;
            bf16* out = (bf16*)g.C + (size_t)m * cols + n0 + c;
            for (int t = 0; t < g.terms; ++t, out += (size_t)rows * cols) {
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                uint32_t h[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                  float* const y2 = x + 16 * k + 2 * e;
                  if (g.terms > 1) {   // the leading bits, the remainder stays
                    const uint32_t b0 = __float_as_uint(y2[0]) & 0xffff0000u, b1 = __float_as_uint(y2[1]) & 0xffff0000u;
                    h[e] = b0 >> 16 | b1;
                    y2[0] -= __uint_as_float(b0);
                    y2[1] -= __uint_as_float(b1);
                  } else {
                    const __nv_bfloat162 b = __floats2bfloat162_rn(y2[0], y2[1]);
                    h[e] = *reinterpret_cast<const uint32_t*>(&b);
                  }
                }
                asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + 16 * k), "r"(h[0]), "r"(h[1]), "r"(h[2]),
                             "r"(h[3]), "r"(h[4]), "r"(h[5]), "r"(h[6]), "r"(h[7])
                             : "memory");
              }
            }
          } else {
            if (lane == 0) bulk_wait_read0();   // the store before has read the buffer
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              uint4 u;
              if constexpr (CH == 32) {
                u = make_uint4(__float_as_uint(x[4 * k]), __float_as_uint(x[4 * k + 1]), __float_as_uint(x[4 * k + 2]),
                               __float_as_uint(x[4 * k + 3]));
              } else {
                u = pack_word(*reinterpret_cast<const float (*)[8]>(x + 8 * k));
              }
              *reinterpret_cast<uint4*>(srow + ((k ^ (lane & 7)) << 4)) = u;
            }
            fence_async_smem();
            __syncwarp();
            if (lane == 0) {
              if (row0 < rows && n0 + c < cols) {
                if (KIND == kOut32 && g.add) tma_reduce_add3d(&tcm, sbuf, n0 + c, row0, split);
                else tma_store3d(&tcm, sbuf, n0 + c, row0, split);
              }
              bulk_commit();
            }
          }
        }
      }
      if (lane == 0) bulk_wait_all();
      __syncwarp();
#pragma unroll 1
      for (; !ok && unit < num_units; unit += ustride) {
        int tm, tn;
        unit_tile(g, unit, num_tiles, PAIR, crank, tm, tn);
        const int m = tm * BM + q * 32 + lane;
        if (m >= rows) continue;
        const size_t at = ((size_t)(unit / num_tiles) * rows + m) * cols;
        for (int c = CH * half; c < g.bn; c += 2 * CH)
          for (int e = 0; e < CH && tn * g.bn + c + e < cols; ++e) {
            if (CH == 32) ((float*)g.C)[at + tn * g.bn + c + e] = nan;
            else ((bf16*)g.C)[at + tn * g.bn + c + e] = __float2bfloat16_rn(nan);
          }
      }
    }
  }

  __syncthreads();
  if (warp == 1) {
    if (lane == 0) {   // (bounded) the final commit
      const unsigned long long t0 = gtimer();
      while (!mbar_test(fin, 0) && gtimer() - t0 < 100000000ull) {
      }
    }
    __syncwarp();
  }
  if (PAIR) {   // neither CTA leaves while the other may still use its shared memory
    __syncthreads();
    cluster_sync();
  }
  if (warp == 1) {
    fence_after();
    if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
  }
}

// ------------------------------------------------------------------------------------------------
// host side
// ------------------------------------------------------------------------------------------------
bool map2d(CUtensorMap* m, const void* p, uint64_t inner, uint64_t outer, uint64_t pitch, uint32_t box_outer) {
  cuuint64_t dims[2] = {inner, outer};
  cuuint64_t strides[1] = {pitch * 2};
  cuuint32_t box[2] = {64, box_outer};
  cuuint32_t es[2] = {1, 1};
  return g_encode(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                  CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool map_out(CUtensorMap* m, void* p, bool f32, uint64_t cols, uint64_t rows, uint64_t slices) {
  const uint64_t esz = f32 ? 4 : 2;
  cuuint64_t dims[3] = {cols, rows, slices};
  cuuint64_t strides[2] = {cols * esz, rows * cols * esz};
  cuuint32_t box[3] = {f32 ? 32u : 64u, 32u, 1u};
  cuuint32_t es[3] = {1, 1, 1};
  return g_encode(m, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, p, dims, strides, box, es,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <bool A_MN, bool B_MN, int KIND, bool PAIR, bool DIRECT = false>
bool launch(const Args& a, const CUtensorMap& ta, const CUtensorMap& tb, const CUtensorMap& tcm, cudaStream_t s) {
  struct Ready {
    int max_pairs = 0;
  };
  static PerDevice<Ready> devices;
  auto kern = vocab_gemm_k<A_MN, B_MN, KIND, PAIR, DIRECT>;
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  const Ready* const ready = devices.get(dev, [&](Ready& r) {
    cudaFuncAttributes fa;   // the register split must fit the pool that the CTA is launched with
    constexpr int need = 128 * kRegsLow + 32 * kEpiWarps * (DIRECT ? kRegsEpiDirect : kRegsEpi) + (DIRECT ? 32 * kCutWarps * kRegsCut : 0);
    if (cudaFuncGetAttributes(&fa, kern) != cudaSuccess || need > (DIRECT ? kThreadsDirect : kThreads) * fa.numRegs ||
        (DIRECT && fa.numRegs > 96)) {
      cudaGetLastError();
      return false;
    }
    if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem) != cudaSuccess) return false;
    if (PAIR) {
      cudaLaunchConfig_t oc = {};
      oc.gridDim = dim3(2u * (unsigned)g_sms);
      oc.blockDim = dim3(kThreads);
      oc.dynamicSmemBytes = kSmem;
      cudaLaunchAttribute ca[1];
      ca[0].id = cudaLaunchAttributeClusterDimension;
      ca[0].val.clusterDim.x = 2;
      ca[0].val.clusterDim.y = 1;
      ca[0].val.clusterDim.z = 1;
      oc.attrs = ca;
      oc.numAttrs = 1;
      if (cudaOccupancyMaxActiveClusters(&r.max_pairs, kern, &oc) != cudaSuccess || r.max_pairs < 1) {
        cudaGetLastError();
        return false;
      }
    }
    return true;
  });
  if (!ready) return false;
  const int units = (PAIR ? (a.tiles_m + 1) / 2 : a.tiles_m) * a.tiles_n * a.splits;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(PAIR ? 2 * std::min(units, ready->max_pairs) : std::min(units, g_sms)));
  cfg.blockDim = dim3(DIRECT ? kThreadsDirect : kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = 2;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = PAIR ? 2 : 1;
  note_launch(1);
  return cudaLaunchKernelEx(&cfg, kern, ta, tb, tcm, a) == cudaSuccess;
}

// Fills in what every product has and encodes its operands' maps.
bool prepare(Args& a, CUtensorMap& ta, CUtensorMap& tb, int M, int N, int K, const Operands& o, const Tiles& t) {
  if (!init()) return false;
  a.M = M;
  a.N = N;
  a.nk1 = (K + BK - 1) / BK;
  a.nk = a.nk1 * (o.terms == kTerms && !o.direct ? kPairs : 1);
  a.bn = t.bn;
  const int bw = t.pair ? t.bn / 2 : t.bn;
  a.b_bytes = (o.b_mn ? (bw + 63) / 64 * 64 : bw) * BK * 2;
  // Fewer than 128 rows: only they are copied (the products read on into B's part, rows of the result that nobody reads).
  const int box_a = o.a_mn ? BM : std::min(BM, (M + 7) / 8 * 8);
  a.a_bytes = box_a * BK * 2;
  if (o.direct) a.b_bytes = kTerms * kDirectN * BK * 2;
  a.stages = std::min(kMaxStages, kStageSpace / ((o.direct ? kTerms : 1) * a.a_bytes + a.b_bytes));
  a.tiles_m = (M + BM - 1) / BM;
  a.tiles_n = (N + t.bn - 1) / t.bn;
  // one group of every tile row (each tile of B fetched once) when A fits well inside L2 or is the smaller operand
  const double ab = 2.0 * M * a.nk * BK, bb = 2.0 * N * a.nk * BK;
  a.group_m = (ab <= 48e6 || ab <= bb) ? a.tiles_m : std::min(8, a.tiles_m);
  if (t.pair) a.group_m = (a.group_m + 1) / 2;
  a.kb_per_split = t.kb_per_split;
  a.splits = t.splits;
  a.kb_per_seg = t.kb_per_seg;
  a.kb_small = o.terms == kTerms && !o.direct ? (kPairs - 1) * a.nk1 : 0;
  a.pair_a = o.terms == kTerms ? pair_table(false) : 0u;
  a.pair_b = o.terms == kTerms ? pair_table(true) : 0u;
  a.a_term = o.a_term;
  a.b_term = o.b_term;
  a.b_first = o.b_first;
  const bool okA = o.a_mn ? map2d(&ta, o.A, (uint64_t)M, (uint64_t)o.a_rows, (uint64_t)o.lda, 64)
                          : map2d(&ta, o.A, (uint64_t)K, (uint64_t)o.a_rows, (uint64_t)o.lda, (uint32_t)box_a);
  a.Bf = (const float*)o.B;
  a.b_rows = o.b_rows;
  a.ldb = o.ldb;
  if (o.direct) {
    tb = ta;   // (not used)
    return okA;
  }
  const bool okB = o.b_mn ? map2d(&tb, o.B, (uint64_t)N, (uint64_t)o.b_rows, (uint64_t)o.ldb, 64)
                          : map2d(&tb, o.B, (uint64_t)K, (uint64_t)o.b_rows, (uint64_t)o.ldb, (uint32_t)bw);
  return okA && okB;
}

}  // namespace

// The tiling with the least predicted time: waves of units on 152 SMs (76 pairs), a k block of a unit at a rate linear in the
// tile's width (fitted to the engine's kernels of widths 64 to 256) and no faster than HBM delivers its part of B, a tile no
// shorter than its epilogue.
Tiles plan_direct(int M, int N, int K, int seg, int max_splits, int runs) {
  init();
  const int sms = g_sms > 0 ? g_sms : 152, nk = (K + BK - 1) / BK;
  const long tm = (M + BM - 1) / BM, tiles = tm * ((N + kDirectN - 1) / kDirectN);
  Tiles best{};
  best.us = 1e30;
  for (int sp = 1; sp <= max_splits; ++sp) {
    if (sp > 1 && (nk / sp < 4 || tiles * sp > 4l * sms)) break;
    const int kps = (nk + sp - 1) / sp;
    if ((nk + kps - 1) / kps != sp) continue;
    // six products of 128 x 128 x 64, which the terms' way into shared memory shares with
    double us = 4.0 + (double)((tiles * sp + sms - 1) / sms) * (kps * 1.2 + 0.5) + 1.0;
    if (sp > 1) us += (8.0 * (sp - 1) * M * (double)N / 6e6 + 2.0) / runs;
    if (us < best.us * 0.995) best = Tiles{kDirectN, 0, sp, kps, seg, us};
  }
  return best;
}
Tiles plan(Kind kind, int M, int N, int K, int terms, int out_step, int seg, int max_splits, int runs) {
  init();   // (its SM count)
  const int sms = g_sms > 0 ? g_sms : 152;
  const int nk = (K + BK - 1) / BK * (terms == kTerms ? kPairs : 1);
  const long tm = (M + BM - 1) / BM;
  Tiles best{};
  best.us = 1e30;
  for (int pair = M > BM ? 1 : 0; pair >= 0; --pair) {
    const long rows = pair ? (tm + 1) / 2 : tm, slots = pair ? sms / 2 : sms;
    const int step = std::max(out_step, pair ? 32 : 16);
    for (int bn = 256; bn >= step; bn -= step) {
      if (bn % step) { bn -= bn % step; }
      const long tiles = rows * ((N + bn - 1) / bn);
      const double hbm = 128.0 * bn * (double)slots / (double)std::min(rows, slots) / 6.3e6;
      const double kb = std::max((pair ? 0.105 + 0.00074 * bn : 0.13 + 0.00086 * bn) * (kind >= kOut16 ? 1.05 : 1.0), hbm);
      const double epi = kind == kLse ? 0.4 + 0.005 * bn : kind == kGradZ ? 0.5 + 0.008 * bn * terms : 0.4 + 0.006 * bn;
      for (int sp = 1; sp <= max_splits; ++sp) {
        if (sp > 1 && (nk / sp < 8 || tiles * sp > 4 * slots)) break;
        const int kps = (nk + sp - 1) / sp;
        if ((nk + kps - 1) / kps != sp) continue;   // no empty split
        const long waves = (tiles * sp + slots - 1) / slots;
        double us = 2.8 + waves * std::max(kps * kb, epi) + epi;
        if (sp > 1) us += (8.0 * (sp - 1) * M * (double)N / 6e6 + 2.0) / runs;   // the slices are summed once
        if (us < best.us * 0.995) {
          best = Tiles{bn, pair, sp, kps, seg, us};
        }
      }
    }
  }
  return best;
}

bool gemm_lse(int M, int V, int K, const Operands& o, const Tiles& t, const int32_t* labels, float2* part, float* zl,
              unsigned* counter, cudaStream_t s) {
  Args a = {};
  CUtensorMap ta, tb;
  if (!prepare(a, ta, tb, M, V, K, o, t)) return false;
  a.labels = labels;
  a.part = part;
  a.zl = zl;
  a.counter = counter;
  if (o.direct) return launch<false, false, kLse, false, true>(a, ta, tb, ta, s);
  return t.pair ? launch<false, false, kLse, true>(a, ta, tb, ta, s) : launch<false, false, kLse, false>(a, ta, tb, ta, s);
}

bool gemm_grad_z(int M, int n, int K, const Operands& o, const Tiles& t, const int32_t* labels, const float* lse, int first, int V, void* dz, int rows_p, int ldz, cudaStream_t s) {
  Args a = {};
  CUtensorMap ta, tb;
  if (!prepare(a, ta, tb, M, n, K, o, t)) return false;
  a.labels = labels;
  a.lse = lse;
  a.first = first;
  a.V = V;
  a.rows_p = rows_p;
  a.ldz = ldz;
  a.terms = o.terms;
  a.C = dz;
  if (o.direct) return launch<false, false, kGradZ, false, true>(a, ta, tb, ta, s);
  return t.pair ? launch<false, false, kGradZ, true>(a, ta, tb, ta, s) : launch<false, false, kGradZ, false>(a, ta, tb, ta, s);
}

bool gemm_out(int M, int N, int K, const Operands& o, const Tiles& t, int out_f32, void* C, int add, const float* omega,
              const float* dloss, cudaStream_t s) {
  Args a = {};
  CUtensorMap ta, tb, tcm;
  if (!o.b_mn || !prepare(a, ta, tb, M, N, K, o, t) || !map_out(&tcm, C, out_f32 != 0, N, M, t.splits)) return false;
  a.C = C;
  a.add = add;
  a.omega = omega;
  a.dloss = dloss;
  if (o.direct) return launch<false, true, kOut32, false, true>(a, ta, tb, tcm, s);
  if (!o.a_mn) return t.pair ? launch<false, true, kOut32, true>(a, ta, tb, tcm, s) : launch<false, true, kOut32, false>(a, ta, tb, tcm, s);
  if (out_f32) return t.pair ? launch<true, true, kOut32, true>(a, ta, tb, tcm, s) : launch<true, true, kOut32, false>(a, ta, tb, tcm, s);
  return t.pair ? launch<true, true, kOut16, true>(a, ta, tb, tcm, s) : launch<true, true, kOut16, false>(a, ta, tb, tcm, s);
}

}  // namespace vocab
}  // namespace zl
