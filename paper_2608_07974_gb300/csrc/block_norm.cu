// The step between two blocks of a layer, fused (zl_op_block_norm): p = PostNorm(f), h' = alpha h + beta gate * p,
// n = PreNorm(h'), with f and n written in 8 bits (act8.cuh) in the same pass where the caller keeps them so, and its
// backward, which reads f from there.
#include <algorithm>

#include "act8.cuh"
#include "ops.h"
#include "per_device.h"
#include "tcgen05.cuh"

namespace zl {

namespace {
using namespace act8;

// VEC: rows start on 16 bytes and are whole 8-column vectors.
constexpr int mode_of(bool vec) { return vec ? kWhole : kSingle; }

// ------------------------------------------------------------------------------------------------
// Forward
// ------------------------------------------------------------------------------------------------
struct Fwd {
  const void *h, *f;
  const float *pw, *pb, *gate, *nw, *nb;
  void *ho, *no;
  float* stats;
  uint8_t *fq, *fe, *nq, *ne;
  int N, d, D;               // D: columns in whole groups
  int post, pre, gate_rows;
  float eps, alpha, beta;
  int fmt;
  bool vec, wvec;            // whole 16-byte vectors in the rows of the tensors, of the parameters
  bool words;                // rows of the tensors in whole 4-byte words
};

__device__ __forceinline__ size_t gate_row(int n, int gate_rows) { return gate_rows ? (size_t)(n / gate_rows) : 0; }

// 8 values at column c of a row of D columns as codes (every lane of the warp calls).
template <int FMT>
__device__ __forceinline__ void put_codes(const float* x, uint8_t* q, uint8_t* e, int c, int D) {
  uint2 w;
  const uint32_t byte = encode_quarter<FMT>(x, w);
  if (c >= D) return;
  *reinterpret_cast<uint2*>(q + c) = w;
  if ((c & 31) == 0) e[c >> 5] = (uint8_t)byte;
}

// ------------------------------------------------------------------------------------------------
// Rows through a ring in shared memory, shared by forward and backward (rows of at most 8192 columns): a block, of as many
// threads as a row has 8-column vectors or half as many, works through neighbouring rows one after another while the next
// rows' tensors are copied in (bulk copies of whole rows on an mbarrier). What a row costs is then its block-wide sums, two
// in turn forward and one backward, and the issue slots of its arithmetic, not the wait for memory.
// Rows that do not start on 16 bytes, or not of whole vectors, are copied in by the block's threads, a row ahead, and shifted
// between neighbouring lanes to be written in whole 16-byte words. RMSNorm, 2048 rows,
// bf16, forward and backward: 4096 columns 16 and 27 us, 4094 25 and 43 (36 and 67 without running ahead), 4095 31 and 54.
// ------------------------------------------------------------------------------------------------
constexpr int kStages = 4;

__device__ __forceinline__ void bulk_row(void* dst, const void* src, uint32_t bytes, uint64_t* bar) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(tc::su32(dst)),
               "l"(src), "r"(bytes), "r"(tc::su32(bar))
               : "memory");
}

// A row whose start and length are multiples of 4 bytes (every fp32 row's are), copied in 4 bytes at a time without waiting.
__device__ __forceinline__ void words_in(uint8_t* sm, const void* g, int n, int t, int nt) {
  for (int i = t; i < n / 4; i += nt)
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(tc::su32(sm + 4 * i)), "l"((const uint32_t*)g + i) : "memory");
}
// A bf16 row of n bytes that starts anywhere, to where it starts as far behind a 16-byte boundary: its whole 16-byte words, and
// the ends 4 bytes, or a bf16 alone, to each of four threads from `first` on. (Rows of 4-byte words too would be copied in
// fewer steps, but every vector of them read in two and shifted: 2048 x 4094 forward 28 us against 23, backward 48 against 43.)
__device__ __forceinline__ uint32_t phase_of(const void* g) { return (uint32_t)(uintptr_t)g & 15u; }
__device__ __forceinline__ void halves_in(uint8_t* sm, const void* g, int n, int t, int nt, int first) {
  const int ph = (int)phase_of(g), end = ph + n, b0 = ph ? 16 : 0, b1 = end & ~15;
  const uint8_t* const base = (const uint8_t*)g - ph;
#pragma unroll 4
  for (int b = b0 + t * 16; b < b1; b += nt * 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(tc::su32(sm + b)), "l"(base + b) : "memory");
  const int u = t >= first ? t - first : t - first + nt;
  if (u < 4 ? ph == 0 : u >= 8 || b1 < b0) return;
  const int w = u < 4 ? 4 * u : b1 + 4 * (u - 4);
  if (w >= ph && w + 4 <= end) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(tc::su32(sm + w)), "l"(base + w) : "memory");
  } else {
    const int v = w + 2;
    if (w >= ph && w + 2 <= end) *reinterpret_cast<uint16_t*>(sm + w) = *reinterpret_cast<const uint16_t*>(base + w);
    if (v >= ph && v + 2 <= end) *reinterpret_cast<uint16_t*>(sm + v) = *reinterpret_cast<const uint16_t*>(base + v);
  }
}
template <typename T>
__device__ __forceinline__ void row_in(bool words, uint8_t* sm, const void* g, int n, int t, int nt, int first) {
  if (sizeof(T) == 4 || words) words_in(sm, g, n, t, nt);
  else halves_in(sm, g, n, t, nt, first);
}
__device__ __forceinline__ void row_wait() { asm volatile("cp.async.wait_all;" ::: "memory"); }
constexpr uint32_t kPhase = 16;   // bytes more that a row's place takes then
// Columns c .. c + 7 of row g in shared memory (0 from d on).
template <bool VEC, typename T>
__device__ __forceinline__ void row_get(Raw8<T>& r, bool words, const uint8_t* sm, const T* g, int c, int d) {
  if (VEC || sizeof(T) == 4 || words) {
    r.get(sm + c * sizeof(T));
  } else {
    r.get_around(sm + phase_of(g) + c * sizeof(T));
    if (c + 8 > d) r.trim(d - c);
  }
}

// Sums over the block; every thread gets them. The scratch (zeroed before, for the warps that do not exist) alternates between
// two buffers, so one barrier per sum is enough: who writes a buffer again has passed the barrier of the sum between, after
// which everyone had read it.
struct Reducer {
  float (*sh)[16];
  int turn;
  __device__ __forceinline__ static float total(const float* b) {
    uint64_t v[8];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 f = reinterpret_cast<const float4*>(b)[i];
      v[2 * i] = f2(f.x, f.y);
      v[2 * i + 1] = f2(f.z, f.w);
    }
#pragma unroll
    for (int i = 4; i > 0; i >>= 1)
#pragma unroll
      for (int k = 0; k < i; ++k) v[k] = add2(v[k], v[k + i]);
    const float2 f = uf2(v[0]);
    return f.x + f.y;
  }
  __device__ __forceinline__ void sum(float& x) {
    float* b = sh[turn];
    turn ^= 1;
    x = warp_sum(x);
    if ((threadIdx.x & 31) == 0) b[threadIdx.x >> 5] = x;
    __syncthreads();
    x = total(b);
  }
  // Four sums at once (b: 64 floats of scratch, warps that do not exist zero). Within a warp each step hands half of the
  // values to the other half of the lanes, so that every lane ends with one value; then the lanes take the warps' results.
  __device__ __forceinline__ static float lanes4(const float* x) {
    const int lane = threadIdx.x & 31;
    const bool hi = lane & 16, q = lane & 8;
    const float a = hi ? x[2] : x[0], b = hi ? x[3] : x[1];
    const float a2 = a + __shfl_xor_sync(0xffffffffu, hi ? x[0] : x[2], 16);
    const float b2 = b + __shfl_xor_sync(0xffffffffu, hi ? x[1] : x[3], 16);
    float v = (q ? b2 : a2) + __shfl_xor_sync(0xffffffffu, q ? a2 : b2, 8);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;   // of value lane / 8
  }
  __device__ __forceinline__ static void warps4(const float* b, float* x) {
    const int lane = threadIdx.x & 31;
    float v = b[(lane >> 3) * 16 + (lane & 7)] + b[(lane >> 3) * 16 + 8 + (lane & 7)];
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __shfl_sync(0xffffffffu, v, 8 * i);
  }
};

// The ring's place of the row at hand.
struct Turn {
  int st = 0;
  uint32_t phase = 0;
  __device__ __forceinline__ void next(int stages) {
    if (++st == stages) {
      st = 0;
      phase ^= 1u;
    }
  }
};
// Waits for the row at hand. A wait that gives up (its limit is about 2 s) raises the block's flag, which every thread sees
// after its next barrier: it writes NaN to its columns of the outputs that are not formed then.
__device__ __forceinline__ void wait_row(uint64_t* full, const Turn& at, volatile int* abort_flag) {
  tc::mbar_wait(&full[at.st], at.phase, abort_flag, nullptr);
}
// After a wait that gave up: lets the copies in flight land before the block ends (n of them, from the row at hand on).
__device__ __forceinline__ void drain(uint64_t* full, Turn at, int stages, int n) {
  for (int i = 0; i < n; ++i) {
    const unsigned long long t0 = tc::gtimer();
    while (!tc::mbar_test(&full[at.st], at.phase) && tc::gtimer() - t0 < 100000000ull) {
    }
    at.next(stages);
  }
}

// NaN in the 8 columns from c on of a row (VEC kernels, after a wait that gave up).
template <typename T>
__device__ __forceinline__ void put_nan(T* p, int c, int d) {
  const uint64_t nan2 = f2(__uint_as_float(0x7FC00000u), __uint_as_float(0x7FC00000u));
  const uint64_t v[4] = {nan2, nan2, nan2, nan2};
  Raw8<T> r;
  pack8(v, r);
  store_raw(p, c, d, r);
}

// What a launch of a ring kernel is given besides its operands.
struct Ring {
  int stages;
  int rows, more;     // forward: neighbouring rows of a block, one more of the first `more` blocks
  uint32_t pitch;     // bytes of a row of T in shared memory (whole groups)
  uint32_t stage;     // bytes of a stage
};

// 8 columns of a parameter row as pairs: `none` where it is NULL, 0 past d.
template <bool VEC>
__device__ __forceinline__ void row8(const float* p, int c, int d, float none, uint64_t* w) {
  if (p) load_raw<mode_of(VEC)>(p, c, d).pairs(w);
  else {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = f2(none, none);
  }
}
// 8 fp32 columns of a row in shared memory as pairs, the row as two planes (columns 0-3 and 4-7 of every vector), so that the
// 16-byte accesses of neighbouring lanes are neighbours.
__device__ __forceinline__ void get_pairs(const float* p, int c, int D, uint64_t* v) {
  const float4 lo = *reinterpret_cast<const float4*>(p + c / 2), hi = *reinterpret_cast<const float4*>(p + D / 2 + c / 2);
  v[0] = f2(lo.x, lo.y);
  v[1] = f2(lo.z, lo.w);
  v[2] = f2(hi.x, hi.y);
  v[3] = f2(hi.z, hi.w);
}
__device__ __forceinline__ void put_pairs(float* p, int c, int D, const uint64_t* v) {
  float f[8];
  unpair(v, f);
  *reinterpret_cast<float4*>(p + c / 2) = make_float4(f[0], f[1], f[2], f[3]);
  *reinterpret_cast<float4*>(p + D / 2 + c / 2) = make_float4(f[4], f[5], f[6], f[7]);
}
// Sums of the two halves of pairs.
__device__ __forceinline__ float fold(uint64_t v) {
  const float2 f = uf2(v);
  return f.x + f.y;
}
// Pairs with 0 in the columns from d on (VEC: d is a multiple of 8).
template <bool VEC>
__device__ __forceinline__ void cut(uint64_t* v, int c, int d) {
  if (VEC) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = c < d ? v[i] : 0;
    return;
  }
  if (c + 8 <= d) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = uf2(v[i]);
    v[i] = f2(c + 2 * i < d ? f.x : 0.f, c + 2 * i + 1 < d ? f.y : 0.f);
  }
}

// The parameters of a thread's columns: a = beta gate w_post, b = beta gate b_post, w = w_pre, v = b_pre, all 0 past d (so is
// then what they multiply). They stay in registers from row to row (a and b until the gate's row changes): read for every row
// they were 48 KB more a row than its 32 KB of traffic (d = 4096, bf16), and their latency the longest part of it.
template <int VPT, bool VEC, bool LN>
struct Params {
  uint64_t a[VPT][4], b[LN ? VPT : 1][4], w[VPT][4], v[LN ? VPT : 1][4];
  __device__ __forceinline__ void post(int j, int c, int d, const float* pw, const float* pb, const float* gate, float beta) {
    uint64_t g[4];
    row8<VEC>(gate, c, d, 1.f, g);
    row8<VEC>(pw, c, d, 1.f, a[j]);
    if (LN) row8<VEC>(pb, c, d, 0.f, b[j]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      g[i] = mul2(g[i], f2(beta, beta));
      a[j][i] = mul2(a[j][i], g[i]);
      if (LN) b[j][i] = mul2(b[j][i], g[i]);
    }
    cut<VEC>(a[j], c, d);
  }
  __device__ __forceinline__ void pre(int j, int c, int d, const float* nw, const float* nb) {
    row8<VEC>(nw, c, d, 1.f, w[j]);
    if (LN) row8<VEC>(nb, c, d, 0.f, v[j]);
    cut<VEC>(w[j], c, d);
  }
};

// NaN in this thread's columns of what rows n .. end - 1 have not got (a call apart: written inside the kernel it changed how
// the row loop is compiled, 2048 x 4096 with LayerNorms 22.4 us against 21.0).
template <typename T, int KEEP>
__device__ __noinline__ void fwd_give_up(const Fwd& a, int n, int end) {
  for (; n < end; ++n) {
    const size_t row = n;
    for (int c = threadIdx.x * 8; c < a.d; c += blockDim.x * 8) {
      put_nan((T*)a.ho + row * a.d, c, a.d);
      if (a.pre) put_nan((T*)a.no + row * a.d, c, a.d);
      const uint32_t w = KEEP == ZL_ACT8_E4M3 ? 0x7F7F7F7Fu : 0x80808080u;
      if (a.fq) *reinterpret_cast<uint2*>(a.fq + row * a.D + c) = make_uint2(w, w);
      if (a.nq) *reinterpret_cast<uint2*>(a.nq + row * a.D + c) = make_uint2(w, w);
    }
    if (threadIdx.x < 4) a.stats[threadIdx.x * (size_t)a.N + row] = __uint_as_float(0x7FC00000u);
  }
}

// Forward. VEC: rows come by bulk copies. KEEP: the format that f or n are written in, -1: neither is. LN: one of the norms
// is a LayerNorm. HBM-bound on large batches, 8 bytes a value in bf16 (10.06 with both checkpoints): 4096 x 8192 with RMS
// norms 46 us (5.8 TB/s, 86% of the measured copy rate; with checkpoints 69 us); on 2048 x 4096, where a block has six or seven
// rows, the launch, the first rows' copies and the sums' latency show: 15.7 us (20.9 with checkpoints), LayerNorms, with four
// sums a row, 21.1. A block for each row, which waits for it and reads the parameters anew, took 35 and 43 us.
template <typename T, int VPT, bool VEC, bool LN, int KEEP>
__global__ void __launch_bounds__(512) __maxnreg__(LN || (VPT == 2 && sizeof(T) == 4) ? 128 : VPT == 1 ? 64 : 80)
    fwd_ring_k(const __grid_constant__ Fwd a, const Ring g) {
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ uint64_t full[kStages];
  __shared__ __align__(16) float sh[2][16];
  __shared__ int abort_word;
  volatile int* abort_flag = &abort_word;
  const int t = threadIdx.x, nt = blockDim.x;
  const int r0 = (int)blockIdx.x * g.rows + min((int)blockIdx.x, g.more), rows = g.rows + ((int)blockIdx.x < g.more ? 1 : 0);
  const uint32_t bytes = (uint32_t)a.d * sizeof(T);
  if (t == 0) {
    for (int i = 0; i < g.stages; ++i) tc::mbar_init(&full[i], 1);
    abort_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (t < 32) (&sh[0][0])[t] = 0.f;
  for (int k = 0; k < 2 * g.stages; ++k)   // columns past d read 0
    for (int c = a.d + t; c < a.D; c += nt) reinterpret_cast<T*>(ring + (k >> 1) * g.stage + (k & 1) * g.pitch)[c] = from_f<T>(0.f);
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  const bool ahead = !VEC && g.stages > 1;   // the next row is copied in meanwhile
  auto fill = [&](int k, int st) {   // row number k of this block into a stage
    uint8_t* p = ring + st * g.stage;
    const size_t o = (size_t)(r0 + k) * a.d;
    if (VEC) {
      uint64_t* bar = &full[st];
      tc::mbar_expect_tx(bar, 2 * bytes);
      bulk_row(p, (const T*)a.f + o, bytes, bar);
      bulk_row(p + g.pitch, (const T*)a.h + o, bytes, bar);
    } else {
      row_in<T>(a.words, p, (const T*)a.f + o, (int)bytes, t, nt, 0);
      row_in<T>(a.words, p + g.pitch, (const T*)a.h + o, (int)bytes, t, nt, 32 % nt);
    }
  };
  if (VEC && t == 0)
    for (int k = 0; k < min(rows, g.stages); ++k) fill(k, k);
  if (ahead) fill(0, 0);
  Params<VPT, VEC, LN> pa;
#pragma unroll
  for (int j = 0; j < VPT; ++j) pa.pre(j, (t + j * nt) * 8, a.d, a.nw, a.nb);
  int gate_left = 0;   // rows of the gate row at hand that are still to come
  Reducer red{sh, 0};
  Turn at;
  const float inv_d = 1.f / a.d;
  const uint64_t alpha = f2(a.alpha, a.alpha);
  int k = 0;
  for (; k < rows; ++k, at.next(g.stages)) {
    const int row = r0 + k, st = at.st;
    const size_t o = (size_t)row * a.d;
    if (gate_left == 0) {
      const size_t gr = gate_row(row, a.gate_rows);
      gate_left = a.gate_rows ? a.gate_rows - row % a.gate_rows : a.N;
#pragma unroll
      for (int j = 0; j < VPT; ++j) pa.post(j, (t + j * nt) * 8, a.d, a.pw, a.pb, a.gate ? a.gate + gr * a.d : nullptr, a.beta);
    }
    --gate_left;
    if (VEC) {
      wait_row(full, at, abort_flag);
    } else {
      if (!ahead) {
        __syncthreads();
        fill(k, 0);
      }
      row_wait();
      __syncthreads();
    }
    Raw8<T> rf[VPT], rh[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int c = (t + j * nt) * 8;
      rf[j].zero();
      rh[j].zero();
      if (c < a.D) {
        row_get<VEC>(rf[j], a.words, ring + st * g.stage, (const T*)a.f + o, c, a.d);
        row_get<VEC>(rh[j], a.words, ring + st * g.stage + g.pitch, (const T*)a.h + o, c, a.d);
      }
    }
    // 1 / deviation of the values val(j, x) of every vector, and with a LayerNorm their mean; after the first barrier of a row
    // everyone has it in registers, and its stage takes the row `stages` further on
    auto stat = [&](int kind, auto&& val, bool first, float& mean, float& rstd) {
      mean = 0.f;
      rstd = 1.f;
      auto next = [&]() {
        if (VEC && first && t == 0 && k + g.stages < rows && !*abort_flag) fill(k + g.stages, st);
        if (ahead && first && k + 1 < rows) fill(k + 1, st ^ 1);
        first = false;
      };
      if (kind == ZL_NORM_NONE) {
        if (first) {
          __syncthreads();
          next();
        }
        return;
      }
      if (LN && kind == ZL_NORM_LAYER) {
        uint64_t s = 0;
#pragma unroll
        for (int j = 0; j < VPT; ++j) {
          uint64_t x[4];
          val(j, x);
          s = add2(s, add2(add2(x[0], x[1]), add2(x[2], x[3])));
        }
        mean = fold(s);
        red.sum(mean);
        next();
        mean *= inv_d;
      }
      const uint64_t mm = f2(-mean, -mean);
      uint64_t q2 = 0;
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int c = (t + j * nt) * 8;
        uint64_t x[4];
        val(j, x);
        if (LN) {   // columns past d are not 0 any more
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = add2(x[i], mm);
          if (!VEC) cut<VEC>(x, c, a.d);
        }
        if (!LN || !VEC || c < a.d) {
#pragma unroll
          for (int i = 0; i < 4; ++i) q2 = fma2(x[i], x[i], q2);
        }
      }
      float q = fold(q2);
      red.sum(q);
      next();
      rstd = rsqrtf(q * inv_d + a.eps);
    };
    if (KEEP >= 0 && a.fq) {
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        float x[8];
        floats(rf[j], x);
        put_codes<KEEP < 0 ? 0 : KEEP>(x, a.fq + (size_t)row * a.D, a.fe + (size_t)row * (a.D >> 5), (t + j * nt) * 8, a.D);
      }
    }
    float pm, pr, m, r;
    stat(a.post, [&](int j, uint64_t* x) { rf[j].pairs(x); }, true, pm, pr);
    if (VEC && *abort_flag) break;
    uint64_t h[VPT][4];
    {
      const uint64_t mm = f2(-pm, -pm), rr = f2(pr, pr);
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int c = (t + j * nt) * 8;
        uint64_t f[4];
        rf[j].pairs(f);
        rh[j].pairs(h[j]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (LN) f[i] = add2(f[i], mm);
          h[j][i] = fma2(mul2(f[i], rr), pa.a[j][i], mul2(alpha, h[j][i]));
          if (LN) h[j][i] = add2(h[j][i], pa.b[j][i]);
        }
        if (!VEC) cut<VEC>(h[j], c, a.d);   // (0 past d is NaN times 0 in a row with a NaN)
        Raw8<T> out;
        pack8(h[j], out);
        if (VEC) store_raw((T*)a.ho + o, c, a.d, out);
        else store_any((T*)a.ho + o, c, a.d, out);
      }
    }
    stat(a.pre, [&](int j, uint64_t* x) {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = h[j][i];
    }, false, m, r);
    if (t == 0) {
      float* q = a.stats + row;
      q[0] = pm;
      q[a.N] = pr;
      q[2 * (size_t)a.N] = m;
      q[3 * (size_t)a.N] = r;
    }
    if (!a.pre) continue;
    const uint64_t mm = f2(-m, -m), rr = f2(r, r);
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int c = (t + j * nt) * 8;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (LN) h[j][i] = add2(h[j][i], mm);
        h[j][i] = mul2(mul2(h[j][i], rr), pa.w[j][i]);
        if (LN) h[j][i] = add2(h[j][i], pa.v[j][i]);
      }
      if (!VEC || KEEP >= 0) cut<VEC>(h[j], c, a.d);
      Raw8<T> out;
      pack8(h[j], out);
      if (VEC) store_raw((T*)a.no + o, c, a.d, out);
      else store_any((T*)a.no + o, c, a.d, out);
      if (KEEP >= 0 && a.nq) {   // of n as it is stored
        float n[8];
        floats(out, n);
        put_codes<KEEP < 0 ? 0 : KEEP>(n, a.nq + (size_t)row * a.D, a.ne + (size_t)row * (a.D >> 5), c, a.D);
      }
    }
  }
  if (!VEC || k == rows) return;
  if (t == 0) drain(full, at, g.stages, min(rows - k, g.stages + 1));   // (one more: the row at hand's stage may be filling again)
  fwd_give_up<T, KEEP>(a, r0 + k, r0 + rows);
}

__device__ __forceinline__ void put_any(int fmt, const float* x, uint8_t* q, uint8_t* e, size_t row, int c, int D) {
  if (fmt == ZL_ACT8_E4M3) put_codes<ZL_ACT8_E4M3>(x, q + row * D, e + row * (D >> 5), c, D);
  else put_codes<ZL_ACT8_INT8>(x, q + row * D, e + row * (D >> 5), c, D);
}

// Rows of any width (the ring kernels take up to 8192 columns): a block per row that reads it again for every sum.
template <typename T, bool VEC>
__global__ void __launch_bounds__(512) fwd_any_k(const Fwd a) {
  pdl_wait();
  pdl_trigger();
  __shared__ float sh[32];
  const int row = blockIdx.x;
  const size_t o = (size_t)row * a.d;
  const float inv_d = 1.f / a.d;
  const float* gr = a.gate ? a.gate + gate_row(row, a.gate_rows) * a.d : nullptr;
  float pm = 0.f, pr = 1.f, m = 0.f, r = 1.f;
  auto fval = [&](int c, float* x) { load8<mode_of(VEC)>((const T*)a.f + o, c, a.d, x); };
  auto hval = [&](int c, float* x) {   // h' before its rounding
    float f[8], w[8];
    fval(c, f);
    load8<mode_of(VEC)>((const T*)a.h + o, c, a.d, x);
    if (a.post) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = (f[i] - pm) * pr;
      if (a.pw) {
        load8<mode_of(VEC)>(a.pw, c, a.d, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] *= w[i];
      }
      if (a.pb) {
        load8<mode_of(VEC)>(a.pb, c, a.d, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] += w[i];
      }
    }
    if (gr) {
      load8<mode_of(VEC)>(gr, c, a.d, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] *= w[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = a.alpha * x[i] + a.beta * f[i];
  };
  auto stat = [&](auto&& val, int kind, float& mean, float& rstd) {
    if (kind == ZL_NORM_NONE) return;
    float x[8], s = 0.f, q = 0.f, mu = 0.f;
    if (kind == ZL_NORM_LAYER) {
      for (int c = threadIdx.x * 8; c < a.d; c += blockDim.x * 8) {
        val(c, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) s += c + i < a.d ? x[i] : 0.f;
      }
      mu = block_sum(s, sh) * inv_d;
    }
    for (int c = threadIdx.x * 8; c < a.d; c += blockDim.x * 8) {
      val(c, x);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = c + i < a.d ? x[i] - mu : 0.f;
        q += v * v;
      }
    }
    rstd = 1.f / sqrtf(block_sum(q, sh) * inv_d + a.eps);
    mean = mu;
  };
  stat(fval, a.post, pm, pr);
  stat(hval, a.pre, m, r);
  if (threadIdx.x == 0) {
    a.stats[row] = pm;
    a.stats[(size_t)a.N + row] = pr;
    a.stats[2 * (size_t)a.N + row] = m;
    a.stats[3 * (size_t)a.N + row] = r;
  }
  const int last = (a.D + blockDim.x * 8 - 1) / (blockDim.x * 8);
  for (int k = 0; k < last; ++k) {   // every lane of a warp takes every turn: four lanes form a group
    const int c = (threadIdx.x + k * blockDim.x) * 8;
    float x[8], w[8];
    if (a.fq) {
      fval(c, x);
      put_any(a.fmt, x, a.fq, a.fe, (size_t)row, c, a.D);
    }
    hval(c, x);
    store8<mode_of(VEC)>((T*)a.ho + o, c, a.d, x);
    if (!a.pre) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (x[i] - m) * r;
    if (a.nw) {
      load8<mode_of(VEC)>(a.nw, c, a.d, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= w[i];
    }
    if (a.nb) {
      load8<mode_of(VEC)>(a.nb, c, a.d, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] += w[i];
    }
    store8<mode_of(VEC)>((T*)a.no + o, c, a.d, x);
    if (a.nq) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = c + i < a.d ? to_f(from_f<T>(x[i])) : 0.f;
      put_any(a.fmt, x, a.nq, a.ne, (size_t)row, c, a.D);
    }
  }
}

// Blocks of a kernel (th threads, `smem` dynamic bytes) that an SM holds, from the registers that it was compiled with. Finding
// out also lets the kernel take that much shared memory, which holds for one device.
struct Occupancy {
  int regs = 0, fixed = 0;
  template <typename K>
  bool find(K kern) {
    cudaFuncAttributes fa;
    if (cudaFuncGetAttributes(&fa, kern) != cudaSuccess ||
        cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxSmem - (int)fa.sharedSizeBytes) != cudaSuccess)
      return false;
    regs = (fa.numRegs + 7) / 8 * 8;
    fixed = (int)fa.sharedSizeBytes + 1024;
    return true;
  }
  int blocks(int th, size_t smem) const {
    return std::max(1, std::min({2048 / th, 65536 / (regs * th), (int)((kMaxSmem + 1024) / (smem + fixed)), 32}));
  }
  static constexpr int kMaxSmem = 232448;
};
// That of the current device (NULL: the kernel cannot run there; the CUDA error says why).
template <typename K>
const Occupancy* occupancy(PerDevice<Occupancy>& devices, K kern) {
  int dev = 0;
  return cudaGetDevice(&dev) == cudaSuccess ? devices.get(dev, [&](Occupancy& o) { return o.find(kern); }) : nullptr;
}

constexpr int kRingCols = 8192;   // the widest row of the ring kernels
// Threads of a block for a row of nvec vectors, one vector a thread or two.
int ring_threads(int nvec) { return nvec <= 224 ? (nvec + 31) / 32 * 32 : (nvec + 63) / 64 * 32; }

template <typename T, int VPT, bool VEC, bool LN, int KEEP>
bool fwd_ring(const Fwd& a, int th, cudaStream_t s) {
  static PerDevice<Occupancy> devices;
  const Occupancy* const found = occupancy(devices, fwd_ring_k<T, VPT, VEC, LN, KEEP>);
  if (!found) return false;
  const Occupancy& occ = *found;
  Ring g;
  g.pitch = (uint32_t)a.D * sizeof(T) + (VEC ? 0 : kPhase);
  g.stage = 2 * g.pitch;
  const int want = std::max(1, std::min({2048 / th, 65536 / (occ.regs * th), 16}));   // blocks that the registers allow
  const size_t room = std::max((size_t)(Occupancy::kMaxSmem + 1024) / want, (size_t)occ.fixed) - occ.fixed;
  g.stages = VEC ? (int)std::min<size_t>(kStages, std::max<size_t>(2, room / g.stage)) : 2;
  if ((size_t)g.stages * g.stage + occ.fixed > (size_t)Occupancy::kMaxSmem) g.stages = 1;
  const size_t smem = (size_t)g.stages * g.stage;
  if (smem + occ.fixed > (size_t)Occupancy::kMaxSmem) return false;
  const int slots = sm_count() * occ.blocks(th, smem);
  const int grid = std::min(a.N, slots);
  g.rows = a.N / grid;
  g.more = a.N % grid;
  return launch_pdl(fwd_ring_k<T, VPT, VEC, LN, KEEP>, grid, th, smem, s, a, g) == cudaSuccess;
}
template <typename T, int VPT, bool VEC, bool LN>
bool fwd_ring_by(const Fwd& a, int th, cudaStream_t s) {
  if (!a.fq && !a.nq) return fwd_ring<T, VPT, VEC, LN, -1>(a, th, s);
  return a.fmt == ZL_ACT8_E4M3 ? fwd_ring<T, VPT, VEC, LN, ZL_ACT8_E4M3>(a, th, s)
                               : fwd_ring<T, VPT, VEC, LN, ZL_ACT8_INT8>(a, th, s);
}

// One vector a thread up to 512 threads with RMS norms, up to 224 with a LayerNorm, whose parameters leave no second block of
// 512 threads on an SM: 2048 x 4096 bf16 with RMS norms 15.7 us, with
// LayerNorms 21.1 us (one vector in 64 registers 22.7).
template <typename T, bool VEC>
bool forward_as(const Fwd& a, cudaStream_t s) {
  const int nvec = a.D / 8;
  const bool ln = a.post == ZL_NORM_LAYER || a.pre == ZL_NORM_LAYER;
  note_launch(1);
  if (a.d <= kRingCols) {
    const int th = !ln && nvec <= 512 ? (nvec + 31) / 32 * 32 : ring_threads(nvec);
    if (th >= nvec) return ln ? fwd_ring_by<T, 1, VEC, true>(a, th, s) : fwd_ring_by<T, 1, VEC, false>(a, th, s);
    return ln ? fwd_ring_by<T, 2, VEC, true>(a, th, s) : fwd_ring_by<T, 2, VEC, false>(a, th, s);
  }
  return launch_pdl(fwd_any_k<T, VEC>, a.N, 512, 0, s, a) == cudaSuccess;
}
template <typename T>
bool forward(const Fwd& a, cudaStream_t s) {
  return a.vec && a.wvec ? forward_as<T, true>(a, s) : forward_as<T, false>(a, s);
}

// ------------------------------------------------------------------------------------------------
// Backward. With xh = (h' - m) r, u = w_pre dn, fh = (f - m_p) r_p, p = fh w_post + b_post:
//   G  = dh' + r (u - [LN] mean(u) - xh mean(u xh))         gradient at h'
//   dh = alpha G,  dp = beta gate G,  v = w_post dp,  df = r_p (v - [LN] mean(v) - fh mean(v fh))
//   dw_pre = sum dn xh, db_pre = sum dn, dw_post = sum dp fh, db_post = sum dp, dgate = sum beta G p  (over rows)
// ------------------------------------------------------------------------------------------------
struct Bwd {
  const void *ho, *f;
  const uint8_t *fq, *fe;
  const float *pw, *pb, *gate, *nw, *stats;
  const void *dn, *dho;
  void *dh, *df;
  float* s12;                // [2, N]: mean(u), mean(u xh)
  float* part;               // [chunks, slots, D] partial sums, see kDw .. (NULL: no gradient of a parameter is asked for)
  float *dpw, *dpb, *dgate, *dnw, *dnb;
  int N, d, D;
  int post, pre, gate_rows;
  float alpha, beta;
  int fmt, accumulate;
  bool vec, wvec, words;
  int rows, per_group, chunks;   // the chunks of rows that partial sums are of
  int slots;
  bool ring;                 // by bwd_ring_k
};
// Slots of a chunk's partial sums: sum dn xh, s, and with a LayerNorm sum dn, z. s = sum G fh and z = sum G where a chunk lies
// in one gate group (per_group > 0), else both already times beta gate.
enum { kDw = 0, kS = 1, kDb = 2, kZ = 3 };

// Rows [r0, r1) of chunk k. Gate groups longer than a chunk are cut into per_group chunks each; shorter ones lie whole in
// a chunk (per_group 0), which then knows their dgate alone.
__host__ __device__ __forceinline__ void chunk_rows(int k, int N, int gate_rows, int rows, int per_group, int& r0, int& r1) {
  if (per_group) {
    const long long g0 = (long long)(k / per_group) * gate_rows, b = g0 + (long long)(k % per_group) * rows;
    const long long end = g0 + gate_rows < N ? g0 + gate_rows : N;
    r0 = (int)(b < end ? b : end);
    r1 = (int)(b + rows < end ? b + rows : end);
  } else {
    const long long b = (long long)k * rows;
    r0 = (int)(b < N ? b : N);
    r1 = (int)(b + rows < N ? b + rows : N);
  }
}

// f of row n, columns c .. c + 7.
template <typename T, bool VEC>
__device__ __forceinline__ void f8(const Bwd& a, int n, int c, float* x) {
  if (a.fq) {
    const size_t at = (size_t)n * a.D + c;
    if (c < a.D) {
      const uint2 w = *reinterpret_cast<const uint2*>(a.fq + at);
      if (a.fmt == ZL_ACT8_E4M3) decode8<ZL_ACT8_E4M3>(w, a.fe[at >> 5], x);
      else decode8<ZL_ACT8_INT8>(w, a.fe[at >> 5], x);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = 0.f;
    }
  } else {
    load8<mode_of(VEC)>((const T*)a.f + (size_t)n * a.d, c, a.d, x);
  }
}

// G of row n, columns c .. (0 past d).
template <typename T, bool VEC>
__device__ __forceinline__ void grad8(const Bwd& a, int n, int c, float s1, float s2, float* G) {
  const size_t o = (size_t)n * a.d;
#pragma unroll
  for (int i = 0; i < 8; ++i) G[i] = 0.f;
  if (a.dho) load8<mode_of(VEC)>((const T*)a.dho + o, c, a.d, G);
  if (a.pre) {
    const float m = a.stats[2 * (size_t)a.N + n], r = a.stats[3 * (size_t)a.N + n];
    float u[8], x[8], w[8];
    load8<mode_of(VEC)>((const T*)a.dn + o, c, a.d, u);
    load8<mode_of(VEC)>((const T*)a.ho + o, c, a.d, x);
    if (a.nw) {
      load8<mode_of(VEC)>(a.nw, c, a.d, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] *= w[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) G[i] += c + i < a.d ? r * (u[i] - s1 - (x[i] - m) * r * s2) : 0.f;
  }
}

// mean(u) (LayerNorm) and mean(u xh) of every row.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) bwd_sums_k(const Bwd a) {
  pdl_wait();
  pdl_trigger();
  __shared__ float sh[32];
  const int n = blockIdx.x;
  const size_t o = (size_t)n * a.d;
  const float m = a.stats[2 * (size_t)a.N + n], r = a.stats[3 * (size_t)a.N + n];
  float s1 = 0.f, s2 = 0.f;
  for (int c = threadIdx.x * 8; c < a.d; c += blockDim.x * 8) {
    float u[8], x[8], w[8];
    load8<mode_of(VEC)>((const T*)a.dn + o, c, a.d, u);
    load8<mode_of(VEC)>((const T*)a.ho + o, c, a.d, x);
    if (a.nw) {
      load8<mode_of(VEC)>(a.nw, c, a.d, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] *= w[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      s1 += u[i];
      s2 += u[i] * ((x[i] - m) * r);
    }
  }
  s1 = block_sum(s1, sh);
  s2 = block_sum(s2, sh);
  if (threadIdx.x == 0) {
    a.s12[n] = a.pre == ZL_NORM_LAYER ? s1 / a.d : 0.f;
    a.s12[(size_t)a.N + n] = s2 / a.d;
  }
}

// Partial column sums of a chunk: 32 vectors of columns x 8 row lanes a block, the lanes' sums added in order.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) bwd_cols_k(const Bwd a) {
  pdl_wait();
  pdl_trigger();
  __shared__ float sh[8][256];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, c = (blockIdx.y * 32 + tx) * 8;
  int r0, r1;
  chunk_rows(blockIdx.x, a.N, a.gate_rows ? a.gate_rows : a.N, a.rows, a.per_group, r0, r1);
  // sums dn xh, G fh, dn, G; and the last two of the post norm times beta gate, of gate groups within the chunk
  float acc[4][8], post[2][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) acc[0][i] = acc[1][i] = acc[2][i] = acc[3][i] = post[0][i] = post[1][i] = 0.f;
  // the sum over the row lanes of v at this thread's column blockIdx.y * 256 + threadIdx.x
  auto join = [&](const float* v) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) sh[ty][tx * 8 + i] = v[i];
    __syncthreads();
    float s = 0.f;
#pragma unroll
    for (int y = 0; y < 8; ++y) s += sh[y][threadIdx.x];
    return s;
  };
  const int col = blockIdx.y * 256 + threadIdx.x;
  const int gr = a.per_group || !a.gate_rows ? r1 - r0 : a.gate_rows;   // rows of a gate group within the chunk
  for (int g0 = r0; g0 < r1; g0 += gr) {
    for (int n = g0 + ty; n < min(g0 + gr, r1) && c < a.d; n += 8) {
      float G[8], w[8], x[8];
      grad8<T, VEC>(a, n, c, a.pre ? a.s12[n] : 0.f, a.pre ? a.s12[(size_t)a.N + n] : 0.f, G);
      if (a.pre) {
        const float m = a.stats[2 * (size_t)a.N + n], r = a.stats[3 * (size_t)a.N + n];
        load8<mode_of(VEC)>((const T*)a.dn + (size_t)n * a.d, c, a.d, w);
        load8<mode_of(VEC)>((const T*)a.ho + (size_t)n * a.d, c, a.d, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          acc[kDw][i] += w[i] * ((x[i] - m) * r);
          acc[kDb][i] += w[i];
        }
      }
      f8<T, VEC>(a, n, c, x);
      const float pm = a.stats[n], pr = a.stats[(size_t)a.N + n];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        acc[kS][i] += G[i] * (a.post ? (x[i] - pm) * pr : x[i]);
        acc[kZ][i] += G[i];
      }
    }
    if (a.per_group) continue;
    float gt[8];
    const size_t grow = gate_row(g0, a.gate_rows);
#pragma unroll
    for (int i = 0; i < 8; ++i) gt[i] = 1.f;
    if (a.gate) load8<mode_of(VEC)>(a.gate + grow * a.d, c, a.d, gt);
    const float sv = join(acc[kS]), zv = join(acc[kZ]);
    if (a.dgate && col < a.d) {
      const float v = a.beta * ((a.pw ? a.pw[col] : 1.f) * sv + (a.pb ? a.pb[col] : 0.f) * zv);
      float* p = a.dgate + grow * a.d + col;
      *p = a.accumulate ? *p + v : v;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      post[0][i] += a.beta * gt[i] * acc[kS][i];
      post[1][i] += a.beta * gt[i] * acc[kZ][i];
      acc[kS][i] = acc[kZ][i] = 0.f;
    }
  }
  float* const part = a.part + (size_t)blockIdx.x * a.slots * a.D;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (k >= a.slots) continue;
    const float s = join(k == kS && !a.per_group ? post[0] : k == kZ && !a.per_group ? post[1] : acc[k]);
    if (col < a.D) part[k * (size_t)a.D + col] = col < a.d ? s : 0.f;
  }
}

// dh and df of every row.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) bwd_rows_k(const Bwd a) {
  pdl_wait();
  pdl_trigger();
  __shared__ float sh[32];
  const int n = blockIdx.x;
  const size_t o = (size_t)n * a.d;
  const float s1 = a.pre ? a.s12[n] : 0.f, s2 = a.pre ? a.s12[(size_t)a.N + n] : 0.f;
  const float pm = a.stats[n], pr = a.stats[(size_t)a.N + n];
  const float* gr = a.gate ? a.gate + gate_row(n, a.gate_rows) * a.d : nullptr;
  // G, v and fh of columns c ..
  auto vals = [&](int c, float* G, float* v, float* fh) {
    float w[8];
    grad8<T, VEC>(a, n, c, s1, s2, G);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = a.beta * G[i];
    if (gr) {
      load8<mode_of(VEC)>(gr, c, a.d, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= w[i];
    }
    if (!a.post) return;
    if (a.pw) {
      load8<mode_of(VEC)>(a.pw, c, a.d, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= w[i];
    }
    f8<T, VEC>(a, n, c, fh);
#pragma unroll
    for (int i = 0; i < 8; ++i) fh[i] = (fh[i] - pm) * pr;
  };
  float t1 = 0.f, t2 = 0.f, G[8], v[8], fh[8];
  if (a.post) {
    for (int c = threadIdx.x * 8; c < a.d; c += blockDim.x * 8) {
      vals(c, G, v, fh);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (c + i >= a.d) continue;
        t1 += v[i];
        t2 += v[i] * fh[i];
      }
    }
    t1 = block_sum(t1, sh) / a.d;
    t2 = block_sum(t2, sh) / a.d;
    if (a.post == ZL_NORM_RMS) t1 = 0.f;
  }
  for (int c = threadIdx.x * 8; c < a.d; c += blockDim.x * 8) {
    vals(c, G, v, fh);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      G[i] *= a.alpha;
      if (a.post) v[i] = pr * (v[i] - t1 - fh[i] * t2);
    }
    if (a.dh) store8<mode_of(VEC)>((T*)a.dh + o, c, a.d, G);
    store8<mode_of(VEC)>((T*)a.df + o, c, a.d, v);
  }
}

// ------------------------------------------------------------------------------------------------
// Backward in one pass over the rows: a block takes a chunk of neighbouring rows through the ring (dn, dh', h', f of a row a
// stage) and keeps its columns' sums over them in registers. With s = sum G fh and z = sum G over rows of one gate row,
//   dgate = beta (w_post s + b_post z),  dw_post = beta gate s,  db_post = beta gate z
// so two sums (four with a LayerNorm's bias) are kept for five gradients.
// G = dh' + r (u - m1 - xh m2) needs the row's means m1 of u and m2 of u xh, df the means of v = A G (A = beta gate w_post)
// and of v fh. These are linear in m1 and m2: with g = dh' + r u,
//   sum v fh = sum A fh g - r m1 sum A fh - r m2 sum A fh xh,   sum v = sum A g - r m1 sum A - r m2 sum A xh
// so one barrier a row yields every mean: three sums with RMS norms, eight at most.
// HBM-bound on large batches, 11.03 bytes a value in bf16 with f from its checkpoint: 4096 x 8192 71 us (5.2 TB/s, 76% of the
// measured copy rate; without gradients of parameters 65 us); 2048 x 4096 27.1 us, of which the partial sums and their
// joining kernel take 6, launch and the first rows 4; LayerNorms 34.2. Three kernels that each read the rows took 91 us, two
// barriers a row in one kernel 38.6.
// ------------------------------------------------------------------------------------------------
// The normalised f, (f - pm) pr, at column c of row g in shared memory (a row of T, or of codes whose group byte is e).
template <typename T, bool VEC, bool LN>
__device__ __forceinline__ void norm_f(const Bwd& a, const uint8_t* row, const T* g, uint32_t e, int c, float pm, float pr,
                                       uint64_t* f) {
  float sc = 1.f;
  if (a.fq) {
    const uint2 w = *reinterpret_cast<const uint2*>(row + c);
    float x[8];
    if (a.fmt == ZL_ACT8_E4M3) {
      codes4<ZL_ACT8_E4M3>(w.x, x);
      codes4<ZL_ACT8_E4M3>(w.y, x + 4);
    } else {
      codes4<ZL_ACT8_INT8>(w.x, x);
      codes4<ZL_ACT8_INT8>(w.y, x + 4);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = f2(x[2 * i], x[2 * i + 1]);
    sc = group_scale(e);
  } else {
    Raw8<T> r;
    row_get<VEC>(r, a.words, row, g, c, a.d);
    r.pairs(f);
  }
  if (LN) {   // the product with a power of two is exact
    const uint64_t ss = f2(sc, sc), mm = f2(-pm, -pm), rr = f2(pr, pr);
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = mul2(fma2(f[i], ss, mm), rr);
  } else {
    // (a group's scale is at most the row's largest value, pr its deviation's inverse: their product does not overflow)
    const uint64_t rr = f2(sc * pr, sc * pr);
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = mul2(f[i], rr);
  }
}

// NaN in this thread's columns of what the block's rows from number k on have not got, and of its partial sums.
template <typename T>
__device__ __noinline__ void bwd_give_up(const Bwd& a, int k) {
  int r0, r1;
  chunk_rows(blockIdx.x, a.N, a.gate_rows ? a.gate_rows : a.N, a.rows, a.per_group, r0, r1);
  for (int c = threadIdx.x * 8; c < a.d; c += blockDim.x * 8) {
    for (int n = r0 + k; n < r1; ++n) {
      if (a.dh) put_nan((T*)a.dh + (size_t)n * a.d, c, a.d);
      put_nan((T*)a.df + (size_t)n * a.d, c, a.d);
      if (a.dgate && !a.per_group) put_nan(a.dgate + gate_row(n, a.gate_rows) * a.d, c, a.d);
    }
    for (int slot = 0; a.part && slot < a.slots; ++slot) put_nan(a.part + ((size_t)blockIdx.x * a.slots + slot) * a.D, c, a.d);
  }
}

// LN: one of the norms is a LayerNorm (its sums of u, v and A, and the biases' gradients).
template <typename T, int VPT, bool VEC, bool LN>
__global__ void __launch_bounds__(512) bwd_ring_k(const __grid_constant__ Bwd a, const Ring g) {
  extern __shared__ __align__(128) uint8_t ring[];
  __shared__ uint64_t full[kStages];
  __shared__ __align__(16) float sh[2][LN ? 2 : 1][64];
  __shared__ int abort_word;
  volatile int* abort_flag = &abort_word;
  const int t = threadIdx.x, nt = blockDim.x;
  const int gate_rows = a.gate_rows ? a.gate_rows : a.N;
  int r0, r1;
  chunk_rows(blockIdx.x, a.N, gate_rows, a.rows, a.per_group, r0, r1);
  const int rows = r1 - r0;
  const uint32_t bytes = (uint32_t)a.d * sizeof(T);
  if (t == 0) {
    for (int i = 0; i < g.stages; ++i) tc::mbar_init(&full[i], 1);
    abort_word = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  for (int i = t; i < (LN ? 256 : 128); i += nt) (&sh[0][0][0])[i] = 0.f;
  if (a.d != a.D || !a.dho) {   // columns past d, and a tensor that is not given, read 0
    for (int k = 0; k < 4 * g.stages; ++k) {
      const int which = k & 3;
      if (which == 3 && a.fq) continue;
      for (int c = (which == 1 && !a.dho ? 0 : a.d) + t; c < a.D; c += nt)
        reinterpret_cast<T*>(ring + (k >> 2) * g.stage + which * g.pitch)[c] = from_f<T>(0.f);
    }
  }
  __syncthreads();
  pdl_wait();
  pdl_trigger();
  const bool next_in = !VEC && g.stages > 1;   // the next row is copied in meanwhile
  auto fill = [&](int k, int st) {   // row number k of this block into a stage
    uint8_t* p = ring + st * g.stage;
    const int n = r0 + k;
    const size_t o = (size_t)n * a.d;
    if (VEC) {
      uint64_t* bar = &full[st];
      tc::mbar_expect_tx(bar, bytes * ((a.pre ? 2 : 0) + (a.dho ? 1 : 0) + (a.fq ? 0 : 1)) + (a.fq ? (uint32_t)a.D : 0u));
      if (a.pre) {
        bulk_row(p, (const T*)a.dn + o, bytes, bar);
        bulk_row(p + 2 * g.pitch, (const T*)a.ho + o, bytes, bar);
      }
      if (a.dho) bulk_row(p + g.pitch, (const T*)a.dho + o, bytes, bar);
      if (a.fq) bulk_row(p + 3 * g.pitch, a.fq + (size_t)n * a.D, (uint32_t)a.D, bar);
      else bulk_row(p + 3 * g.pitch, (const T*)a.f + o, bytes, bar);
    } else {
      if (a.pre) {
        row_in<T>(a.words, p, (const T*)a.dn + o, (int)bytes, t, nt, 0);
        row_in<T>(a.words, p + 2 * g.pitch, (const T*)a.ho + o, (int)bytes, t, nt, 64 % nt);
      }
      if (a.dho) row_in<T>(a.words, p + g.pitch, (const T*)a.dho + o, (int)bytes, t, nt, 32 % nt);
      if (a.fq) row_in<T>(a.words, p + 3 * g.pitch, a.fq + (size_t)n * a.D, a.D, t, nt, 0);
      else row_in<T>(a.words, p + 3 * g.pitch, (const T*)a.f + o, (int)bytes, t, nt, 96 % nt);
    }
  };
  if (VEC && t == 0)
    for (int k = 0; k < min(rows, g.stages); ++k) fill(k, k);
  if (next_in && rows > 0) fill(0, 0);
  // w_pre and A = beta gate w_post of the block's columns, behind the ring, and where gate groups end within the chunk the
  // post norm's sums over them (every thread reads what it wrote)
  float* const prm = reinterpret_cast<float*>(ring + g.stages * g.stage);
  uint64_t s[VPT][4], z[LN ? VPT : 1][4];                // sums G fh, G of the gate row at hand
  uint64_t dw[VPT][4], db[LN ? VPT : 1][4];              // sums dn xh, dn
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int c = (t + j * nt) * 8;
    uint64_t w[4];
    row8<VEC>(a.nw, c, a.d, 1.f, w);
    if (c < a.D) {
      put_pairs(prm, c, a.D, w);
      const uint64_t none[4] = {0, 0, 0, 0};
      if (!a.per_group) put_pairs(prm + 2 * a.D, c, a.D, none);
      if (LN && !a.per_group) put_pairs(prm + 3 * a.D, c, a.D, none);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[j][i] = dw[j][i] = 0;
      if (LN) z[j][i] = db[j][i] = 0;
    }
  }
  float* const part = a.part ? a.part + (size_t)blockIdx.x * a.slots * a.D : nullptr;
  // gate groups within the chunk: at the end of one its dgate, and its part of the post norm's gradients
  auto flush = [&](int n) {
    const float* gr = a.gate ? a.gate + gate_row(n, a.gate_rows) * a.d : nullptr;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int c = (t + j * nt) * 8;
      if (c >= a.D) continue;
      uint64_t p[4], v[4], gt[4], pb[4];
      float x[8], y[8];
      row8<VEC>(a.pw, c, a.d, 1.f, p);   // every load first
      row8<VEC>(gr, c, a.d, 1.f, gt);
      if (LN) row8<VEC>(a.pb, c, a.d, 0.f, pb);
      if (a.dgate) {
        float* q = a.dgate + gate_row(n, a.gate_rows) * a.d;
        if (a.accumulate) load8<mode_of(VEC)>((const float*)q, c, a.d, y);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[i] = mul2(p[i], s[j][i]);
          if (LN) v[i] = fma2(pb[i], z[j][i], v[i]);
          v[i] = mul2(v[i], f2(a.beta, a.beta));
        }
        unpair(v, x);
        if (a.accumulate) {
#pragma unroll
          for (int i = 0; i < 8; ++i) x[i] += y[i];
        }
        store8<mode_of(VEC)>(q, c, a.d, x);
      }
#pragma unroll
      for (int k = 0; k < (LN ? 2 : 1); ++k) {
        float* q = prm + (2 + k) * a.D;
        get_pairs(q, c, a.D, v);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = fma2(mul2(gt[i], f2(a.beta, a.beta)), k ? z[j][i] : s[j][i], v[i]);
        put_pairs(q, c, a.D, v);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[j][i] = 0;
        if (LN) z[j][i] = 0;
      }
    }
  };
  int turn = 0;
  const float inv_d = 1.f / a.d;
  const uint64_t alpha = f2(a.alpha, a.alpha);
  // statistics and group bytes of the next row, read a row ahead
  float st4[4];
  uint32_t eb[VPT];
  auto ahead = [&](int n) {
#pragma unroll
    for (int i = 0; i < 4; ++i) st4[i] = a.stats[(size_t)i * a.N + n];
    if (a.fq) {
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int c = (t + j * nt) * 8;
        eb[j] = c < a.D ? a.fe[((size_t)n * a.D + c) >> 5] : 0u;
      }
    }
  };
  if (rows > 0) ahead(r0);
  bool new_gate = true;
  int gate_left = min(gate_rows, rows);   // rows of the gate group at hand to come, this one among them
  Turn at;
  int k = 0;
  for (; k < rows; ++k, at.next(g.stages)) {
    const int n = r0 + k, st = at.st;
    const size_t o = (size_t)n * a.d;
    const uint8_t* p = ring + st * g.stage;
    if (new_gate) {
      const float* gr = a.gate ? a.gate + gate_row(n, a.gate_rows) * a.d : nullptr;
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int c = (t + j * nt) * 8;
        uint64_t A[4], p[4];
        row8<VEC>(gr, c, a.d, 1.f, A);
        row8<VEC>(a.pw, c, a.d, 1.f, p);
#pragma unroll
        for (int i = 0; i < 4; ++i) A[i] = mul2(mul2(A[i], f2(a.beta, a.beta)), p[i]);
        cut<VEC>(A, c, a.d);
        if (c < a.D) put_pairs(prm + a.D, c, a.D, A);
      }
      new_gate = false;
    }
    const float pm = st4[0], pr = st4[1], m = st4[2], r = st4[3];
    uint32_t e[VPT];
#pragma unroll
    for (int j = 0; j < VPT; ++j) e[j] = eb[j];
    if (k + 1 < rows) ahead(n + 1);
    if (VEC) {
      wait_row(full, at, abort_flag);
    } else {
      if (!next_in) {
        __syncthreads();
        fill(k, 0);
      }
      row_wait();
      __syncthreads();
    }
    // g, xh and fh of the row, and its sums
    uint64_t G[VPT][4], xh[VPT][4], fh[VPT][4];
    {
      const uint64_t mm = f2(m, m), rr = f2(r, r), prr = f2(pr, pr);
      uint64_t ux = 0, vf = 0, fx = 0, u1 = 0, v1 = 0, af = 0, ax = 0, a1 = 0;
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int c = (t + j * nt) * 8;
#pragma unroll
        for (int i = 0; i < 4; ++i) G[j][i] = xh[j][i] = fh[j][i] = 0;
        if (c >= a.D) continue;
        Raw8<T> rd, rn, rx;
        row_get<VEC>(rd, a.words || !a.dho, p + g.pitch, (const T*)a.dho + o, c, a.d);
        uint64_t u[4], w[4], A[4];
        get_pairs(prm + a.D, c, a.D, A);
        norm_f<T, VEC, LN>(a, p + 3 * g.pitch, (const T*)a.f + o, e[j], c, pm, pr, fh[j]);
        rd.pairs(G[j]);
        if (a.pre) {
          row_get<VEC>(rn, a.words, p, (const T*)a.dn + o, c, a.d);
          row_get<VEC>(rx, a.words, p + 2 * g.pitch, (const T*)a.ho + o, c, a.d);
          get_pairs(prm, c, a.D, w);
          rn.pairs(u);
          rx.pairs(xh[j]);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (LN) {
              xh[j][i] = sub2(xh[j][i], mm);
              db[j][i] = add2(db[j][i], u[i]);
            }
            xh[j][i] = mul2(xh[j][i], rr);
            dw[j][i] = fma2(u[i], xh[j][i], dw[j][i]);
            u[i] = mul2(u[i], w[i]);
            ux = fma2(u[i], xh[j][i], ux);
            if (LN) u1 = add2(u1, u[i]);
            G[j][i] = fma2(rr, u[i], G[j][i]);
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint64_t y = mul2(A[i], fh[j][i]);
          vf = fma2(y, G[j][i], vf);
          fx = fma2(y, xh[j][i], fx);
          if (LN) {
            af = add2(af, y);
            v1 = fma2(A[i], G[j][i], v1);
            ax = fma2(A[i], xh[j][i], ax);
            a1 = add2(a1, A[i]);
          }
        }
      }
      float* const b = &sh[turn][0][0];
      turn ^= 1;
      const float x4[4] = {fold(ux), fold(vf), fold(fx), LN ? fold(u1) : 0.f};
      const float v4 = Reducer::lanes4(x4);
      if ((t & 7) == 0) b[((t & 31) >> 3) * 16 + (t >> 5)] = v4;
      if (LN) {
        const float y4[4] = {fold(v1), fold(af), fold(ax), fold(a1)};
        const float w4 = Reducer::lanes4(y4);
        if ((t & 7) == 0) b[64 + ((t & 31) >> 3) * 16 + (t >> 5)] = w4;
      }
      __syncthreads();
      if (VEC && *abort_flag) break;
      // everyone has the row in registers
      if (VEC && t == 0 && k + g.stages < rows) fill(k + g.stages, st);
      if (next_in && k + 1 < rows) fill(k + 1, st ^ 1);
      float sx[4], sy[4];
      Reducer::warps4(b, sx);
      if (LN) Reducer::warps4(b + 64, sy);
      const float m2 = a.pre ? sx[0] * inv_d : 0.f, m1 = a.pre == ZL_NORM_LAYER ? sx[3] * inv_d : 0.f;
      float q2 = a.post ? (sx[1] - r * m2 * sx[2]) * inv_d : 0.f, q1 = 0.f;
      if (LN) {
        q2 = a.post ? (sx[1] - r * (m1 * sy[1] + m2 * sx[2])) * inv_d : 0.f;
        q1 = a.post == ZL_NORM_LAYER ? (sy[0] - r * (m1 * sy[3] + m2 * sy[2])) * inv_d : 0.f;
      }
      const uint64_t c1 = f2(-r * m1, -r * m1), c2 = f2(-r * m2, -r * m2), d1 = f2(-q1, -q1), d2 = f2(-q2, -q2);
#pragma unroll
      for (int j = 0; j < VPT; ++j) {
        const int c = (t + j * nt) * 8;
        if (VEC && c >= a.d) continue;   // (else every lane stores)
        uint64_t v[4], A[4] = {0, 0, 0, 0};
        if (VEC || c < a.D) get_pairs(prm + a.D, c, a.D, A);
        if (a.pre) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            G[j][i] = fma2(xh[j][i], c2, G[j][i]);
            if (LN) G[j][i] = add2(G[j][i], c1);
          }
          if (!VEC) cut<VEC>(G[j], c, a.d);   // (a vector of VEC is all before d)
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[j][i] = fma2(G[j][i], fh[j][i], s[j][i]);
          if (LN) z[j][i] = add2(z[j][i], G[j][i]);
          v[i] = mul2(G[j][i], alpha);
        }
        if (a.dh) {
          Raw8<T> out;
          pack8(v, out);
          if (VEC) store_raw((T*)a.dh + o, c, a.d, out);
          else store_any((T*)a.dh + o, c, a.d, out);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          v[i] = mul2(A[i], G[j][i]);
          if (a.post) {   // (without a post norm df holds no f: 0 times a NaN or an infinity of it would be NaN)
            v[i] = fma2(fh[j][i], d2, v[i]);
            if (LN) v[i] = add2(v[i], d1);
            v[i] = mul2(v[i], prr);
          }
        }
        Raw8<T> out;
        pack8(v, out);
        if (VEC) store_raw((T*)a.df + o, c, a.d, out);
        else store_any((T*)a.df + o, c, a.d, out);
      }
    }
    if (--gate_left == 0 && !a.per_group) {
      if (part) flush(n);
      new_gate = true;
      gate_left = min(gate_rows, rows - 1 - k);
    }
  }
  if (VEC && k < rows) {
    if (t == 0) drain(full, at, g.stages, min(rows - k, g.stages));
    bwd_give_up<T>(a, k);
    return;
  }
  if (part) {
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int c = (t + j * nt) * 8;
      if (c >= a.D) continue;
      auto put = [&](int slot, const uint64_t* v) {
        float x[8];
        unpair(v, x);
        Vec8<float>::store(part + slot * (size_t)a.D + c, x);
      };
      put(kDw, dw[j]);
      if (!a.per_group) get_pairs(prm + 2 * a.D, c, a.D, s[j]);
      put(kS, s[j]);
      if (LN) {
        if (!a.per_group) get_pairs(prm + 3 * a.D, c, a.D, z[j]);
        put(kDb, db[j]);
        put(kZ, z[j]);
      }
    }
  }
}

// The gradients from the chunks' partial sums: a block takes 32 columns (8 lanes of four), 32 lanes of chunks each adding every
// 32nd one, eight of them under way together, then the lanes' sums in a fixed tree. blockIdx.y 0: the post norm's gradients,
// and dgate where there is one gate group (or none); 1, 2: the pre norm's; 3 + g: dgate of group g where there are a few. Where
// there are more, of fewer chunks each, the lanes of y = 0 take whole groups and write their dgate on the way: 2048 x 4096, 8
// groups of 38 chunks, 28.4 us against 32.5 with blocks for each group (32 groups of 8 chunks 27.4, 54 with blocks and more
// chunks than run at once); 4096 x 768, 8 groups of 95 chunks, 24.4 against 21.4, and 4 of 76 (2048 x 4096) 31.0 against 30.2.
// Bound by latency (launch, one round of loads from L2, stores: 5 us at 128 x 4096): one wave of small blocks, what the last
// step reads besides is read first.
__host__ __device__ __forceinline__ bool many_groups(int groups, int per_group) { return groups > 1 && per_group <= 6 * groups; }
template <bool LN>
__global__ void __launch_bounds__(256) bwd_join_k(const Bwd a) {
  pdl_wait();
  pdl_trigger();
  __shared__ float4 sh[LN ? 2 : 1][32][9];
  constexpr int U = 8;
  const int tx = threadIdx.x & 7, ty = threadIdx.x >> 3, y = blockIdx.y, c = blockIdx.x * 32 + tx * 4;
  const int col = blockIdx.x * 32 + ty;   // of the last step, eight threads to a column
  const int groups = a.per_group ? a.chunks / a.per_group : 1;
  const bool gvec = a.wvec && a.d % 4 == 0 && c < a.d, one = a.per_group && groups == 1, many = many_groups(groups, a.per_group);
  const bool two = LN && (y == 0 || y > 2);
  if (y == 0 ? !a.dpw && !a.dpb && !(a.dgate && (one || many)) : y == 1 ? !a.dnw : y == 2 && !a.dnb) return;
  float pw = 1.f, pb = 0.f, gt = 1.f;
  if (tx == 0 && col < a.d) {
    if (a.pw) pw = a.pw[col];
    if (LN && a.pb) pb = a.pb[col];
    if (one && a.gate) gt = a.gate[col];
  }
  auto four = [&](const float* p, float none) {   // of a row of parameters, at column c
    float4 v = make_float4(none, none, none, none);
    if (!p) return v;
    if (gvec) return *reinterpret_cast<const float4*>(p + c);
    if (c < a.d) v.x = p[c];
    if (c + 1 < a.d) v.y = p[c + 1];
    if (c + 2 < a.d) v.z = p[c + 2];
    if (c + 3 < a.d) v.w = p[c + 3];
    return v;
  };
  auto add = [](float4& s, const float4& v) { s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w; };
  auto scale = [](float4& v, const float4& g) { v.x *= g.x; v.y *= g.y; v.z *= g.z; v.w *= g.w; };
  // the partial sums of chunks b, b + step .. below b1 (at most U of them) at once
  auto load = [&](int slot, int b, int step, int b1, float4* v, float4* w) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      v[u] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (LN) w[u] = v[u];
      if (b + step * u < b1) {
        const float* p = a.part + ((size_t)(b + step * u) * a.slots + slot) * a.D + c;
        v[u] = *reinterpret_cast<const float4*>(p);
        if (two) w[u] = *reinterpret_cast<const float4*>(p + (kZ - kS) * (size_t)a.D);
      }
    }
  };
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f), z = s, v[U], w[LN ? U : 1];
  if (y == 0 && many) {
    const float4 pw4 = four(a.pw, 1.f), pb4 = four(LN ? a.pb : nullptr, 0.f);
    for (int g = ty; g < groups; g += 32) {
      float4 gs = make_float4(0.f, 0.f, 0.f, 0.f), gz = gs;
      const float4 gate = four(a.gate ? a.gate + (size_t)g * a.d : nullptr, 1.f);
      const int end = (g + 1) * a.per_group;
      for (int b = g * a.per_group; b < end; b += U) {
        load(kS, b, 1, end, v, w);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          add(gs, v[u]);
          if (LN) add(gz, w[u]);
        }
      }
      if (a.dgate) {
        float* q = a.dgate + (size_t)g * a.d;
        float4 r = gs;
        scale(r, pw4);
        if (LN) { r.x += pb4.x * gz.x; r.y += pb4.y * gz.y; r.z += pb4.z * gz.z; r.w += pb4.w * gz.w; }
        scale(r, make_float4(a.beta, a.beta, a.beta, a.beta));
        if (a.accumulate) add(r, four(q, 0.f));
        if (gvec) {
          *reinterpret_cast<float4*>(q + c) = r;
        } else {
          if (c < a.d) q[c] = r.x;
          if (c + 1 < a.d) q[c + 1] = r.y;
          if (c + 2 < a.d) q[c + 2] = r.z;
          if (c + 3 < a.d) q[c + 3] = r.w;
        }
      }
      scale(gs, gate);
      add(s, gs);
      if (LN) {
        scale(gz, gate);
        add(z, gz);
      }
    }
    if (!a.dpw && !a.dpb) return;
  } else {
    const int b0 = y > 2 ? (y - 3) * a.per_group : 0, b1 = y > 2 ? b0 + a.per_group : a.chunks;
    const bool weigh = y == 0 && a.per_group && groups > 1 && a.gate;   // every chunk's sums times its gate row
    for (int b = b0 + ty; b < b1; b += 32 * U) {
      load(y == 1 ? kDw : y == 2 ? kDb : kS, b, 32, b1, v, w);
      if (weigh) {
        float4 g[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
          g[u] = four(b + 32 * u < b1 ? a.gate + (size_t)((b + 32 * u) / a.per_group) * a.d : nullptr, 1.f);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          scale(v[u], g[u]);
          if (LN) scale(w[u], g[u]);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        add(s, v[u]);
        if (LN) add(z, w[u]);
      }
    }
  }
  sh[0][ty][tx] = s;
  if (LN) sh[LN ? 1 : 0][ty][tx] = z;
  __syncthreads();
  // column ty of the block's 32: thread tx of eight takes lanes 4 tx .. 4 tx + 3
  float sv = 0.f, zv = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    sv += reinterpret_cast<const float*>(&sh[0][4 * tx + i][0])[ty];
    if (LN) zv += reinterpret_cast<const float*>(&sh[LN ? 1 : 0][4 * tx + i][0])[ty];
  }
#pragma unroll
  for (int o = 4; o > 0; o >>= 1) {
    sv += __shfl_xor_sync(0xffffffffu, sv, o);
    if (LN) zv += __shfl_xor_sync(0xffffffffu, zv, o);
  }
  if (tx != 0 || col >= a.d) return;
  auto put = [&](float* o, float v) {
    if (o) o[col] = a.accumulate ? o[col] + v : v;
  };
  if (y == 1) put(a.dnw, sv);
  else if (y == 2) put(a.dnb, sv);
  else {
    const float dg = a.beta * (pw * sv + pb * zv);
    if (y > 2) put(a.dgate + (size_t)(y - 3) * a.d, dg);
    else {
      if (one) put(a.dgate, dg);
      const float f = a.per_group ? a.beta * gt : 1.f;
      put(a.dpw, f * sv);
      put(a.dpb, f * zv);
    }
  }
}

// Chunks of rows for the partial sums, `slots` of them at most where that is possible (the blocks that run at once): whole gate
// groups together, whose dgate a chunk then writes itself, or where a group has more than twice the rows of an even share,
// groups cut into equal chunks, their dgate joined from these (2048 x 4096 bf16: a gate row for each row 51 us, for 3, 32, 64 rows
// 37, 28, 27; chunks of a fixed length, more than run at once, 47, 78, 54). A row for each chunk only up to 256 rows: beyond, the
// join's reads cost more than a second row (512 x 768 fp32, LayerNorms 12.1 us against 9.0; 128 x 4096 8.5 against 9.5).
void plan_chunks(int N, int gate_rows, int slots, int& rows, int& per_group, int& chunks) {
  const int gr = gate_rows && gate_rows < N ? gate_rows : std::max(N, 1);
  const int share = std::max(N > 256 ? 2 : 1, (N + slots - 1) / slots);
  if (gr > 2 * share) {
    const int groups = (N + gr - 1) / gr;
    per_group = std::min((gr + share - 1) / share, std::max(1, slots / groups));
    rows = (gr + per_group - 1) / per_group;
    per_group = (gr + rows - 1) / rows;
    chunks = groups * per_group;
  } else {
    per_group = 0;
    rows = (share + gr - 1) / gr * gr;
    chunks = (N + rows - 1) / rows;
  }
}
constexpr int kAnyRows = 64;      // rows of a chunk of bwd_cols_k
// (LayerNorm's sums leave no room for two vectors a thread up to 512 threads)
int bwd_threads(int nvec, bool ln) { return ln && nvec <= 512 ? (nvec + 31) / 32 * 32 : ring_threads(nvec); }
// Chunks of bwd_ring_k: as many as blocks fit on 152 SMs at once (4096 x 768, LayerNorms: five an SM 20.8 us, four 21.5).
int ring_slots(int d, bool ln) {
  return 152 * std::max(1, std::min(8, 512 / bwd_threads(pitch(d) / 8, ln)));
}
// What the ring kernel needs behind the ring: w_pre, A, and with gate groups within a chunk the post norm's sums.
size_t bwd_prm(int D, bool ln, int per_group) { return (size_t)D * 4 * (2 + (per_group ? 0 : ln ? 2 : 1)); }
// The chunks, and whether the ring kernel takes the rows: up to 8192 columns, and what does not fit in shared memory not (fp32
// with gate groups that lie whole in a chunk: LayerNorms beyond 7136 columns, RMS norms beyond 8128).
bool plan_chunks(const zl_block_norm& p, int& rows, int& per_group, int& chunks) {
  const bool ln = p.post_norm == ZL_NORM_LAYER || p.pre_norm == ZL_NORM_LAYER;
  if (p.d <= kRingCols) {
    const int D = pitch(p.d);
    plan_chunks(p.N, p.gate_rows, ring_slots(p.d, ln), rows, per_group, chunks);
    if (4 * (size_t)D * dt_size(p.dtype) + bwd_prm(D, ln, per_group) + 4096 <= (size_t)Occupancy::kMaxSmem) return true;
  }
  plan_chunks(p.N, p.gate_rows, std::max(1, (p.N + kAnyRows - 1) / kAnyRows), rows, per_group, chunks);
  return false;
}

template <typename T, int VPT, bool VEC, bool LN>
bool bwd_ring(const Bwd& a, int th, cudaStream_t s) {
  static PerDevice<Occupancy> devices;
  const Occupancy* const found = occupancy(devices, bwd_ring_k<T, VPT, VEC, LN>);
  if (!found) return false;
  const Occupancy& occ = *found;
  Ring g = {};
  const size_t prm = bwd_prm(a.D, LN, a.per_group);
  g.pitch = (uint32_t)a.D * sizeof(T) + (VEC ? 0 : kPhase);
  g.stage = 3 * g.pitch + (a.fq ? (uint32_t)a.D : g.pitch);
  const int want = std::max(1, std::min({2048 / th, 65536 / (occ.regs * th), (a.chunks + sm_count() - 1) / sm_count()}));
  const size_t room = std::max((size_t)(Occupancy::kMaxSmem + 1024) / want, occ.fixed + prm) - occ.fixed - prm;
  g.stages = VEC ? (int)std::min<size_t>(kStages, std::max<size_t>(2, room / g.stage)) : 2;
  if ((size_t)g.stages * g.stage + prm + occ.fixed > (size_t)Occupancy::kMaxSmem) g.stages = 1;
  const size_t smem = (size_t)g.stages * g.stage + prm;
  if (smem + occ.fixed > (size_t)Occupancy::kMaxSmem) return false;
  return launch_pdl(bwd_ring_k<T, VPT, VEC, LN>, a.chunks, th, smem, s, a, g) == cudaSuccess;
}

template <typename T, bool VEC>
bool backward_as(const Bwd& a, cudaStream_t s) {
  const int nvec = a.D / 8;
  const bool ln = a.slots > 2;
  const int groups = a.per_group ? a.chunks / a.per_group : 1;
  const dim3 join((a.D + 31) / 32, 3 + (a.dgate && groups > 1 && !many_groups(groups, a.per_group) ? groups : 0));
  const bool sums = a.dpw || a.dpb || a.dnw || a.dnb || (a.dgate && a.per_group);   // (dgate of short groups is done by then)
  if (a.ring) {
    note_launch(sums ? 2 : 1);
    const int th = bwd_threads(nvec, ln);
    if (th >= nvec) {
      if (!(ln ? bwd_ring<T, 1, VEC, true>(a, th, s) : bwd_ring<T, 1, VEC, false>(a, th, s))) return false;
    } else {
      if (!(ln ? bwd_ring<T, 2, VEC, true>(a, th, s) : bwd_ring<T, 2, VEC, false>(a, th, s))) return false;
    }
    if (sums) launch_pdl(ln ? bwd_join_k<true> : bwd_join_k<false>, join, 256, 0, s, a);
    return true;
  }
  if (a.pre) {
    note_launch(1);
    launch_pdl(bwd_sums_k<T, VEC>, a.N, 256, 0, s, a);
  }
  if (sums || a.dgate) {   // before dh, which may overwrite dh_out
    note_launch(2);
    launch_pdl(bwd_cols_k<T, VEC>, dim3(a.chunks, (a.D + 255) / 256), 256, 0, s, a);
    launch_pdl(ln ? bwd_join_k<true> : bwd_join_k<false>, join, 256, 0, s, a);
  }
  note_launch(1);
  launch_pdl(bwd_rows_k<T, VEC>, a.N, 256, 0, s, a);
  return true;
}
template <typename T>
bool backward(const Bwd& a, cudaStream_t s) {
  return a.vec && a.wvec ? backward_as<T, true>(a, s) : backward_as<T, false>(a, s);
}

int part_slots(const zl_block_norm& p) { return p.post_norm == ZL_NORM_LAYER || p.pre_norm == ZL_NORM_LAYER ? 4 : 2; }

bool dims_ok(const zl_block_norm* p) {
  auto norm = [](int k) { return k >= ZL_NORM_NONE && k <= ZL_NORM_LAYER; };
  return p && (p->dtype == ZL_DTYPE_F32 || p->dtype == ZL_DTYPE_BF16) && norm(p->post_norm) && norm(p->pre_norm) && p->N >= 0 &&
         p->N <= ZL_ACT8_MAX_ROWS && p->d >= 1 && p->d <= ZL_ACT8_MAX_COLS && (long long)p->N * pitch(p->d) / 8 < (1ll << 31) &&
         p->gate_rows >= 0 && p->eps > 0.f && (p->fmt == ZL_ACT8_E4M3 || p->fmt == ZL_ACT8_INT8) &&
         (p->accumulate == 0 || p->accumulate == 1);
}
const char* const kDimsMsg =
    "bad dtype, norm, code format or size (0 <= N <= 2^24, 1 <= d <= 2^20, N x d in whole groups below 2^34, gate_rows >= 0, "
    "eps > 0, accumulate 0 or 1)";
const char* const kElementsMsg = "a tensor off the alignment of its elements";
bool al16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
zl_status ended(bool done, const char* what) {
  const zl_status st = act8::launched(what);
  return done || st != ZL_OK ? st : act8::fail(ZL_ERR_CUDA, (std::string(what) + ": the kernel cannot be launched on this device").c_str());
}

}  // namespace
}  // namespace zl

using namespace zl;
using zl::act8::entry;
using zl::act8::launched;
using zl::act8::on_elements;
using zl::act8::kWhole;
using zl::act8::row_mode;

extern "C" {

zl_status zl_op_block_norm(const zl_block_norm* p, const void* h, const void* f, const float* post_w, const float* post_b,
                           const float* gate, const float* pre_w, const float* pre_b, void* h_out, void* n_out, float* stats,
                           uint8_t* f_q, uint8_t* f_e, uint8_t* n_q, uint8_t* n_e, void* stream) {
  return entry([&]() -> zl_status {
    if (!dims_ok(p)) return act8::fail(ZL_ERR_ARG, kDimsMsg);
    if ((p->post_norm != ZL_NORM_LAYER && post_b) || (p->pre_norm != ZL_NORM_LAYER && pre_b) || (!p->post_norm && post_w) ||
        (!p->pre_norm && pre_w))
      return act8::fail(ZL_ERR_ARG, "a weight without its norm, or a bias without a LayerNorm");
    if (p->N == 0) return ZL_OK;
    if (!h || !f || !h_out || !stats || !n_out != !p->pre_norm)
      return act8::fail(ZL_ERR_ARG, "NULL pointer, or n_out without a pre norm");
    if (!f_q != !f_e || !n_q != !n_e || (n_q && !p->pre_norm) || !al16(f_q) || !al16(n_q))
      return act8::fail(ZL_ERR_ARG, "codes come with their group bytes and 16-byte aligned, n's with a pre norm");
    if (!on_elements({h, f, h_out, n_out}, dt_size(p->dtype)) || !on_elements({post_w, post_b, gate, pre_w, pre_b, stats}, 4))
      return act8::fail(ZL_ERR_ARG, kElementsMsg);
    Fwd a = {};
    a.h = h; a.f = f; a.pw = post_w; a.pb = post_b; a.gate = gate; a.nw = pre_w; a.nb = pre_b;
    a.ho = h_out; a.no = n_out; a.stats = stats; a.fq = f_q; a.fe = f_e; a.nq = n_q; a.ne = n_e;
    a.N = p->N; a.d = p->d; a.D = act8::pitch(p->d); a.post = p->post_norm; a.pre = p->pre_norm; a.gate_rows = p->gate_rows;
    a.eps = p->eps; a.alpha = p->res_scale; a.beta = p->branch_scale; a.fmt = p->fmt;
    a.vec = true;
    a.words = p->d * dt_size(p->dtype) % 4 == 0 && !(((uintptr_t)h | (uintptr_t)f) & 3u);
    for (const void* t : {h, f, (const void*)h_out, (const void*)n_out}) a.vec &= !t || row_mode(t, p->d, p->d, p->dtype) == kWhole;
    a.wvec = al16(post_w) && al16(post_b) && al16(pre_w) && al16(pre_b) && al16(gate);
    const bool done = p->dtype == ZL_DTYPE_BF16 ? forward<bf16>(a, (cudaStream_t)stream) : forward<float>(a, (cudaStream_t)stream);
    return ended(done, "zl_op_block_norm");
  });
}

zl_status zl_op_block_norm_bwd_bytes(const zl_block_norm* p, size_t* bytes) {
  return entry([&]() -> zl_status {
    if (!dims_ok(p) || !bytes) return act8::fail(ZL_ERR_ARG, kDimsMsg);
    int rows, per_group, chunks;
    plan_chunks(*p, rows, per_group, chunks);
    *bytes = p->N ? up256((size_t)p->N * 8) + up256((size_t)chunks * part_slots(*p) * act8::pitch(p->d) * 4) : 0;
    return ZL_OK;
  });
}

zl_status zl_op_block_norm_bwd(const zl_block_norm* p, const void* h_out, const void* f, const uint8_t* f_q, const uint8_t* f_e,
                               const float* post_w, const float* post_b, const float* gate, const float* pre_w, const float* stats,
                               const void* dn, const void* dh_out, void* dh, void* df, float* dpost_w, float* dpost_b,
                               float* dgate, float* dpre_w, float* dpre_b, void* ws, size_t ws_bytes, void* stream) {
  return entry([&]() -> zl_status {
    if (!dims_ok(p)) return act8::fail(ZL_ERR_ARG, kDimsMsg);
    if ((p->post_norm != ZL_NORM_LAYER && (post_b || dpost_b)) || (p->pre_norm != ZL_NORM_LAYER && dpre_b) ||
        (!p->post_norm && (post_w || dpost_w)) || (!p->pre_norm && (pre_w || dpre_w)) || (dgate && !gate))
      return act8::fail(ZL_ERR_ARG,
                        "a weight or its gradient without its norm, a bias gradient without a LayerNorm, or dgate without gate");
    cudaStream_t s = (cudaStream_t)stream;
    const size_t d = (size_t)p->d;
    if (p->N == 0) {
      if (!p->accumulate) {
        for (float* o : {dpost_w, dpost_b, dpre_w, dpre_b, p->gate_rows ? nullptr : dgate})
          if (o && cudaMemsetAsync(o, 0, d * 4, s) != cudaSuccess) return launched("zl_op_block_norm_bwd");
      }
      return ZL_OK;
    }
    if ((!h_out && p->pre_norm) || !stats || !df || !dn != !p->pre_norm || (!dn && !dh_out))
      return act8::fail(ZL_ERR_ARG, "NULL pointer, or dn without a pre norm, or no gradient at all");
    if (!f == !f_q || !f_q != !f_e || !al16(f_q))
      return act8::fail(ZL_ERR_ARG, "f either in dtype or as 16-byte aligned codes with their group bytes");
    if (!on_elements({h_out, f, dn, dh_out, dh, df}, dt_size(p->dtype)) ||
        !on_elements({post_w, post_b, gate, pre_w, stats, dpost_w, dpost_b, dgate, dpre_w, dpre_b}, 4))
      return act8::fail(ZL_ERR_ARG, kElementsMsg);
    size_t need = 0;
    zl_op_block_norm_bwd_bytes(p, &need);
    if (!ws || ((uintptr_t)ws & 255u) || ws_bytes < need)
      return act8::fail(ZL_ERR_ARG, "the workspace must be 256-byte aligned and hold zl_op_block_norm_bwd_bytes() bytes");
    Bwd a = {};
    a.ho = h_out; a.f = f; a.fq = f_q; a.fe = f_e; a.pw = post_w; a.pb = post_b; a.gate = gate; a.nw = pre_w; a.stats = stats;
    a.dn = dn; a.dho = dh_out; a.dh = dh; a.df = df;
    a.s12 = (float*)ws;
    if (dpre_w || dpre_b || dpost_w || dpost_b || dgate) a.part = (float*)((char*)ws + up256((size_t)p->N * 8));
    a.dnw = dpre_w; a.dnb = dpre_b; a.dpw = dpost_w; a.dpb = dpost_b; a.dgate = dgate;
    a.slots = part_slots(*p);
    a.N = p->N; a.d = p->d; a.D = act8::pitch(p->d); a.post = p->post_norm; a.pre = p->pre_norm;
    a.gate_rows = p->gate_rows < p->N ? p->gate_rows : 0;   // one group holds every row
    a.alpha = p->res_scale; a.beta = p->branch_scale; a.fmt = p->fmt; a.accumulate = p->accumulate;
    a.ring = plan_chunks(*p, a.rows, a.per_group, a.chunks);
    a.vec = true;
    a.words = d * dt_size(p->dtype) % 4 == 0 && !(((uintptr_t)h_out | (uintptr_t)f | (uintptr_t)dn | (uintptr_t)dh_out) & 3u);
    for (const void* t : {h_out, f, dn, dh_out, (const void*)dh, (const void*)df})
      a.vec &= !t || row_mode(t, d, d, p->dtype) == kWhole;
    a.wvec = al16(post_w) && al16(post_b) && al16(pre_w) && al16(dgate) && al16(gate);
    const bool done = p->dtype == ZL_DTYPE_BF16 ? backward<bf16>(a, s) : backward<float>(a, s);
    return ended(done, "zl_op_block_norm_bwd");
  });
}

}  // extern "C"
