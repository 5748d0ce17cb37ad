// Sums over a vocabulary (device side): running log-sum-exps in base 2, the mean of the rows' losses.
#pragma once
#include "common.cuh"

namespace zl {
namespace vocab {

constexpr float kL2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// 2^x by the SFU's ex2.approx (relative error about 2^-22; results below 2^-126 become 0).
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// sum e^{x / T} = s e^{m / T}, with m the largest x so far (-inf, 0: the empty sum); scale = log2 e / T. Exponents are (x - m) scale, the
// difference first: it is exact or nearly so, while x scale - m scale carries the rounding of numbers of the size of x / T, which at a
// low temperature is larger than the exponent (T = 1e-6, logits of 20: a probability of 4 instead of 1). m stays in the units of x.
struct Lse {
  float m, s;
};
__device__ __forceinline__ Lse lse_empty() { return Lse{-INFINITY, 0.f}; }
__device__ __forceinline__ void lse_raise(Lse& A, float m, float scale) {
  if (m > A.m) {
    A.s *= ex2((A.m - m) * scale);
    A.m = m;
  }
}
// What is taken off an exponent's x: m, or 0 where nothing but -inf has come.
__device__ __forceinline__ float lse_ref(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ void lse_add1(Lse& A, float x, float scale) {
  lse_raise(A, x, scale);
  A.s += ex2((x - lse_ref(A.m)) * scale);
}
// N values whose largest is mx (NaN if one is). With m scale below kNear one FMA instead: its rounding is that of the log-sum-exp itself
// (under the products' epilogue 3% of their time).
constexpr float kNear = 4096.f;
template <int N>
__device__ __forceinline__ void lse_add(Lse& A, const float (&x)[N], float mx, float scale) {
  lse_raise(A, mx, scale);
  const float m = lse_ref(A.m), b = m * scale;
  const uint64_t s2 = f2(scale, scale);
  uint64_t t = 0ull;
  if (fabsf(b) < kNear) {
    const uint64_t nb = f2(-b, -b);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const float2 v = uf2(fma2(f2(x[2 * i], x[2 * i + 1]), s2, nb));
      const uint64_t e = f2(ex2(v.x), ex2(v.y));
      t = i == 0 ? e : add2(t, e);
    }
  } else {
    const uint64_t nm = f2(-m, -m);
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
      const float2 v = uf2(mul2(add2(f2(x[2 * i], x[2 * i + 1]), nm), s2));
      const uint64_t e = f2(ex2(v.x), ex2(v.y));
      t = i == 0 ? e : add2(t, e);
    }
  }
  const float2 v = uf2(t);
  A.s += v.x + v.y;
}
// The same for many values a thread, in as few instructions as may be (a loop whose rare paths are long waits for its
// instructions): the sum's reference m is raised only when a value would lie more than 2^kSlack above it.
struct LseRun {
  float m, limit, nm;   // reference, the value up to which it holds, -m (0 while m is -inf)
  uint64_t s;           // two lanes
  float slack;
};
constexpr float kSlack = 24.f;
__device__ __forceinline__ LseRun run_empty(float scale) { return LseRun{-INFINITY, -INFINITY, 0.f, 0ull, kSlack / scale}; }
template <int N>
__device__ __forceinline__ void run_add(LseRun& A, const float (&x)[N], float mx, float scale) {
  if (!(mx <= A.limit)) {   // (a NaN stays in the sum)
    const float c = A.m == -INFINITY ? 0.f : ex2((A.m - mx) * scale);
    A.s = mul2(A.s, f2(c, c));
    A.m = mx;
    A.nm = -mx;
    A.limit = mx + A.slack;
  }
  const uint64_t s2 = f2(scale, scale), nm = f2(A.nm, A.nm);
  uint64_t t = 0ull;
#pragma unroll
  for (int i = 0; i < N / 2; ++i) {
    const float2 v = uf2(mul2(add2(f2(x[2 * i], x[2 * i + 1]), nm), s2));
    const uint64_t e = f2(ex2(v.x), ex2(v.y));
    t = i == 0 ? e : add2(t, e);
  }
  A.s = add2(A.s, t);
}
__device__ __forceinline__ Lse run_sum(const LseRun& A) {
  const float2 s = uf2(A.s);
  return A.m == -INFINITY ? lse_empty() : Lse{A.m, s.x + s.y};
}
__device__ __forceinline__ Lse lse_merge(Lse a, Lse b, float scale) {
  const float M = fmaxf(a.m, b.m);
  if (M == -INFINITY) return Lse{M, a.s + b.s};
  return Lse{M, a.s * ex2((a.m - M) * scale) + b.s * ex2((b.m - M) * scale)};
}
// The merged sum of the warp, for every lane: the largest reference first (floats as integers of the same order), then one sum.
__device__ __forceinline__ Lse warp_merge(Lse v, float scale) {
  const int i = __float_as_int(v.m);
  const int top = __reduce_max_sync(0xffffffffu, i ^ ((i >> 31) & 0x7FFFFFFF));
  const float M = __int_as_float(top ^ ((top >> 31) & 0x7FFFFFFF));
  return Lse{M, warp_sum(M == -INFINITY ? v.s : v.s * ex2((v.m - M) * scale))};
}
// log sum e^{x / T} (-inf of the empty sum).
__device__ __forceinline__ float lse_value(const Lse& A, float inv_T) { return A.m * inv_T + log2f(A.s) * kLn2; }

// dloss / |Omega|, the weight of a row of Omega (dloss NULL: 1; 0 without rows).
__device__ __forceinline__ float loss_weight(const float* omega, const float* dloss) {
  const float om = *omega;
  return om > 0.f ? (dloss ? *dloss : 1.f) / om : 0.f;
}

// A 16-byte word of T from floats (bf16: rounded to nearest even).
__device__ __forceinline__ uint4 pack_word(const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<const uint32_t*>(&h);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 pack_word(const float (&x)[4]) {
  return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}

// By one block of up to 1024 threads, in a fixed order, sums in fp64: loss[1] = |Omega| = #(0 <= labels < V) (part 1), loss[0] =
// sum(row_loss) / |Omega| (part 2, 0 without rows in Omega; by the |Omega| that is in loss[1], or with part 3 both). row_loss may have been
// written by other blocks of the same launch: no __restrict__, which would allow loads that need not see them.
__device__ __forceinline__ void finish_loss(const float* row_loss, const int32_t* __restrict__ labels, int N, int V,
                                            float* loss, int part) {
  __shared__ double sum[32];
  __shared__ int num[32];
  double acc = 0.0;
  int n = 0;
#pragma unroll 1
  for (int i0 = threadIdx.x; i0 < N; i0 += 4 * (int)blockDim.x) {
    float v[4];
    int l[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const int i = i0 + q * (int)blockDim.x;
      v[q] = (part & 2) && i < N ? row_loss[i] : 0.f;
      l[q] = (part & 1) && i < N ? labels[i] : -1;
    }
    acc += ((double)v[0] + (double)v[1]) + ((double)v[2] + (double)v[3]);
#pragma unroll
    for (int q = 0; q < 4; ++q) n += l[q] >= 0 && l[q] < V;
  }
  n = __reduce_add_sync(0xffffffffu, n);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (lane == 0) {
    sum[warp] = acc;
    num[warp] = n;
  }
  __syncthreads();
  if (warp == 0) {
    const bool in = lane < ((int)blockDim.x >> 5);
    acc = in ? sum[lane] : 0.0;
    n = __reduce_add_sync(0xffffffffu, in ? num[lane] : 0);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
    if (lane == 0) {
      const float count = (part & 1) ? (float)n : loss[1];   // exact up to 2^24
      if (part & 1) loss[1] = count;
      if (part & 2) loss[0] = count > 0.f ? (float)(acc / (double)count) : 0.f;
    }
  }
}

}  // namespace vocab
}  // namespace zl
