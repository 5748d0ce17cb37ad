// The 8-bit form of activations (device side): codes of 32 consecutive columns of a row share a power of two.
// For a group with the largest finite magnitude A, E is the smallest integer with A <= Q 2^E and E >= -117 (Q = 448
// for e4m3 codes, 127 for integer ones); a value x is held as the code nearest to x 2^-E (ties to even), and the
// group's byte is E + 127. A power of two keeps the division exact and makes every held value, a code of at most 8
// significant bits times 2^E >= 2^-126, exactly a bf16: reading a checkpoint rounds nothing, in bf16 as in fp32.
// NaN and infinities are held as NaN (code 0x7f, integer code -128); magnitudes above 1.875 2^127 as that value, since
// the next code would be infinite in fp32.
#pragma once
#include <cuda_fp8.h>

#include <string>

#include "common.cuh"
#include "ops.h"

namespace zl {
namespace act8 {

constexpr int kGroup = 32;
constexpr uint32_t kTopBits = 0x7F700000u;    // 1.875 2^127
constexpr uint32_t kInfBits = 0x7F800000u;

__host__ __device__ __forceinline__ int pitch(int d) { return (d + kGroup - 1) / kGroup * kGroup; }

// n / d for 0 <= n < 2^31, d >= 1: with 2^(s-1) < d <= 2^s and m = ceil(2^(31+s) / d) the error of n m / 2^(31+s) against
// n / d is below 1 / d, so the quotient is exact (division by invariant integers, Granlund and Montgomery 1994).
struct FastDiv {
  uint32_t d, mul, shift;
  FastDiv() = default;
  explicit FastDiv(uint32_t div) : d(div), shift(31) {
    while ((1ull << (shift - 31)) < div) ++shift;
    mul = (uint32_t)(((1ull << shift) + div - 1) / div);
  }
  __device__ __forceinline__ uint32_t quot(uint32_t n) const { return (uint32_t)(((uint64_t)n * mul) >> shift); }
};

// E of a group from the bits of its largest magnitude (448 = 1.75 2^8, 127 = 1.984375 2^6).
template <int FMT>
__device__ __forceinline__ int group_exp(uint32_t amax_bits) {
  const int ex = (int)(amax_bits >> 23) - 127;
  const uint32_t man = amax_bits & 0x7FFFFFu;
  const int e = FMT == ZL_ACT8_E4M3 ? ex - 8 + (man > 0x600000u) : ex - 6 + (man > 0x7E0000u);
  return max(e, -117);
}
// 2^k, -126 <= k <= 127.
__device__ __forceinline__ float pow2(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }
// The scale of a group byte.
__device__ __forceinline__ float group_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// Bits of the largest magnitude of N values that a group counts: finite ones, none above the top.
template <int N>
__device__ __forceinline__ uint32_t amax_bits(const float* x) {
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) m = max(m, __float_as_uint(x[i]) & 0x7FFFFFFFu);
  if (m > kTopBits) {   // hardly ever: a NaN, an infinity or a value beyond the top among them
    m = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t u = __float_as_uint(x[i]) & 0x7FFFFFFFu;
      m = max(m, u < kInfBits ? min(u, kTopBits) : 0u);
    }
  }
  return m;
}

// Four codes of four values, given 2^-E of their group.
template <int FMT>
__device__ __forceinline__ uint32_t encode4(const float* x, float inv) {
  const float top = __uint_as_float(kTopBits);
  float y[4];
  bool odd = false;   // a value that the plain conversion would not keep as it should
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    y[i] = x[i] * inv;
    odd |= (__float_as_uint(x[i]) & 0x7FFFFFFFu) > kTopBits;
  }
  if (odd) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t u = __float_as_uint(x[i]) & 0x7FFFFFFFu;
      y[i] = u >= kInfBits ? __uint_as_float(0x7FC00000u) : fminf(fmaxf(x[i], -top), top) * inv;
    }
  }
  if (FMT == ZL_ACT8_E4M3) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(y[0], y[1]), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(y[2], y[3]), __NV_SATFINITE, __NV_E4M3);
    uint32_t w = lo | (hi << 16);
    if (odd) {   // one NaN code: the positive one
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (((w >> (8 * i)) & 0x7Fu) == 0x7Fu) w &= ~(0x80u << (8 * i));
    }
    return w;
  }
  uint32_t w = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int c = odd && y[i] != y[i] ? -128 : __float2int_rn(y[i]);
    w |= ((uint32_t)c & 0xFFu) << (8 * i);
  }
  return w;
}

// The four values of four codes, given their group's 2^E.
template <int FMT>
__device__ __forceinline__ void decode4(uint32_t w, float scale, float* x) {
  if (FMT == ZL_ACT8_E4M3) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> (16 * i)), __NV_E4M3);
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
      x[2 * i] = f.x * scale;
      x[2 * i + 1] = f.y * scale;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i)) * scale;
    const uint32_t v = w ^ 0x80808080u;   // a zero byte where a code is -128
    if ((v - 0x01010101u) & ~v & 0x80808080u) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (((w >> (8 * i)) & 0xFFu) == 0x80u) x[i] = __uint_as_float(0x7FC00000u);
    }
  }
}

// 8 values of a row at column c of d: one or two wide accesses where the row is 16-byte aligned (vec) and has all eight,
// else one value at a time; columns from d on read 0 and are not written.
template <typename T>
__device__ __forceinline__ void load8(const T* p, int c, int d, bool vec, float* f) {
  if (vec && c + 8 <= d) {
    Vec8<T>::load(p + c, f);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = c + i < d ? to_f(p[c + i]) : 0.f;
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int c, int d, bool vec, const float* f) {
  if (vec && c + 8 <= d) {
    Vec8<T>::store(p + c, f);
    return;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (c + i < d) p[c + i] = from_f<T>(f[i]);
}

// Encodes this thread's 8 values as its quarter of a group (the four lanes 4 g .. 4 g + 3 of the warp hold the group,
// every lane of the warp calls): returns the codes in q and E + 127.
template <int FMT>
__device__ __forceinline__ uint32_t encode_quarter(const float* x, uint2& q) {
  uint32_t m = amax_bits<8>(x);
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
  const int E = group_exp<FMT>(m);
  const float inv = pow2(-E);
  q.x = encode4<FMT>(x, inv);
  q.y = encode4<FMT>(x + 4, inv);
  return (uint32_t)(E + 127);
}
template <int FMT>
__device__ __forceinline__ void decode8(uint2 q, uint32_t e, float* x) {
  const float s = group_scale(e);
  decode4<FMT>(q.x, s, x);
  decode4<FMT>(q.y, s, x + 4);
}

// Runs the body of a C entry point: no exception leaves it.
template <typename F>
zl_status entry(F&& body) {
  try {
    return body();
  } catch (...) {
    return ZL_ERR_CUDA;
  }
}
inline zl_status fail(zl_status st, const char* msg) {
  set_last_error(msg);
  return st;
}
inline zl_status launched(const char* what) {
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? ZL_OK : fail(ZL_ERR_CUDA, (std::string(what) + ": " + cudaGetErrorString(e)).c_str());
}

// Whether rows of ld values from p can be read 16 bytes at a time.
inline bool rows_aligned(const void* p, size_t ld, int dt) {
  return ((uintptr_t)p & 15u) == 0 && ld * (dt == ZL_DTYPE_BF16 ? 2 : 4) % 16 == 0;
}

}  // namespace act8
}  // namespace zl
