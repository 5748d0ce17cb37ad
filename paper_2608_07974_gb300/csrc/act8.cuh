// The 8-bit form of activations (device side): codes of 32 consecutive columns of a row share a power of two.
// For a group with the largest finite magnitude A, E is the smallest integer with A <= Q 2^E and E >= -117 (Q = 448
// for e4m3 codes, 127 for integer ones); a value x is held as the code nearest to x 2^-E (ties to even), and the
// group's byte is E + 127. A power of two keeps the division exact and makes every held value, a code of at most 8
// significant bits times 2^E >= 2^-126, exactly a bf16: reading a checkpoint rounds nothing, in bf16 as in fp32.
// NaN and infinities are held as NaN (code 0x7f, integer code -128); magnitudes above 1.875 2^127 as that value, since
// the next code would be infinite in fp32.
#pragma once
#include <cuda_fp8.h>

#include <exception>
#include <initializer_list>
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

// E + 127 of a group from the bits of its largest magnitude (448 = 1.75 2^8, 127 = 1.984375 2^6): the exponent, one up
// where the mantissa is above Q's, which the addition carries into it.
template <int FMT>
__device__ __forceinline__ uint32_t group_byte(uint32_t amax_bits) {
  const int e = FMT == ZL_ACT8_E4M3 ? (int)((amax_bits + 0x1FFFFFu) >> 23) - 8 : (int)((amax_bits + 0x1FFFFu) >> 23) - 6;
  return (uint32_t)max(e, 10);
}
// The scale of a group byte.
__device__ __forceinline__ float group_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
// And its inverse (bytes 10 .. 249).
__device__ __forceinline__ float group_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// max(|a|, |b|, |c|), a NaN if one is among them.
__device__ __forceinline__ float absmax3(float a, float b, float c) {
  float r;
  asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
// Bits of the largest magnitude of 8 values (of a NaN if one is among them).
__device__ __forceinline__ uint32_t amax_bits(const float* x) {
  float v = absmax3(x[0], x[1], x[2]);
  v = absmax3(v, x[3], x[4]);
  v = absmax3(v, x[5], x[6]);
  return __float_as_uint(absmax3(v, x[7], x[7]));
}
// Four codes of four numbers. Integer codes: adding 1.5 2^23 rounds to the nearest integer, ties to even, and leaves it in
// the low bits.
template <int FMT>
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  if (FMT == ZL_ACT8_E4M3) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
    return __byte_perm(lo, hi, 0x5410);
  }
  const uint32_t x = __float_as_uint(a + 12582912.f), y = __float_as_uint(b + 12582912.f);
  const uint32_t z = __float_as_uint(c + 12582912.f), w = __float_as_uint(d + 12582912.f);
  return __byte_perm(__byte_perm(x, y, 0x0040), __byte_perm(z, w, 0x0040), 0x5410);
}

// The four numbers that four codes are (not yet times 2^E). Integer codes: code + 128 as the low mantissa byte of 2^23,
// less 2^23 + 128.
template <int FMT>
__device__ __forceinline__ void codes4(uint32_t w, float* x) {
  if (FMT == ZL_ACT8_E4M3) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> (16 * i)), __NV_E4M3);
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
      x[2 * i] = f.x;
      x[2 * i + 1] = f.y;
    }
  } else {
    const uint32_t v = w ^ 0x80808080u;
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(__byte_perm(v, 0x4B000000u, 0x7540 + i)) - 8388736.f;
    if ((v - 0x01010101u) & ~v & 0x80808080u) {   // a zero byte: a code of -128
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (((v >> (8 * i)) & 0xFFu) == 0u) x[i] = __uint_as_float(0x7FC00000u);
    }
  }
}

// The 16 bytes from byte b (0 .. 15) of two neighbouring 16-byte words on; b a multiple of 2 (HALF) or of 4.
template <bool HALF>
__device__ __forceinline__ uint4 shift16(const uint4& lo, const uint4& hi, uint32_t b) {
  uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
  const bool two = b & 8u, one = b & 4u;
#pragma unroll
  for (int i = 0; i < 6; ++i) w[i] = two ? w[i + 2] : w[i];
#pragma unroll
  for (int i = 0; i < 5; ++i) w[i] = one ? w[i + 1] : w[i];
  if (HALF) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], (b & 2u) << 3);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// 8 values of a row at column c of d. MODE kWhole: rows start on 16 bytes and d is a multiple of 8; kTail: rows start on 16
// bytes, and all but a row's last few values are read 16 bytes at a time; kSingle: rows start anywhere, their values are read
// in the 16-byte words around them, those near its ends one at a time. Columns from d on read 0 and are not written. What is
// loaded stays packed until it is used, so that the loads of a thread are all under way before the first of them is waited for.
enum { kSingle = 0, kTail = 1, kWhole = 2 };
template <typename T>
struct Raw8;
template <>
struct Raw8<bf16> {
  uint4 u;
  __device__ __forceinline__ void zero() { u = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void get(const void* p) { u = *reinterpret_cast<const uint4*>(p); }
  // from any address of a bf16 (the 16-byte words around it are read)
  __device__ __forceinline__ void get_around(const void* p) {
    const uint32_t b = (uint32_t)(uintptr_t)p & 15u;
    from_words(reinterpret_cast<const uint4*>((const char*)p - b), b);
  }
  __device__ __forceinline__ void from_words(const uint4* w, uint32_t b) { u = shift16<true>(w[0], w[1], b); }
  __device__ __forceinline__ void words(uint4* w) const { w[0] = u; }
  __device__ __forceinline__ void set(void* p) const { *reinterpret_cast<uint4*>(p) = u; }
  __device__ __forceinline__ void pairs(uint64_t* f) const {
    f[0] = bf2_to_f2(u.x); f[1] = bf2_to_f2(u.y); f[2] = bf2_to_f2(u.z); f[3] = bf2_to_f2(u.w);
  }
  __device__ __forceinline__ void trim(int n) {   // zeros but for the first n
    auto keep = [n](int i) { return n >= i + 2 ? ~0u : n == i + 1 ? 0xFFFFu : 0u; };
    u.x &= keep(0); u.y &= keep(2); u.z &= keep(4); u.w &= keep(6);
  }
  __device__ __forceinline__ void put(int i, bf16 v) {
    const uint32_t b = __bfloat16_as_ushort(v);
    uint32_t& w = i < 2 ? u.x : i < 4 ? u.y : i < 6 ? u.z : u.w;
    w |= i & 1 ? b << 16 : b;
  }
};
template <>
struct Raw8<float> {
  float4 u, v;
  __device__ __forceinline__ void zero() { u = v = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ __forceinline__ void get(const void* p) {
    u = reinterpret_cast<const float4*>(p)[0];
    v = reinterpret_cast<const float4*>(p)[1];
  }
  __device__ __forceinline__ void get_around(const void* p) {
    const uint32_t b = (uint32_t)(uintptr_t)p & 15u;
    from_words(reinterpret_cast<const uint4*>((const char*)p - b), b);
  }
  __device__ __forceinline__ void words(uint4* w) const {
    w[0] = make_uint4(__float_as_uint(u.x), __float_as_uint(u.y), __float_as_uint(u.z), __float_as_uint(u.w));
    w[1] = make_uint4(__float_as_uint(v.x), __float_as_uint(v.y), __float_as_uint(v.z), __float_as_uint(v.w));
  }
  __device__ __forceinline__ void from_words(const uint4* w, uint32_t b) {
    const uint4 lo = shift16<false>(w[0], w[1], b), hi = shift16<false>(w[1], w[2], b);
    u = make_float4(__uint_as_float(lo.x), __uint_as_float(lo.y), __uint_as_float(lo.z), __uint_as_float(lo.w));
    v = make_float4(__uint_as_float(hi.x), __uint_as_float(hi.y), __uint_as_float(hi.z), __uint_as_float(hi.w));
  }
  __device__ __forceinline__ void set(void* p) const {
    reinterpret_cast<float4*>(p)[0] = u;
    reinterpret_cast<float4*>(p)[1] = v;
  }
  __device__ __forceinline__ void pairs(uint64_t* f) const {
    f[0] = f2(u.x, u.y); f[1] = f2(u.z, u.w); f[2] = f2(v.x, v.y); f[3] = f2(v.z, v.w);
  }
  __device__ __forceinline__ void trim(int n) {
    auto keep = [n](int i, float& x) { if (i >= n) x = 0.f; };
    keep(0, u.x); keep(1, u.y); keep(2, u.z); keep(3, u.w); keep(4, v.x); keep(5, v.y); keep(6, v.z); keep(7, v.w);
  }
  __device__ __forceinline__ void put(int i, float x) {
    (i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : i == 3 ? u.w : i == 4 ? v.x : i == 5 ? v.y : i == 6 ? v.z : v.w) = x;
  }
};
__device__ __forceinline__ void unpair(const uint64_t* p, float* f) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 v = uf2(p[i]);
    f[2 * i] = v.x;
    f[2 * i + 1] = v.y;
  }
}
template <int MODE, typename T>
__device__ __forceinline__ Raw8<T> load_raw(const T* p, int c, int d) {
  Raw8<T> r;
  if (MODE == kWhole) {
    if (c < d) r.get(p + c);
    else r.zero();
  } else if (MODE == kTail && c + 8 <= d) {
    r.get(p + c);
  } else {
    if (MODE == kSingle) {
      const int s = (int)(((uintptr_t)(p + c) & 15u) / sizeof(T));   // values of the row before these in their first word
      if (s <= c && c - s + 8 + 16 / (int)sizeof(T) <= d) {
        r.get_around(p + c);
        return r;
      }
    }
    r.zero();
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (c + i < d) r.put(i, p[c + i]);
  }
  return r;
}
// Rounds pairs to T.
__device__ __forceinline__ void pack8(const uint64_t* v, Raw8<bf16>& r) {
  auto two = [](uint64_t p) {
    const float2 f = uf2(p);
    const __nv_bfloat162 h = __floats2bfloat162_rn(f.x, f.y);
    return *reinterpret_cast<const uint32_t*>(&h);
  };
  r.u = make_uint4(two(v[0]), two(v[1]), two(v[2]), two(v[3]));
}
__device__ __forceinline__ void pack8(const uint64_t* v, Raw8<float>& r) {
  const float2 a = uf2(v[0]), b = uf2(v[1]), c = uf2(v[2]), d = uf2(v[3]);
  r.u = make_float4(a.x, a.y, b.x, b.y);
  r.v = make_float4(c.x, c.y, d.x, d.y);
}
template <typename T>
__device__ __forceinline__ void floats(const Raw8<T>& r, float* f) {
  uint64_t p[4];
  r.pairs(p);
  unpair(p, f);
}
template <int MODE, typename T>
__device__ __forceinline__ void load8(const T* p, int c, int d, float* f) {
  floats(load_raw<MODE>(p, c, d), f);
}
// What load_raw reads, packed until floats() asks for it: the 16-byte words around the values where they start anywhere, so
// that the shift does not wait for them where they are loaded.
template <int MODE, typename T>
struct Piece {
  Raw8<T> r;
  __device__ __forceinline__ void load(const T* p, int c, int d) { r = load_raw<MODE>(p, c, d); }
  __device__ __forceinline__ void floats(float* f) const { act8::floats(r, f); }
};
template <typename T>
struct Piece<kSingle, T> {
  static constexpr int W = sizeof(T) == 2 ? 2 : 3;
  uint4 w[W];
  uint32_t b;
  __device__ __forceinline__ void load(const T* p, int c, int d) {
    b = (uint32_t)(uintptr_t)(p + c) & 15u;
    const int s = (int)b / (int)sizeof(T);
    if (s <= c && c - s + 8 + 16 / (int)sizeof(T) <= d) {
      const uint4* q = reinterpret_cast<const uint4*>((const char*)(p + c) - b);
#pragma unroll
      for (int i = 0; i < W; ++i) w[i] = q[i];
    } else {
      Raw8<T> r;
      r.zero();
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (c + i < d) r.put(i, p[c + i]);
      r.words(w);
      w[W - 1] = make_uint4(0, 0, 0, 0);
      b = 0;
    }
  }
  __device__ __forceinline__ void floats(float* f) const {
    Raw8<T> r;
    r.from_words(w, b);
    act8::floats(r, f);
  }
};
// Rows of whole vectors (kWhole).
template <typename T>
__device__ __forceinline__ void store_raw(T* p, int c, int d, const Raw8<T>& r) {
  if (c < d) r.set(p + c);
}
template <int MODE, typename T>
__device__ __forceinline__ void store8(T* p, int c, int d, const float* f) {
  if (MODE == kWhole ? c < d : MODE == kTail && c + 8 <= d) {
    Vec8<T>::store(p + c, f);
    return;
  }
  if (MODE == kWhole) return;
#pragma unroll
  for (int i = 0; i < 8; ++i)
    if (c + i < d) p[c + i] = from_f<T>(f[i]);
}

// 8 values of a row that starts anywhere, at column c of d, by a warp whose lanes hold neighbouring columns (where the next one
// is of the same row; every lane calls, with d = 0 one that has none): a lane writes the 16-byte words that begin in its
// columns, which end in those of the next lane. Only values before the row's or the warp's first word or behind its last one
// go one at a time.
template <typename T>
__device__ __forceinline__ void store_any(T* p, int c, int d, const Raw8<T>& r) {
  const int lane = threadIdx.x & 31;
  const int h = (int)((0u - (uint32_t)(uintptr_t)(p + c)) & 15u) / (int)sizeof(T);   // values before the first word
  constexpr int W = sizeof(T) / 2;
  uint4 w[W + 1];
  r.words(w);
  uint4& next = w[W];
  next = w[0];
  next.x = __shfl_down_sync(0xffffffffu, next.x, 1);
  next.y = __shfl_down_sync(0xffffffffu, next.y, 1);
  next.z = __shfl_down_sync(0xffffffffu, next.z, 1);
  if (sizeof(T) == 2) next.w = __shfl_down_sync(0xffffffffu, next.w, 1);
  const bool words = c + h + 8 <= d && (h == 0 || lane < 31);
  if (words) {
#pragma unroll
    for (int i = 0; i < W; ++i)
      reinterpret_cast<uint4*>(p + c + h)[i] = shift16<sizeof(T) == 2>(w[i], w[i + 1], h * (uint32_t)sizeof(T));
  }
  // what neither this lane's words nor those of the lane before hold
  const int from = lane > 0 && c > 0 && c + h <= d ? h : 0, to = words ? h : min(8, d - c);
  if (from < to) {
    float f[8];
    floats(r, f);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i >= from && i < to) p[c + i] = from_f<T>(f[i]);
  }
}

// Encodes this thread's 8 values as its quarter of a group (the four lanes 4 g .. 4 g + 3 of the warp hold the group,
// every lane of the warp calls): the codes in q, returns E + 127.
template <int FMT>
__device__ __forceinline__ uint32_t encode_quarter(const float* x, uint2& q) {
  const uint32_t mine = amax_bits(x);
  uint32_t m = max(mine, __shfl_xor_sync(0xffffffffu, mine, 1));
  m = max(m, __shfl_xor_sync(0xffffffffu, m, 2));
  if (__any_sync(0xffffffffu, m > kTopBits)) {   // hardly ever: a NaN, an infinity or a value beyond the top in the warp
    uint32_t v = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint32_t u = __float_as_uint(x[i]) & 0x7FFFFFFFu;
      v = max(v, u < kInfBits ? min(u, kTopBits) : 0u);
    }
    v = max(v, __shfl_xor_sync(0xffffffffu, v, 1));
    v = max(v, __shfl_xor_sync(0xffffffffu, v, 2));
    const uint32_t byte = group_byte<FMT>(v);
    const float inv = group_inverse(byte), top = __uint_as_float(kTopBits);
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = fminf(fmaxf(x[i], -top), top) * inv;
    uint32_t w[2] = {encode4<FMT>(y[0], y[1], y[2], y[3]), encode4<FMT>(y[4], y[5], y[6], y[7])};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if ((__float_as_uint(x[i]) & 0x7FFFFFFFu) >= kInfBits)
        w[i >> 2] = (w[i >> 2] & ~(0xFFu << (8 * (i & 3)))) | ((FMT == ZL_ACT8_E4M3 ? 0x7Fu : 0x80u) << (8 * (i & 3)));
    }
    q = make_uint2(w[0], w[1]);
    return byte;
  }
  const uint32_t byte = group_byte<FMT>(m);
  const float inv = group_inverse(byte);
  q.x = encode4<FMT>(x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv);
  q.y = encode4<FMT>(x[4] * inv, x[5] * inv, x[6] * inv, x[7] * inv);
  return byte;
}
template <int FMT>
__device__ __forceinline__ void decode8(uint2 q, uint32_t e, float* x) {
  const float s = group_scale(e);
  codes4<FMT>(q.x, x);
  codes4<FMT>(q.y, x + 4);
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] *= s;
}

// Runs the body of a C entry point: no exception leaves it.
template <typename F>
zl_status entry(F&& body) {
  try {
    return body();
  } catch (const std::exception& e) {   // (out of host memory)
    try {
      set_last_error(e.what());
    } catch (...) {
    }
  } catch (...) {
  }
  return ZL_ERR_CUDA;
}
inline zl_status fail(zl_status st, const char* msg) {
  set_last_error(msg);
  return st;
}
inline zl_status launched(const char* what) {
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? ZL_OK : fail(ZL_ERR_CUDA, (std::string(what) + ": " + cudaGetErrorString(e)).c_str());
}

// Bytes of a workspace's piece, so that the next one starts on 256.
inline size_t up256(size_t b) { return (b + 255) / 256 * 256; }
// Whether every pointer lies on elements of that many bytes (a kernel faults on others).
inline bool on_elements(std::initializer_list<const void*> ps, size_t bytes) {
  for (const void* p : ps)
    if ((uintptr_t)p % bytes) return false;
  return true;
}
// The mode of rows of d values from p, ld apart.
inline int row_mode(const void* p, size_t d, size_t ld, int dt) {
  if (((uintptr_t)p & 15u) || ld * (dt == ZL_DTYPE_BF16 ? 2 : 4) % 16) return kSingle;
  return d % 8 ? kTail : kWhole;
}

}  // namespace act8
}  // namespace zl
