// Activations kept in 8 bits between a chunk's forward and its local backward (zl_op_act8_*): rows written and read
// back, the activation functions that write the checkpoint of their input in the same pass and whose backward reads
// it, and the weight gradient of a linear from the checkpoint of its input. Form of the codes: act8.cuh.
#include <algorithm>

#include "act8.cuh"
#include "ops.h"

namespace zl {

namespace {
using namespace act8;

constexpr int kThreads = 256;

// Items of a kernel over the 8-column pieces of N rows in whole groups, four neighbouring lanes to a group: every lane of
// a warp runs the loop, `in` says whether its item exists.
struct Items {
  uint32_t n;      // N * D / 8, below 2^31
  FastDiv row;     // D / 8 pieces to a row
};

// ------------------------------------------------------------------------------------------------
// Rows to 8 bits and back. HBM-bound: 3.03 bytes a value in bf16, 5.03 in fp32.
// ------------------------------------------------------------------------------------------------
template <typename T, int FMT>
__global__ void __launch_bounds__(kThreads) store_k(const T* __restrict__ x, size_t ldx, int d, bool vec, Items it,
                                                    uint2* __restrict__ q, uint8_t* __restrict__ e) {
  pdl_wait();
  pdl_trigger();
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
  const bool in = i < it.n;
  float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (in) {
    const uint32_t r = it.row.quot(i);
    load8(x + r * ldx, (int)(i - r * it.row.d) * 8, d, vec, f);
  }
  uint2 w;
  const uint32_t b = encode_quarter<FMT>(f, w);
  if (in) {
    q[i] = w;
    if ((i & 3u) == 0) e[i >> 2] = (uint8_t)b;
  }
}

template <typename T, int FMT>
__global__ void __launch_bounds__(kThreads) load_k(const uint2* __restrict__ q, const uint8_t* __restrict__ e, Items it,
                                                   T* __restrict__ x, size_t ldx, int d, bool vec) {
  pdl_wait();
  pdl_trigger();
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= it.n) return;
  const uint32_t r = it.row.quot(i);
  float f[8];
  decode8<FMT>(q[i], e[i >> 2], f);
  store8(x + r * ldx, (int)(i - r * it.row.d) * 8, d, vec, f);
}

// ------------------------------------------------------------------------------------------------
// Activations. SwiGLU: y = g s u, s = 1 / (1 + e^-g); dg = dy u s (1 + g (1 - s)), du = dy g s. GELU (tanh form):
// y = x s(2a), a = k (x + c x^3), k = sqrt(2 / pi), c = 0.044715 (0.5 (1 + tanh a) = s(2a));
// dx = dy (s + 2 x s (1 - s) k (1 + 3 c x^2)). bf16: e^x and the reciprocal by the fast instructions (a few fp32 ulp,
// far below the rounding to bf16); fp32: expf and a true division.
// ------------------------------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ float sigm(float x) {
  if (sizeof(T) == 2) return rcp_approx(1.f + __expf(-x));
  return 1.f / (1.f + expf(-x));
}
constexpr float kGeluK = 0.7978845608028654f, kGeluC = 0.044715f;

// x [N, f] (GELU) or [N, 2 f] (SwiGLU: gate, up); codes of the rows of f values: [N, D] or [N, 2 D], D = pitch(f).
template <typename T, int FMT, int ACT>
__global__ void __launch_bounds__(kThreads) act_k(const T* __restrict__ x, int f, bool vec, Items it, T* __restrict__ y,
                                                  uint2* __restrict__ q, uint8_t* __restrict__ e) {
  constexpr int W = ACT == ZL_ACT_SWIGLU ? 2 : 1;
  pdl_wait();
  pdl_trigger();
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
  const bool in = i < it.n;
  const uint32_t r = in ? it.row.quot(i) : 0, c8 = i - r * it.row.d;
  const int c = (int)c8 * 8;
  float g[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f}, u[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (in) {
    const T* xr = x + (size_t)r * W * f;
    load8(xr, c, f, vec, g);
    if (W == 2) load8(xr + f, c, f, vec, u);
  }
  uint2 w;
  uint32_t b = encode_quarter<FMT>(g, w);
  size_t at = (size_t)r * W * it.row.d + c8;
  if (in) {
    q[at] = w;
    if ((c8 & 3u) == 0) e[at >> 2] = (uint8_t)b;
  }
  if (W == 2) {
    b = encode_quarter<FMT>(u, w);
    at += it.row.d;
    if (in) {
      q[at] = w;
      if ((c8 & 3u) == 0) e[at >> 2] = (uint8_t)b;
    }
  }
  if (!in) return;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (W == 2) g[k] = g[k] * sigm<T>(g[k]) * u[k];
    else g[k] = g[k] * sigm<T>(2.f * kGeluK * (g[k] + kGeluC * g[k] * g[k] * g[k]));
  }
  store8(y + (size_t)r * f, c, f, vec, g);
}

template <typename T, int FMT, int ACT>
__global__ void __launch_bounds__(kThreads) act_bwd_k(const uint2* __restrict__ q, const uint8_t* __restrict__ e,
                                                      const T* __restrict__ dy, int f, bool vec, Items it,
                                                      T* __restrict__ dx, T* __restrict__ y) {
  constexpr int W = ACT == ZL_ACT_SWIGLU ? 2 : 1;
  pdl_wait();
  pdl_trigger();
  const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
  if (i >= it.n) return;
  const uint32_t r = it.row.quot(i), c8 = i - r * it.row.d;
  const int c = (int)c8 * 8;
  const size_t at = (size_t)r * W * it.row.d + c8;
  float g[8], u[8], t[8], a[8];
  decode8<FMT>(q[at], e[at >> 2], g);
  if (W == 2) decode8<FMT>(q[at + it.row.d], e[(at + it.row.d) >> 2], u);
  load8(dy + (size_t)r * f, c, f, vec, t);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    if (W == 2) {
      const float s = sigm<T>(g[k]), gs = g[k] * s, uu = u[k];
      a[k] = gs * uu;
      u[k] = t[k] * gs;                                    // du
      g[k] = t[k] * uu * s * (1.f + g[k] * (1.f - s));     // dg
    } else {
      const float x = g[k], s = sigm<T>(2.f * kGeluK * (x + kGeluC * x * x * x));
      a[k] = x * s;
      g[k] = t[k] * (s + 2.f * x * s * (1.f - s) * kGeluK * (1.f + 3.f * kGeluC * x * x));
    }
  }
  T* dr = dx + (size_t)r * W * f;
  store8(dr, c, f, vec, g);
  if (W == 2) store8(dr + f, c, f, vec, u);
  if (y) store8(y + (size_t)r * f, c, f, vec, a);
}

bool act_shape(int dtype, int fmt, int N, long long d) {
  return (dtype == ZL_DTYPE_F32 || dtype == ZL_DTYPE_BF16) && (fmt == ZL_ACT8_E4M3 || fmt == ZL_ACT8_INT8) && N >= 0 &&
         N <= ZL_ACT8_MAX_ROWS && d >= 1 && d <= ZL_ACT8_MAX_COLS && (long long)N * pitch((int)d) / 8 < (1ll << 31);
}
bool dw_shape(int dtype, int fmt, int M, int N, int K) { return act_shape(dtype, fmt, K, N) && act_shape(dtype, fmt, K, M); }
const char* const kShapeMsg =
    "bad dtype, code format, activation or size (0 <= rows <= 2^24, 1 <= columns <= 2^20, rows x columns in whole groups below 2^34, "
    "row strides >= columns, accumulate 0 or 1)";
bool codes_ok(const void* q, const void* e) { return q && e && ((uintptr_t)q & 15u) == 0; }
const char* const kPtrMsg = "NULL pointer, or codes that are not 16-byte aligned";

Items items(int N, int d) { return Items{(uint32_t)((size_t)N * (pitch(d) / 8)), FastDiv((uint32_t)(pitch(d) / 8))}; }
unsigned blocks_of(const Items& it) { return (it.n + kThreads - 1) / kThreads; }

template <typename T, int FMT>
void store_t(const void* x, size_t ldx, int N, int d, bool vec, uint8_t* q, uint8_t* e, cudaStream_t s) {
  const Items it = items(N, d);
  launch_pdl(store_k<T, FMT>, blocks_of(it), kThreads, 0, s, (const T*)x, ldx, d, vec, it, (uint2*)q, e);
}
template <typename T, int FMT>
void load_t(const uint8_t* q, const uint8_t* e, int N, int d, void* x, size_t ldx, bool vec, cudaStream_t s) {
  const Items it = items(N, d);
  launch_pdl(load_k<T, FMT>, blocks_of(it), kThreads, 0, s, (const uint2*)q, e, it, (T*)x, ldx, d, vec);
}
template <typename T, int FMT, int ACT>
void act_t(const void* x, int N, int f, bool vec, void* y, uint8_t* q, uint8_t* e, cudaStream_t s) {
  const Items it = items(N, f);
  launch_pdl(act_k<T, FMT, ACT>, blocks_of(it), kThreads, 0, s, (const T*)x, f, vec, it, (T*)y, (uint2*)q, e);
}
template <typename T, int FMT, int ACT>
void act_bwd_t(const uint8_t* q, const uint8_t* e, const void* dy, int N, int f, bool vec, void* dx, void* y, cudaStream_t s) {
  const Items it = items(N, f);
  launch_pdl(act_bwd_k<T, FMT, ACT>, blocks_of(it), kThreads, 0, s, (const uint2*)q, e, (const T*)dy, f, vec, it, (T*)dx, (T*)y);
}

// fn<T, FMT>(args) for the run-time dtype and format.
#define ZL_BY_TYPE(fn, dt, fmt, ...)                                                   \
  do {                                                                                 \
    if (dt == ZL_DTYPE_BF16) {                                                         \
      if (fmt == ZL_ACT8_E4M3) fn<bf16, ZL_ACT8_E4M3>(__VA_ARGS__);                    \
      else fn<bf16, ZL_ACT8_INT8>(__VA_ARGS__);                                        \
    } else {                                                                           \
      if (fmt == ZL_ACT8_E4M3) fn<float, ZL_ACT8_E4M3>(__VA_ARGS__);                   \
      else fn<float, ZL_ACT8_INT8>(__VA_ARGS__);                                       \
    }                                                                                  \
  } while (0)

template <typename T, int FMT>
void act_by(int act, const void* x, int N, int f, bool vec, void* y, uint8_t* q, uint8_t* e, cudaStream_t s) {
  if (act == ZL_ACT_SWIGLU) act_t<T, FMT, ZL_ACT_SWIGLU>(x, N, f, vec, y, q, e, s);
  else act_t<T, FMT, ZL_ACT_GELU>(x, N, f, vec, y, q, e, s);
}
template <typename T, int FMT>
void act_bwd_by(int act, const uint8_t* q, const uint8_t* e, const void* dy, int N, int f, bool vec, void* dx, void* y, cudaStream_t s) {
  if (act == ZL_ACT_SWIGLU) act_bwd_t<T, FMT, ZL_ACT_SWIGLU>(q, e, dy, N, f, vec, dx, y, s);
  else act_bwd_t<T, FMT, ZL_ACT_GELU>(q, e, dy, N, f, vec, dx, y, s);
}

size_t up256(size_t b) { return (b + 255) / 256 * 256; }

}  // namespace
}  // namespace zl

using namespace zl;
using zl::act8::entry;
using zl::act8::rows_aligned;

extern "C" {

zl_status zl_op_act8_store(int dtype, int fmt, const void* x, int N, int d, int ldx, uint8_t* q, uint8_t* e, void* stream) {
  return entry([&]() -> zl_status {
    if (!act_shape(dtype, fmt, N, d) || ldx < d) return fail(ZL_ERR_ARG, kShapeMsg);
    if (N == 0) return ZL_OK;
    if (!x || !codes_ok(q, e)) return fail(ZL_ERR_ARG, kPtrMsg);
    note_launch(1);
    ZL_BY_TYPE(store_t, dtype, fmt, x, (size_t)ldx, N, d, rows_aligned(x, (size_t)ldx, dtype), q, e, (cudaStream_t)stream);
    return launched("zl_op_act8_store");
  });
}

zl_status zl_op_act8_load(int dtype, int fmt, const uint8_t* q, const uint8_t* e, int N, int d, int ldx, void* x, void* stream) {
  return entry([&]() -> zl_status {
    if (!act_shape(dtype, fmt, N, d) || ldx < d) return fail(ZL_ERR_ARG, kShapeMsg);
    if (N == 0) return ZL_OK;
    if (!x || !codes_ok(q, e)) return fail(ZL_ERR_ARG, kPtrMsg);
    note_launch(1);
    ZL_BY_TYPE(load_t, dtype, fmt, q, e, N, d, x, (size_t)ldx, rows_aligned(x, (size_t)ldx, dtype), (cudaStream_t)stream);
    return launched("zl_op_act8_load");
  });
}

zl_status zl_op_act8_act(int dtype, int act, int fmt, const void* x, int N, int f, void* y, uint8_t* q, uint8_t* e, void* stream) {
  return entry([&]() -> zl_status {
    if ((act != ZL_ACT_SWIGLU && act != ZL_ACT_GELU) || !act_shape(dtype, fmt, N, f)) return fail(ZL_ERR_ARG, kShapeMsg);
    if (N == 0) return ZL_OK;
    if (!x || !y || !codes_ok(q, e)) return fail(ZL_ERR_ARG, kPtrMsg);
    const bool vec = rows_aligned(x, (size_t)f, dtype) && rows_aligned(y, (size_t)f, dtype);
    note_launch(1);
    ZL_BY_TYPE(act_by, dtype, fmt, act, x, N, f, vec, y, q, e, (cudaStream_t)stream);
    return launched("zl_op_act8_act");
  });
}

zl_status zl_op_act8_act_bwd(int dtype, int act, int fmt, const uint8_t* q, const uint8_t* e, const void* dy, int N, int f,
                             void* dx, void* y, void* stream) {
  return entry([&]() -> zl_status {
    if ((act != ZL_ACT_SWIGLU && act != ZL_ACT_GELU) || !act_shape(dtype, fmt, N, f)) return fail(ZL_ERR_ARG, kShapeMsg);
    if (N == 0) return ZL_OK;
    if (!dy || !dx || !codes_ok(q, e)) return fail(ZL_ERR_ARG, kPtrMsg);
    const bool vec = rows_aligned(dy, (size_t)f, dtype) && rows_aligned(dx, (size_t)f, dtype) &&
                     (!y || rows_aligned(y, (size_t)f, dtype));
    note_launch(1);
    ZL_BY_TYPE(act_bwd_by, dtype, fmt, act, q, e, dy, N, f, vec, dx, y, (cudaStream_t)stream);
    return launched("zl_op_act8_act_bwd");
  });
}

zl_status zl_op_act8_dw_bytes(int dtype, int M, int N, int K, size_t* bytes) {
  return entry([&]() -> zl_status {
    if (!bytes || !dw_shape(dtype, ZL_ACT8_E4M3, M, N, K)) return fail(ZL_ERR_ARG, kShapeMsg);
    *bytes = up256((size_t)K * N * dt_size(dtype));
    return ZL_OK;
  });
}

zl_status zl_op_act8_dw(int dtype, int fmt, int M, int N, int K, const void* A, const uint8_t* q, const uint8_t* e, float* C,
                        int accumulate, void* ws, size_t ws_bytes, void* stream) {
  return entry([&]() -> zl_status {
    if (!dw_shape(dtype, fmt, M, N, K) || (accumulate != 0 && accumulate != 1)) return fail(ZL_ERR_ARG, kShapeMsg);
    if (!C || (K > 0 && (!A || !codes_ok(q, e)))) return fail(ZL_ERR_ARG, kPtrMsg);
    size_t need = 0;
    zl_op_act8_dw_bytes(dtype, M, N, K, &need);
    if (need && (!ws || ((uintptr_t)ws & 255u) || ws_bytes < need))
      return fail(ZL_ERR_ARG, "the workspace must be 256-byte aligned and hold zl_op_act8_dw_bytes() bytes");
    cudaStream_t s = (cudaStream_t)stream;
    if (!accumulate && cudaMemsetAsync(C, 0, (size_t)M * N * 4, s) != cudaSuccess) return launched("zl_op_act8_dw");
    if (K == 0) return ZL_OK;
    note_launch(1);
    ZL_BY_TYPE(load_t, dtype, fmt, q, e, K, N, ws, (size_t)N, rows_aligned(ws, (size_t)N, dtype), s);
    gemm(dtype, 2, M, N, K, A, ws, C, nullptr, nullptr, s);
    return launched("zl_op_act8_dw");
  });
}

}  // extern "C"
