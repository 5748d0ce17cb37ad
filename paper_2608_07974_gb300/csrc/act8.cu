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
// a warp runs the code, `in` says whether its item exists. Rows that do not start on 16 bytes (MODE kSingle) are read and
// written in whole 16-byte words all the same, shifted between neighbouring lanes: 2048 x 22001 bf16 to integer codes 25 us, back
// 34 (value by value 29 and 111, written through shared memory 43); SwiGLU of 2048 x 11001 46 and 55 us.
struct Items {
  uint32_t n;      // N * D / 8, below 2^31
  FastDiv row;     // D / 8 pieces to a row
};
struct Item {
  uint32_t r, c8, at;   // row, piece of it, r * (D / 8) + c8
  bool in;
  __device__ __forceinline__ int c() const { return (int)c8 * 8; }
};
// Items of a thread: their loads are under way together (2048 x 22016 bf16 to e4m3 24.7 / 21.2 / 22.5 us with one, two, four,
// back 24.6 / 21.1 / 21.7; SwiGLU forward of 2048 x 11008 32.2 / 29.5 with one, two; the backward, with more streams an item
// and more registers, gains nothing). Of rows off 16 bytes (kSingle) the activations take one forward, whose inputs then fill
// the registers (2048 x 4097 fp32 27.6 us with two, 23.6 with one), and two backward (32.3 with one, 29.3 with two).
constexpr int kStoreItems = 2, kLoadItems = 2;
constexpr int act_items(int mode) { return mode == kSingle ? 1 : 2; }
constexpr int act_bwd_items(int mode) { return mode == kSingle ? 2 : 1; }
// Blocks of the SwiGLU backward on an SM (0: as many as its registers leave): one register above 40 costs the sixth (2048 x
// 11008 bf16 from integer codes 38.2 us with six, 39.4 with five; 4096 x 8192 fp32 90.3, with 12 bytes spilled, and 99.9). fp32
// rows with a ragged end stay at five.
constexpr int act_bwd_blocks(int act, int mode, size_t bytes) {
  return act != ZL_ACT_SWIGLU || mode == kSingle ? 0 : mode == kTail && bytes == 4 ? 5 : 6;
}
// Item u of U.
template <int U>
__device__ __forceinline__ Item item(const Items& it, int u) {
  Item x;
  x.at = (blockIdx.x * U + u) * kThreads + threadIdx.x;
  x.in = x.at < it.n;
  x.r = x.in ? it.row.quot(x.at) : 0;
  x.c8 = x.in ? x.at - x.r * it.row.d : 0;
  return x;
}
template <int MODE, typename T>
__device__ __forceinline__ void item_out(T* p, const Item& x, int d, const float* f) {
  if (MODE == kSingle) {
    uint64_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = f2(f[2 * i], f[2 * i + 1]);
    Raw8<T> r;
    pack8(v, r);
    store_any(p, x.c(), x.in ? d : 0, r);
  } else if (x.in) {
    store8<MODE>(p, x.c(), d, f);
  }
}

// ------------------------------------------------------------------------------------------------
// Rows to 8 bits and back: code = x 2^-E rounded, value = code 2^E. HBM-bound: 3.03 bytes a value in bf16, 5.03 in fp32.
// 2048 x 22016 bf16 21.0 us written and 20.9 us read (6.5 TB/s, 96% of the measured copy rate), integer codes alike;
// 2048 x 4096 4.8 us, of which about 2 are the launch.
// ------------------------------------------------------------------------------------------------
template <typename T, int FMT, int MODE>
__global__ void __launch_bounds__(kThreads) store_k(const T* __restrict__ x, size_t ldx, int d, Items it, uint2* __restrict__ q,
                                                    uint8_t* __restrict__ e) {
  constexpr int U = kStoreItems;
  pdl_wait();
  pdl_trigger();
  Item i[U];
  Piece<MODE, T> r[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    i[u] = item<U>(it, u);
    r[u].load(x + i[u].r * ldx, i[u].c(), i[u].in ? d : 0);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float f[8];
    r[u].floats(f);
    uint2 w;
    const uint32_t b = encode_quarter<FMT>(f, w);
    if (i[u].in) {
      q[i[u].at] = w;
      if ((i[u].at & 3u) == 0) e[i[u].at >> 2] = (uint8_t)b;
    }
  }
}

template <typename T, int FMT, int MODE>
__global__ void __launch_bounds__(kThreads) load_k(const uint2* __restrict__ q, const uint8_t* __restrict__ e, Items it,
                                                   T* __restrict__ x, size_t ldx, int d) {
  constexpr int U = kLoadItems;
  pdl_wait();
  pdl_trigger();
  Item i[U];
  uint2 w[U];
  uint32_t b[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    i[u] = item<U>(it, u);
    const uint32_t at = i[u].in ? i[u].at : 0;
    w[u] = q[at];
    b[u] = e[at >> 2];
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    float f[8];
    decode8<FMT>(w[u], b[u], f);
    item_out<MODE>(x + i[u].r * ldx, i[u], d, f);
  }
}

// ------------------------------------------------------------------------------------------------
// Activations. SwiGLU: y = g s u, s = 1 / (1 + e^-g); dg = dy u s (1 + g (1 - s)), du = dy g s. GELU (tanh form):
// y = x s(2a), a = k (x + c x^3), k = sqrt(2 / pi), c = 0.044715 (0.5 (1 + tanh a) = s(2a));
// dx = dy (s + 2 x s (1 - s) k (1 + 3 c x^2)). bf16: e^x and the reciprocal by the fast instructions (a few fp32 ulp,
// far below the rounding to bf16); fp32: expf and a true division. HBM-bound: a SwiGLU in bf16 moves 8.06 bytes for each of
// its f values forward, 10.06 backward (y again among them). 2048 x 11008 bf16 from e4m3: forward 29.5 us (6.2 TB/s, 91% of
// the measured copy rate), backward 34.7 us (6.5 TB/s); from integer codes 29.1 and 38.2; GELU 22.6 and 28.4.
// ------------------------------------------------------------------------------------------------
template <typename T>
__device__ __forceinline__ float sigm(float x) {
  if (sizeof(T) == 2) return rcp_approx(1.f + __expf(-x));
  return 1.f / (1.f + expf(-x));
}
constexpr float kGeluK = 0.7978845608028654f, kGeluC = 0.044715f;

// x [N, f] (GELU) or [N, 2 f] (SwiGLU: gate, up); codes of the rows of f values: [N, D] or [N, 2 D], D = pitch(f).
template <typename T, int FMT, int ACT, int MODE>
__global__ void __launch_bounds__(kThreads) act_k(const T* __restrict__ x, int f, Items it, T* __restrict__ y,
                                                  uint2* __restrict__ q, uint8_t* __restrict__ e) {
  constexpr int W = ACT == ZL_ACT_SWIGLU ? 2 : 1, U = act_items(MODE);
  pdl_wait();
  pdl_trigger();
  Item i[U];
  Piece<MODE, T> rg[U], ru[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    i[u] = item<U>(it, u);
    const T* xr = x + (size_t)i[u].r * W * f;
    rg[u].load(xr, i[u].c(), i[u].in ? f : 0);
    if (W == 2) ru[u].load(xr + f, i[u].c(), i[u].in ? f : 0);
  }
#pragma unroll
  for (int n = 0; n < U; ++n) {
    float g[8], u[8];
    rg[n].floats(g);
    if (W == 2) ru[n].floats(u);
    uint2 w;
    uint32_t b = encode_quarter<FMT>(g, w);
    size_t at = (size_t)i[n].r * W * it.row.d + i[n].c8;
    if (i[n].in) {
      q[at] = w;
      if ((i[n].c8 & 3u) == 0) e[at >> 2] = (uint8_t)b;
    }
    if (W == 2) {
      b = encode_quarter<FMT>(u, w);
      at += it.row.d;
      if (i[n].in) {
        q[at] = w;
        if ((i[n].c8 & 3u) == 0) e[at >> 2] = (uint8_t)b;
      }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (W == 2) g[k] = g[k] * sigm<T>(g[k]) * u[k];
      else g[k] = g[k] * sigm<T>(2.f * kGeluK * (g[k] + kGeluC * g[k] * g[k] * g[k]));
    }
    item_out<MODE>(y + (size_t)i[n].r * f, i[n], f, g);
  }
}

template <typename T, int FMT, int ACT, int MODE>
__global__ void __launch_bounds__(kThreads, act_bwd_blocks(ACT, MODE, sizeof(T))) act_bwd_k(const uint2* __restrict__ q, const uint8_t* __restrict__ e,
                                                      const T* __restrict__ dy, int f, Items it,
                                                      T* __restrict__ dx, T* __restrict__ y) {
  constexpr int W = ACT == ZL_ACT_SWIGLU ? 2 : 1, U = act_bwd_items(MODE);
  pdl_wait();
  pdl_trigger();
  Item i[U];
  Piece<MODE, T> rt[U];
  uint2 qg[U], qu[U];
  uint32_t eg[U], eu[U];
#pragma unroll
  for (int n = 0; n < U; ++n) {
    i[n] = item<U>(it, n);
    const size_t at = i[n].in ? (size_t)i[n].r * W * it.row.d + i[n].c8 : 0, at2 = i[n].in && W == 2 ? at + it.row.d : at;
    rt[n].load(dy + (size_t)i[n].r * f, i[n].c(), i[n].in ? f : 0);
    qg[n] = q[at];
    eg[n] = e[at >> 2];
    if (W == 2) {
      qu[n] = q[at2];
      eu[n] = e[at2 >> 2];
    }
  }
#pragma unroll
  for (int n = 0; n < U; ++n) {
    float g[8], u[8], t[8], a[8];
    rt[n].floats(t);
    decode8<FMT>(qg[n], eg[n], g);
    if (W == 2) decode8<FMT>(qu[n], eu[n], u);
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      if (W == 2) {
        const float s = sigm<T>(g[k]), gs = g[k] * s, uu = u[k];
        a[k] = gs * uu;
        u[k] = t[k] * gs;                                    // du
        // dg: half of silu' (which stays below 1.1) times up first, so that no factor is infinite (dy up may be, and s then 0)
        g[k] = 2.f * (t[k] * (s * fmaf(g[k], fmaf(-0.5f, s, 0.5f), 0.5f) * uu));
      } else {
        const float x = g[k], s = sigm<T>(2.f * kGeluK * (x + kGeluC * x * x * x));
        a[k] = x * s;
        // (s (1 - s) is 0 long before 2 x or x^2 overflows: with finite factors their product is 0, not NaN)
        g[k] = t[k] * (s + 2.f * kGeluK * (s * (1.f - s) * x) * (1.f + 3.f * kGeluC * fminf(x * x, 1e30f)));
      }
    }
    T* dr = dx + (size_t)i[n].r * W * f;
    item_out<MODE>(dr, i[n], f, g);
    if (W == 2) item_out<MODE>(dr + f, i[n], f, u);
    if (y) item_out<MODE>(y + (size_t)i[n].r * f, i[n], f, a);
  }
}

// ------------------------------------------------------------------------------------------------
// Weight gradient C = A^T X, X from its checkpoint, on the tensor cores in bf16. X is exactly a bf16 matrix, so it is read
// from its codes once into a workspace (2 bytes a value, which stay in L2 for the product) and the tcgen05 GEMM does the
// rest. An fp32 A is cut into three bf16 terms a = hi + mid + lo, each the leading 8 bits of what is left (truncated, so
// that nothing overflows and 24 bits are covered exactly, down to 2^-133); X being exact, the three products in one fp32
// accumulation are the fp32 product, at a third of the bf16 rate instead of the fp32 units' (about 1/27 of it). The small
// terms go first.
// Tensor-core bound: 22016 x 4096 over 2048 tokens 209 us (1.77 PFLOP/s, 92% of the measured cuBLAS burst; the workspace
// about 5 us of it), 4096 x 4096 over 8192 tokens 190 us (the GEMM on a bf16 X 161; the workspace 16, the segments of its
// sums the rest); fp32 2048 x 2048 over 1021 tokens 26 us (the CUDA-core GEMM 213), 8192 x 8192 over 2048 478 us;
// rows of C off 16 bytes, 4099 x 4099 over 2048 tokens, bf16 80 us.
// ------------------------------------------------------------------------------------------------
struct DwPlan {
  int Mp, Np, Kp, parts;
  bool copy_a;               // A through the workspace: cut into terms, or its rows onto 16 bytes
  size_t b, a, splits;       // bytes of the workspace's pieces
};
DwPlan dw_plan(int dtype, int M, int N, int K) {
  DwPlan p;
  p.Mp = (M + 7) / 8 * 8;
  p.Np = (N + 7) / 8 * 8;
  p.Kp = (K + 63) / 64 * 64;
  p.parts = dtype == ZL_DTYPE_F32 ? 3 : 1;
  p.copy_a = p.parts > 1 || p.Mp != M;
  p.b = up256((size_t)K * p.Np * 2);
  p.a = p.copy_a ? up256((size_t)p.parts * p.Kp * p.Mp * 2) : 0;
  p.splits = up256(gemm_tc_dw_bytes(M, N, K, p.parts));
  return p;
}

struct DwPrep {
  const uint2* q;
  const uint8_t* e;
  bf16* B;                   // [K, Np]
  FastDiv brow;              // Np / 8
  int gpitch;                // 8-column pieces of codes to a row
  uint32_t nb, blocks_b;
  const void* A;
  bf16* Aw;                  // [parts, Kp, Mp], or NULL
  FastDiv arow;              // Mp / 8
  int M, K;
  bool vec;
  uint32_t na;               // pieces of one part
};
// X from its codes, and A padded or cut into terms; HBM- and L2-bound: 3 bytes a value of X in bf16, 10 of an fp32 A.
template <typename T, int FMT>
__global__ void __launch_bounds__(kThreads) dw_prep_k(const DwPrep p) {
  pdl_wait();
  pdl_trigger();
  float f[8];
  if (blockIdx.x < p.blocks_b) {
    constexpr int U = kLoadItems;
    uint2 w[U];
    uint32_t b[U];
    const uint32_t i0 = blockIdx.x * U * kThreads + threadIdx.x;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const uint32_t i = min(i0 + u * kThreads, p.nb - 1), r = p.brow.quot(i);
      const size_t at = (size_t)r * p.gpitch + (i - r * p.brow.d);
      w[u] = p.q[at];
      b[u] = p.e[at >> 2];
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (i0 + u * kThreads >= p.nb) return;
      decode8<FMT>(w[u], b[u], f);
      Vec8<bf16>::store(p.B + (size_t)(i0 + u * kThreads) * 8, f);
    }
    return;
  }
  const uint32_t i = (blockIdx.x - p.blocks_b) * kThreads + threadIdx.x;
  if (i >= p.na) return;
  const uint32_t r = p.arow.quot(i);
  const int c = (int)(i - r * p.arow.d) * 8;
  if ((int)r < p.K) {
    if (p.vec) load8<kTail>((const T*)p.A + (size_t)r * p.M, c, p.M, f);
    else load8<kSingle>((const T*)p.A + (size_t)r * p.M, c, p.M, f);
  }
  else {
#pragma unroll
    for (int k = 0; k < 8; ++k) f[k] = 0.f;
  }
  if (sizeof(T) == 2) {
    Vec8<bf16>::store(p.Aw + (size_t)i * 8, f);
    return;
  }
  const size_t part = (size_t)p.na * 8;
#pragma unroll
  for (int t = 2; t >= 0; --t) {
    float h[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const uint32_t u = __float_as_uint(f[k]);
      const bool fin = (u & kInfBits) != kInfBits;
      h[k] = fin ? __uint_as_float(u & 0xFFFF0000u) : f[k];   // a NaN or an infinity goes whole into the first term
      f[k] = fin ? f[k] - h[k] : 0.f;
    }
    Vec8<bf16>::store(p.Aw + t * part + (size_t)i * 8, h);
  }
}

bool act_shape(int dtype, int fmt, int N, long long d) {
  return (dtype == ZL_DTYPE_F32 || dtype == ZL_DTYPE_BF16) && (fmt == ZL_ACT8_E4M3 || fmt == ZL_ACT8_INT8) && N >= 0 &&
         N <= ZL_ACT8_MAX_ROWS && d >= 1 && d <= ZL_ACT8_MAX_COLS && (long long)N * pitch((int)d) / 8 < (1ll << 31);
}
bool dw_shape(int dtype, int fmt, int M, int N, int K) {
  return act_shape(dtype, fmt, K, N) && act_shape(dtype, fmt, K, M) && act_shape(dtype, fmt, M, N);
}
const char* const kShapeMsg =
    "bad dtype, code format, activation or size (0 <= rows <= 2^24, 1 <= columns <= 2^20, rows x columns in whole groups "
    "below 2^34, row strides >= columns, accumulate 0 or 1)";
bool codes_ok(const void* q, const void* e) { return q && e && ((uintptr_t)q & 15u) == 0; }
const char* const kPtrMsg = "NULL pointer, a tensor off the alignment of its elements, or codes (or A) that are not 16-byte aligned";

// Items of N rows and the blocks that take them.
struct Shape {
  Items it;
  unsigned blocks;
  Shape(int N, int d, unsigned items) {
    const uint32_t pieces = (uint32_t)(pitch(d) / 8), per = kThreads * items;
    it.n = (uint32_t)((size_t)N * pieces);
    it.row = FastDiv(pieces);
    blocks = (it.n + per - 1) / per;
  }
};

// The kernel of a mode.
#define ZL_BY_MODE(kern, ...) \
  (mode == kWhole ? kern<__VA_ARGS__, kWhole> : mode == kTail ? kern<__VA_ARGS__, kTail> : kern<__VA_ARGS__, kSingle>)

template <typename T, int FMT>
void store_t(const void* x, size_t ldx, int N, int d, int mode, uint8_t* q, uint8_t* e, cudaStream_t s) {
  const Shape h(N, d, kStoreItems);
  launch_pdl(ZL_BY_MODE(store_k, T, FMT), h.blocks, kThreads, 0, s, (const T*)x, ldx, d, h.it, (uint2*)q, e);
}
template <typename T, int FMT>
void load_t(const uint8_t* q, const uint8_t* e, int N, int d, void* x, size_t ldx, int mode, cudaStream_t s) {
  const Shape h(N, d, kLoadItems);
  launch_pdl(ZL_BY_MODE(load_k, T, FMT), h.blocks, kThreads, 0, s, (const uint2*)q, e, h.it, (T*)x, ldx, d);
}
template <typename T, int FMT, int ACT>
void act_t(const void* x, int N, int f, int mode, void* y, uint8_t* q, uint8_t* e, cudaStream_t s) {
  const Shape h(N, f, act_items(mode));
  launch_pdl(ZL_BY_MODE(act_k, T, FMT, ACT), h.blocks, kThreads, 0, s, (const T*)x, f, h.it, (T*)y, (uint2*)q, e);
}
template <typename T, int FMT, int ACT>
void act_bwd_t(const uint8_t* q, const uint8_t* e, const void* dy, int N, int f, int mode, void* dx, void* y, cudaStream_t s) {
  const Shape h(N, f, act_bwd_items(mode));
  launch_pdl(ZL_BY_MODE(act_bwd_k, T, FMT, ACT), h.blocks, kThreads, 0, s, (const uint2*)q, e, (const T*)dy, f, h.it, (T*)dx,
             (T*)y);
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
void act_by(int act, const void* x, int N, int f, int mode, void* y, uint8_t* q, uint8_t* e, cudaStream_t s) {
  if (act == ZL_ACT_SWIGLU) act_t<T, FMT, ZL_ACT_SWIGLU>(x, N, f, mode, y, q, e, s);
  else act_t<T, FMT, ZL_ACT_GELU>(x, N, f, mode, y, q, e, s);
}
template <typename T, int FMT>
void act_bwd_by(int act, const uint8_t* q, const uint8_t* e, const void* dy, int N, int f, int mode, void* dx, void* y,
                cudaStream_t s) {
  if (act == ZL_ACT_SWIGLU) act_bwd_t<T, FMT, ZL_ACT_SWIGLU>(q, e, dy, N, f, mode, dx, y, s);
  else act_bwd_t<T, FMT, ZL_ACT_GELU>(q, e, dy, N, f, mode, dx, y, s);
}

template <typename T, int FMT>
void prep_t(const DwPrep& p, unsigned blocks, cudaStream_t s) {
  launch_pdl(dw_prep_k<T, FMT>, blocks, kThreads, 0, s, p);
}

}  // namespace
}  // namespace zl

using namespace zl;
using zl::act8::entry;
using zl::act8::on_elements;
using zl::act8::row_mode;

extern "C" {

zl_status zl_op_act8_store(int dtype, int fmt, const void* x, int N, int d, int ldx, uint8_t* q, uint8_t* e, void* stream) {
  return entry([&]() -> zl_status {
    if (!act_shape(dtype, fmt, N, d) || ldx < d) return fail(ZL_ERR_ARG, kShapeMsg);
    if (N == 0) return ZL_OK;
    if (!x || !on_elements({x}, dt_size(dtype)) || !codes_ok(q, e)) return fail(ZL_ERR_ARG, kPtrMsg);
    note_launch(1);
    ZL_BY_TYPE(store_t, dtype, fmt, x, (size_t)ldx, N, d, row_mode(x, (size_t)d, (size_t)ldx, dtype), q, e, (cudaStream_t)stream);
    return launched("zl_op_act8_store");
  });
}

zl_status zl_op_act8_load(int dtype, int fmt, const uint8_t* q, const uint8_t* e, int N, int d, int ldx, void* x, void* stream) {
  return entry([&]() -> zl_status {
    if (!act_shape(dtype, fmt, N, d) || ldx < d) return fail(ZL_ERR_ARG, kShapeMsg);
    if (N == 0) return ZL_OK;
    if (!x || !on_elements({x}, dt_size(dtype)) || !codes_ok(q, e)) return fail(ZL_ERR_ARG, kPtrMsg);
    note_launch(1);
    ZL_BY_TYPE(load_t, dtype, fmt, q, e, N, d, x, (size_t)ldx, row_mode(x, (size_t)d, (size_t)ldx, dtype), (cudaStream_t)stream);
    return launched("zl_op_act8_load");
  });
}

zl_status zl_op_act8_act(int dtype, int act, int fmt, const void* x, int N, int f, void* y, uint8_t* q, uint8_t* e, void* stream) {
  return entry([&]() -> zl_status {
    if ((act != ZL_ACT_SWIGLU && act != ZL_ACT_GELU) || !act_shape(dtype, fmt, N, f)) return fail(ZL_ERR_ARG, kShapeMsg);
    if (N == 0) return ZL_OK;
    if (!x || !y || !on_elements({x, y}, dt_size(dtype)) || !codes_ok(q, e)) return fail(ZL_ERR_ARG, kPtrMsg);
    const int mode = std::min(row_mode(x, f, f, dtype), row_mode(y, f, f, dtype));
    note_launch(1);
    ZL_BY_TYPE(act_by, dtype, fmt, act, x, N, f, mode, y, q, e, (cudaStream_t)stream);
    return launched("zl_op_act8_act");
  });
}

zl_status zl_op_act8_act_bwd(int dtype, int act, int fmt, const uint8_t* q, const uint8_t* e, const void* dy, int N, int f,
                             void* dx, void* y, void* stream) {
  return entry([&]() -> zl_status {
    if ((act != ZL_ACT_SWIGLU && act != ZL_ACT_GELU) || !act_shape(dtype, fmt, N, f)) return fail(ZL_ERR_ARG, kShapeMsg);
    if (N == 0) return ZL_OK;
    if (!dy || !dx || !on_elements({dy, dx, y}, dt_size(dtype)) || !codes_ok(q, e)) return fail(ZL_ERR_ARG, kPtrMsg);
    const int mode = std::min({row_mode(dy, f, f, dtype), row_mode(dx, f, f, dtype), y ? row_mode(y, f, f, dtype) : kWhole});
    note_launch(1);
    ZL_BY_TYPE(act_bwd_by, dtype, fmt, act, q, e, dy, N, f, mode, dx, y, (cudaStream_t)stream);
    return launched("zl_op_act8_act_bwd");
  });
}

zl_status zl_op_act8_dw_bytes(int dtype, int M, int N, int K, size_t* bytes) {
  return entry([&]() -> zl_status {
    if (!bytes || !dw_shape(dtype, ZL_ACT8_E4M3, M, N, K)) return fail(ZL_ERR_ARG, kShapeMsg);
    const DwPlan p = dw_plan(dtype, M, N, K);
    *bytes = K ? p.b + p.a + p.splits : 0;
    return ZL_OK;
  });
}

zl_status zl_op_act8_dw(int dtype, int fmt, int M, int N, int K, const void* A, const uint8_t* q, const uint8_t* e, float* C,
                        int accumulate, void* ws, size_t ws_bytes, void* stream) {
  return entry([&]() -> zl_status {
    if (!dw_shape(dtype, fmt, M, N, K) || (accumulate != 0 && accumulate != 1)) return fail(ZL_ERR_ARG, kShapeMsg);
    cudaStream_t s = (cudaStream_t)stream;
    if (K == 0) {
      if (!C || !on_elements({C}, 4)) return fail(ZL_ERR_ARG, kPtrMsg);
      if (!accumulate) cudaMemsetAsync(C, 0, (size_t)M * N * 4, s);
      return launched("zl_op_act8_dw");
    }
    if (!A || !C || !codes_ok(q, e) || ((uintptr_t)A & 15u) || !on_elements({C}, 4)) return fail(ZL_ERR_ARG, kPtrMsg);
    const DwPlan p = dw_plan(dtype, M, N, K);
    if (!ws || ((uintptr_t)ws & 255u) || ws_bytes < p.b + p.a + p.splits)
      return fail(ZL_ERR_ARG, "the workspace must be 256-byte aligned and hold zl_op_act8_dw_bytes() bytes");
    uint8_t* w = (uint8_t*)ws;
    DwPrep r = {};
    r.q = (const uint2*)q; r.e = e; r.B = (bf16*)w; r.brow = FastDiv((uint32_t)p.Np / 8); r.gpitch = pitch(N) / 8;
    r.nb = (uint32_t)((size_t)K * (p.Np / 8));
    r.blocks_b = (r.nb + kLoadItems * kThreads - 1) / (kLoadItems * kThreads);
    r.A = A; r.Aw = (bf16*)(w + p.b); r.arow = FastDiv((uint32_t)p.Mp / 8); r.M = M; r.K = K;
    r.vec = row_mode(A, M, M, dtype) != kSingle;
    r.na = p.copy_a ? (uint32_t)((size_t)p.Kp * (p.Mp / 8)) : 0;
    note_launch(1);
    ZL_BY_TYPE(prep_t, dtype, fmt, r, r.blocks_b + (r.na + kThreads - 1) / kThreads, s);
    const GemmDw dw{p.parts, !accumulate, w + p.b + p.a, p.splits};
    if (!gemm_tc_dw(M, N, K, p.copy_a ? (const void*)r.Aw : A, p.copy_a ? p.Mp : M, r.B, p.Np, C, dw, s)) {
      const zl_status st = launched("zl_op_act8_dw");
      return st != ZL_OK ? st : fail(ZL_ERR_CUDA, "zl_op_act8_dw: the tensor-core product could not be launched on this device");
    }
    return launched("zl_op_act8_dw");
  });
}

}  // extern "C"
