// Cross entropy over a large vocabulary without its logits in memory (zl_op_vocab_loss) and its gradient (.._bwd).
//   z = n W^T,   lse_i = log sum_v e^{z_iv},   loss = sum_{Omega} (lse_i - z_iy) / |Omega|
//   dz = e^{z - lse} - [y],   dn = w dz W,   dW = w dz^T n,   w = dloss / |Omega|
// Forward: the product's epilogue reduces each row of a tile to (largest, sum e^{z - largest}) and picks the label's logit; a
// second launch joins the tiles' parts in their order and sums the losses. It moves N (d + tiles) and V d values and is bound by the
// products (2 N d V operations; few rows: by the one reading of W). 2048 x 4096 x 32000 bf16: 294 us in a captured graph, 97% of the burst
// peak; 332 as a call among others (power cap).
// Backward: the logits are formed again, a piece of the vocabulary at a time, and leave the product as dz (bf16; fp32 inputs:
// three bf16 terms); then dn += dz_p W_p in fp32 and dW_p = dz_p^T n. dz rounded to bf16 is off by 2^-9 of each value (but for the label's
// where p is small: -1 exactly), which the sums over columns and rows average; dn's own rounding is as large.
// The same size, both gradients: 889 us in a graph, 96% of the burst peak (a call 1021); 4096 x 768 x 50257, dn alone: 443 us, 75% (491).
#include <algorithm>

#include "act8.cuh"
#include "common.cuh"
#include "ops.h"
#include "vocab.cuh"
#include "vocab_gemm.cuh"

namespace zl {
namespace vocab {
namespace {

constexpr int kPrepThreads = 256;
// Bytes of dz that a piece of the vocabulary may take, where that leaves it kMinPiece columns. Larger pieces need fewer launches
// and lose less in their last wave of tiles; dz goes through HBM either way, under the products' time. Measured at one shape, 4096 x
// 768 x 50257, with pieces of 64 MB 550 us, 128 461, 192 428, 256 420, 512 (all of dz) 406 (logits in one accumulation): more is faster;
// 192 keeps the workspace below half of these logits, whose memory the call is there to save.
constexpr size_t kPieceBytes = 192u << 20;
constexpr int kMinPiece = 1024;
// k blocks (of 64) of one accumulation in TMEM: the tensor cores cut off what does not fit an fp32 sum, always towards zero, each
// time they add 16 products. With bf16 logits summed over 4096 in one accumulation lse was off by 1.7e-6 and the row losses by 2.6e-6,
// relative (an fp32 library product: 2.7e-7, 6.2e-7; in eight: 2e-7, 3e-7). fp32 logits: 2048 x 4096 x 32000 in accumulations of 256
// 1.4e-7 and 2.0e-7 in 1.95 ms, of 128 0.9e-7 and 1.5e-7 in 2.12. The backward's logits too: where the label's p is near 1, dz is the
// difference p - 1, and of a logit of 100 (products of one sign) one accumulation lost 1.2e-3, six times 1 - p = 2e-4; the gradient takes
// 4% longer for it. Sums that leave in bf16 are cut off far below its rounding.
constexpr int kSegLogits = 8, kSegF32 = 4, kSegDirect = 2, kSegAll = 1 << 20;
// Up to so many rows the products with an fp32 W read it as it is and cut it into its terms themselves, once for every 128 rows, and
// no terms of W (6 bytes a value) lie in the workspace. Beyond, the terms' way through memory costs less than cutting again. us, forward
// and both gradients, as it is / cut before:  768 x 50257, 256 rows 121 / 142, 346 / 407; 512: 203 / 196, 599 / 565; 1024: 367 / 317,
// 1137 / 1001; 2048: 691 / 540, 2221 / 1758.  4096 x 32000, 256: 383 / 490, 1039 / 1077; 512: 638 / 683, 1936 / 1694; 1024: 1231 / 1101,
// 3682 / 2861; 2048: 2278 / 1986, 7101 / 5753.  256 x 8000, 1024: 37 / 38, 103 / 96. The times cross at 300 to 1000 rows; up to 1024
// the workspace counts.
constexpr int kDirectRows = 1024;

inline int up64(int n) { return (n + 63) / 64 * 64; }

// An fp32 matrix [rows, d] as its bf16 terms [3][rows_p, d], rows past `rows` zeros.
struct Cut {
  const float* src;
  bf16* dst;
  int rows, rows_p;
};
// |Omega| by block 0 (where omega is not NULL), up to two matrices into their terms by the others, a warp a row.
__global__ void __launch_bounds__(kPrepThreads) vocab_prep_k(const Cut a, const Cut b, int d, const int32_t* __restrict__ labels, int N,
                                                             int V, float* omega) {
  pdl_wait();
  pdl_trigger();
  int block = blockIdx.x;
  if (omega) {
    if (block == 0) {
      __shared__ float sh[32];
      int n = 0;
      for (int i = threadIdx.x; i < N; i += kPrepThreads) {
        const int y = labels[i];
        n += y >= 0 && y < V;
      }
      // (each thread's count and the sum are at most 2^24: exact)
      const float count = block_sum((float)n, sh);
      if (threadIdx.x == 0) *omega = count;
      return;
    }
    --block;
  }
  const int lane = threadIdx.x & 31;
  int row = block * (kPrepThreads / 32) + (threadIdx.x >> 5);
  Cut m = a;
  if (row >= a.rows_p) {
    row -= a.rows_p;
    m = b;
  }
  if (row >= m.rows_p) return;
  const float* const x = m.src + (size_t)row * d;
  const bool in = row < m.rows;
  for (int i = lane; i < d / 8; i += 32) {
    float f[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (in) Vec8<float>::load(x + 8 * i, f);
    bf16* out = m.dst + (size_t)row * d + 8 * i;
#pragma unroll
    for (int t = 0; t < kTerms; ++t, out += (size_t)m.rows_p * d) {
      float h[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const uint32_t u = __float_as_uint(f[k]);
        const bool fin = (u & 0x7F800000u) != 0x7F800000u;
        h[k] = fin ? __uint_as_float(u & 0xFFFF0000u) : f[k];   // a NaN or an infinity goes whole into the first term
        f[k] = fin ? f[k] - h[k] : 0.f;
      }
      Vec8<bf16>::store(out, h);
    }
  }
}

// Joins each row's parts, `per` (32 .. 256) threads a row; the last block to end sums the losses.
__global__ void __launch_bounds__(256) vocab_finish_k(const float2* __restrict__ part, int parts, int per, const float* __restrict__ zl,
                                                      const int32_t* __restrict__ labels, int N, int V, float* row_loss, float* lse,
                                                      float* loss, unsigned* counter) {
  pdl_wait();
  pdl_trigger();
  __shared__ Lse sh[8];
  __shared__ bool last;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const size_t row = (size_t)blockIdx.x * (256 / per) + threadIdx.x / per;
  Lse A = lse_empty();
  if (row < (size_t)N) {
    const float2* p = part + row * parts;
    for (int i = threadIdx.x % per; i < parts; i += 4 * per) {
      float2 v[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) v[u] = i + u * per < parts ? p[i + u * per] : make_float2(-INFINITY, 0.f);
#pragma unroll
      for (int u = 0; u < 4; ++u) A = lse_merge(A, Lse{v[u].x, v[u].y}, kL2e);
    }
  }
  A = warp_merge(A, kL2e);
  if (lane == 0) sh[warp] = A;
  __syncthreads();
  if (row < (size_t)N && threadIdx.x % per == 0) {
    for (int w = 1; w < per / 32; ++w) A = lse_merge(A, sh[warp + w], kL2e);
    const float l = lse_value(A, 1.f);
    const int y = labels[row];
    lse[row] = l;
    row_loss[row] = y >= 0 && y < V ? l - zl[row] : 0.f;
  }
  __threadfence();
  __syncthreads();
  if (threadIdx.x == 0) last = atomicAdd(counter, 1u) == gridDim.x - 1;
  __syncthreads();
  if (last) {
    __threadfence();
    finish_loss(row_loss, labels, N, V, loss, 3);
  }
}

// dn = the sum of `slices` fp32 matrices of n values, in order, times the rows' weight, in T; eight values a thread, four slices'
// loads at a time.
template <typename T>
__global__ void __launch_bounds__(256) vocab_sum_k(const float* __restrict__ x, int slices, size_t n, T* __restrict__ dn,
                                                   const float* omega, const float* dloss) {
  pdl_wait();
  pdl_trigger();
  const size_t i = ((size_t)blockIdx.x * 256 + threadIdx.x) * 8;
  if (i >= n) return;
  float s[8];
  Vec8<float>::load(x + i, s);
  for (int k = 1; k < slices; k += 4) {
    float t[4][8];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (k + u < slices) Vec8<float>::load(x + (size_t)(k + u) * n + i, t[u]);
#pragma unroll
    for (int u = 0; u < 4; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (k + u < slices) s[e] += t[u][e];
  }
  const float w = loss_weight(omega, dloss);
#pragma unroll
  for (int e = 0; e < 8; ++e) s[e] *= w;
  Vec8<T>::store(dn + i, s);
}

size_t up256(size_t b) { return act8::up256(b); }

bool shape_ok(int dtype, int N, int d, int V) {
  return (dtype == ZL_DTYPE_F32 || dtype == ZL_DTYPE_BF16) && N >= 0 && N <= ZL_VOCAB_MAX_ROWS && d >= 8 && d <= ZL_VOCAB_MAX_WIDTH &&
         d % 8 == 0 && V >= 2 && V <= ZL_VOCAB_MAX;
}
const char* const kShapeMsg = "bad dtype or size (0 <= N <= 2^24, 8 <= d <= 2^16 and d % 8 == 0, 2 <= V <= 2^20)";
const char* const kPtrMsg = "NULL pointer, a tensor off the alignment of its elements, or n, W or a gradient that is not 16-byte aligned";
const char* const kWsMsg = "the workspace must be 256-byte aligned and hold what the call's _bytes() says";
bool al16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

// The forward call's tiling and the pieces of its workspace (offsets; `end` its size).
struct FwdPlan {
  Tiles t;
  int terms, parts, direct;
  size_t part, zl, counter, nt, wt, end;
};
FwdPlan fwd_plan(int dtype, int N, int d, int V) {
  FwdPlan p;
  p.terms = dtype == ZL_DTYPE_F32 ? kTerms : 1;
  p.direct = p.terms > 1 && N <= kDirectRows;
  p.t = p.direct ? plan_direct(N, V, d, kSegDirect, 1) : plan(kLse, N, V, d, p.terms, 16, p.terms > 1 ? kSegF32 : kSegLogits, 1);
  p.parts = lse_parts(V, p.t);
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += up256(bytes); return o; };
  p.counter = take(4);
  p.zl = take((size_t)N * 4);
  p.part = take((size_t)p.parts * N * 8);
  p.nt = take(p.terms > 1 ? (size_t)kTerms * N * d * 2 : 0);
  p.wt = take(p.terms > 1 && !p.direct ? (size_t)kTerms * V * d * 2 : 0);
  p.end = at;
  return p;
}

// The backward call's: pieces of `piece` columns.
struct BwdPlan {
  Tiles z, dn, dw;
  int terms, piece, rows_p, v_p, direct;
  size_t omega, dz, acc, nt, wt, end;
};
BwdPlan bwd_plan(int dtype, int N, int d, int V) {
  BwdPlan b;
  b.terms = dtype == ZL_DTYPE_F32 ? kTerms : 1;
  b.rows_p = up64(N);
  b.v_p = up64(V);
  b.direct = b.terms > 1 && N <= kDirectRows;
  const int seg = b.terms > 1 ? kSegF32 : kSegAll;
  const size_t row = (size_t)b.terms * b.rows_p * 2;
  const int most = std::max(kMinPiece, (int)std::min<size_t>(kPieceBytes / row, (size_t)b.v_p));
  const int least = (V + most - 1) / most;
  double best = 1e30;
  for (int k = least; k < least + 4; ++k) {   // as few pieces as may be, or a few more where their waves are fuller
    const int piece = up64((V + k - 1) / k), n = (V + piece - 1) / piece;
    if (k > least && piece < kMinPiece) break;
    const Tiles z = b.direct ? plan_direct(N, piece, d, kSegDirect, 1) : plan(kGradZ, N, piece, d, b.terms, 64, b.terms > 1 ? seg : kSegLogits, 1),
                dn = b.direct ? plan_direct(N, d, piece, kSegDirect, 32, n) : plan(kOut32, N, d, piece, b.terms, 32, seg, 32, n),
                dw = plan(b.terms > 1 ? kOut32 : kOut16, piece, d, N, b.terms, b.terms > 1 ? 32 : 64, seg, 1);
    const double us = n * (z.us + dn.us + dw.us);
    if (us < best) {
      best = us;
      b.z = z;
      b.dn = dn;
      b.dw = dw;
      b.piece = piece;
    }
  }
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t o = at; at += up256(bytes); return o; };
  b.omega = take(4);
  b.dz = take(row * b.piece);
  b.acc = take(b.terms > 1 && b.dn.splits == 1 ? 0 : (size_t)b.dn.splits * N * d * 4);
  b.nt = take(b.terms > 1 ? (size_t)kTerms * b.rows_p * d * 2 : 0);
  b.wt = take(b.terms > 1 && !b.direct ? (size_t)kTerms * b.v_p * d * 2 : 0);
  b.end = at;
  return b;
}

void launch_prep(const Cut& a, const Cut& b, int d, const int32_t* labels, int N, int V, float* omega, cudaStream_t s) {
  note_launch(1);
  constexpr int rows = kPrepThreads / 32;
  const size_t blocks = ((size_t)a.rows_p + b.rows_p + rows - 1) / rows + (omega ? 1 : 0);
  launch_pdl(vocab_prep_k, (unsigned)blocks, kPrepThreads, 0, s, a, b, d, labels, N, V, omega);
}

}  // namespace
}  // namespace vocab
}  // namespace zl

using namespace zl;
using namespace zl::vocab;
using zl::act8::entry;
using zl::act8::fail;
using zl::act8::launched;
using zl::act8::on_elements;

extern "C" {

zl_status zl_op_vocab_loss_bytes(int dtype, int N, int d, int V, size_t* bytes) {
  return entry([&]() -> zl_status {
    if (!bytes || !shape_ok(dtype, N, d, V)) return fail(ZL_ERR_ARG, kShapeMsg);
    *bytes = N ? fwd_plan(dtype, N, d, V).end : 0;
    return ZL_OK;
  });
}

zl_status zl_op_vocab_loss(int dtype, const void* n, const void* W, const int32_t* labels, int N, int d, int V, float* row_loss,
                           float* lse, float* loss, void* ws, size_t ws_bytes, void* stream) {
  return entry([&]() -> zl_status {
    if (!shape_ok(dtype, N, d, V)) return fail(ZL_ERR_ARG, kShapeMsg);
    cudaStream_t s = (cudaStream_t)stream;
    if (!loss || !on_elements({loss}, 4)) return fail(ZL_ERR_ARG, kPtrMsg);
    if (N == 0) {
      cudaMemsetAsync(loss, 0, 8, s);
      return launched("zl_op_vocab_loss");
    }
    if (!n || !W || !labels || !row_loss || !lse || !al16(n) || !al16(W) || !on_elements({labels, row_loss, lse}, 4))
      return fail(ZL_ERR_ARG, kPtrMsg);
    const FwdPlan p = fwd_plan(dtype, N, d, V);
    if (!ws || ((uintptr_t)ws & 255u) || ws_bytes < p.end) return fail(ZL_ERR_ARG, kWsMsg);
    uint8_t* const w = (uint8_t*)ws;
    const void *A = n, *B = W;
    if (p.terms > 1) {
      const Cut cn{(const float*)n, (bf16*)(w + p.nt), N, N};
      Cut cw{};
      if (!p.direct) cw = Cut{(const float*)W, (bf16*)(w + p.wt), V, V};
      launch_prep(cn, cw, d, labels, N, V, nullptr, s);
      A = w + p.nt;
      if (!p.direct) B = w + p.wt;
    }
    const Operands o{A, B, 0, 0, p.terms * N, (p.direct ? 1 : p.terms) * V, d, d, N, V, p.terms, 0, p.direct};
    bool ok = gemm_lse(N, V, d, o, p.t, labels, (float2*)(w + p.part), (float*)(w + p.zl), (unsigned*)(w + p.counter), s);
    if (ok) {
      note_launch(1);
      int per = 32;   // threads a row: four parts each, or more
      while (per < 256 && per * 4 < p.parts) per *= 2;
      const int rows = 256 / per;
      ok = launch_pdl(vocab_finish_k, (N + rows - 1) / rows, 256, 0, s, (const float2*)(w + p.part), p.parts, per,
                      (const float*)(w + p.zl), labels, N, V, row_loss, lse, loss, (unsigned*)(w + p.counter)) == cudaSuccess;
    }
    const zl_status st = launched("zl_op_vocab_loss");
    return st != ZL_OK || ok ? st : fail(ZL_ERR_CUDA, "zl_op_vocab_loss: the kernel could not be launched on this device");
  });
}

zl_status zl_op_vocab_loss_bwd_bytes(int dtype, int N, int d, int V, size_t* bytes) {
  return entry([&]() -> zl_status {
    if (!bytes || !shape_ok(dtype, N, d, V)) return fail(ZL_ERR_ARG, kShapeMsg);
    *bytes = N ? bwd_plan(dtype, N, d, V).end : 0;
    return ZL_OK;
  });
}

zl_status zl_op_vocab_loss_bwd(int dtype, const void* n, const void* W, const int32_t* labels, int N, int d, int V, const float* lse,
                               const float* dloss, void* dn, void* dW, void* ws, size_t ws_bytes, void* stream) {
  return entry([&]() -> zl_status {
    if (!shape_ok(dtype, N, d, V)) return fail(ZL_ERR_ARG, kShapeMsg);
    cudaStream_t s = (cudaStream_t)stream;
    const size_t es = dt_size(dtype);
    if ((N > 0 && !dn && !dW) || !al16(dn) || !al16(dW)) return fail(ZL_ERR_ARG, kPtrMsg);
    if (N == 0) {
      if (dW) cudaMemsetAsync(dW, 0, (size_t)V * d * es, s);
      return launched("zl_op_vocab_loss_bwd");
    }
    if (!n || !W || !labels || !lse || !al16(n) || !al16(W) || !on_elements({labels, lse, dloss}, 4)) return fail(ZL_ERR_ARG, kPtrMsg);
    const BwdPlan p = bwd_plan(dtype, N, d, V);
    if (!ws || ((uintptr_t)ws & 255u) || ws_bytes < p.end) return fail(ZL_ERR_ARG, kWsMsg);
    uint8_t* const w = (uint8_t*)ws;
    const bool f32 = p.terms > 1;
    float* const omega = (float*)(w + p.omega);
    const void *A = n, *B = W;
    int n_rows = N, w_rows = V, n_term = 0, w_term = 0;   // of the operands in memory
    Cut cn{}, cw{};
    if (f32) {
      cn = Cut{(const float*)n, (bf16*)(w + p.nt), N, p.rows_p};
      A = w + p.nt;
      n_rows = kTerms * p.rows_p;
      n_term = p.rows_p;
      if (!p.direct) {
        cw = Cut{(const float*)W, (bf16*)(w + p.wt), V, p.v_p};
        B = w + p.wt;
        w_rows = kTerms * p.v_p;
        w_term = p.v_p;
      }
    }
    launch_prep(cn, cw, d, labels, N, V, omega, s);
    void* const dz = w + p.dz;
    const int z_rows = p.terms * p.rows_p;
    const bool direct = f32 && p.dn.splits == 1;   // dn is where its sums are formed
    float* const acc = direct ? (float*)dn : (float*)(w + p.acc);
    bool ok = true;
    for (int first = 0; ok && first < V; first += p.piece) {
      const int m = std::min(p.piece, V - first), m64 = up64(m);
      ok = gemm_grad_z(N, m64, d, Operands{A, B, 0, 0, n_rows, w_rows, d, d, n_term, w_term, p.terms, first, p.direct}, p.z, labels, lse, first, V, dz, p.rows_p, p.piece, s);
      if (ok && dn)
        ok = gemm_out(N, d, m64, Operands{dz, B, 0, 1, z_rows, w_rows, p.piece, d, p.rows_p, w_term, p.terms, first, p.direct}, p.dn, 1,
                      acc, first > 0, direct ? omega : nullptr, dloss, s);
      if (ok && dW)
        ok = gemm_out(m, d, N, Operands{dz, A, 1, 1, z_rows, n_rows, p.piece, d, p.rows_p, n_term, p.terms, 0, 0}, p.dw, f32,
                      (uint8_t*)dW + (size_t)first * d * es, 0, omega, dloss, s);
    }
    if (ok && dn && !direct) {
      note_launch(1);
      const size_t len = (size_t)N * d;
      const unsigned blocks = (unsigned)((len / 8 + 255) / 256);
      ok = (f32 ? launch_pdl(vocab_sum_k<float>, blocks, 256, 0, s, (const float*)acc, p.dn.splits, len, (float*)dn, (const float*)omega,
                            dloss)
                : launch_pdl(vocab_sum_k<bf16>, blocks, 256, 0, s, (const float*)acc, p.dn.splits, len, (bf16*)dn, (const float*)omega,
                            dloss)) == cudaSuccess;
    }
    const zl_status st = launched("zl_op_vocab_loss_bwd");
    return st != ZL_OK || ok ? st : fail(ZL_ERR_CUDA, "zl_op_vocab_loss_bwd: a kernel could not be launched on this device");
  });
}

}  // extern "C"
