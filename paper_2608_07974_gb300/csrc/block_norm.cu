// The step between two blocks of a layer, fused (zl_op_block_norm): p = PostNorm(f), h' = alpha h + beta gate * p,
// n = PreNorm(h'), with f and n written in 8 bits (act8.cuh) in the same pass where the caller keeps them so, and its
// backward, which reads f from there.
#include <algorithm>

#include "act8.cuh"
#include "ops.h"

namespace zl {

namespace {
using namespace act8;

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
  bool vec, wvec;            // 16-byte rows of the tensors, of the parameters
};

__device__ __forceinline__ size_t gate_row(int n, int gate_rows) { return gate_rows ? (size_t)(n / gate_rows) : 0; }

__device__ __forceinline__ void put_codes(int fmt, const float* x, uint8_t* q, uint8_t* e, size_t at, bool in) {
  uint2 w;
  const uint32_t b = fmt == ZL_ACT8_E4M3 ? encode_quarter<ZL_ACT8_E4M3>(x, w) : encode_quarter<ZL_ACT8_INT8>(x, w);
  if (!in) return;
  reinterpret_cast<uint2*>(q)[at >> 3] = w;
  if ((at & 31) == 0) e[at >> 5] = (uint8_t)b;
}

// A row in registers: a warp per row (WARP: D <= 1024) or a block (D <= 16384), thread t holding the 8-column vectors
// t + j * (threads of the row). One read of h and f, one write of what is asked for; variances are of the centred
// values.
template <typename T, bool WARP, int VPT>
__global__ void __launch_bounds__(WARP ? 256 : 512) fwd_reg_k(const Fwd a) {
  pdl_wait();
  pdl_trigger();
  __shared__ float sh[32];
  const int row = WARP ? (int)((blockIdx.x * blockDim.x + threadIdx.x) >> 5) : (int)blockIdx.x;
  if (row >= a.N) return;
  const int t = WARP ? (threadIdx.x & 31) : threadIdx.x, nt = WARP ? 32 : blockDim.x;
  auto sum = [&](float v) { return WARP ? warp_sum(v) : block_sum(v, sh); };
  const size_t o = (size_t)row * a.d;
  const float inv_d = 1.f / a.d;
  float f[VPT][8], h[VPT][8];
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int c = (t + j * nt) * 8;
    load8((const T*)a.f + o, c, a.d, a.vec, f[j]);
    load8((const T*)a.h + o, c, a.d, a.vec, h[j]);
  }
  if (a.fq) {
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int c = (t + j * nt) * 8;
      put_codes(a.fmt, f[j], a.fq, a.fe, (size_t)row * a.D + c, c < a.D);
    }
  }
  float mean = 0.f, rstd = 1.f;
  auto stat = [&](float (&x)[VPT][8], int kind) {
    mean = 0.f;
    rstd = 1.f;
    if (kind == ZL_NORM_NONE) return;
    if (kind == ZL_NORM_LAYER) {
      float s = 0.f;
#pragma unroll
      for (int j = 0; j < VPT; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) s += x[j][i];
      mean = sum(s) * inv_d;
    }
    float q = 0.f;
#pragma unroll
    for (int j = 0; j < VPT; ++j) {
      const int c = (t + j * nt) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = c + i < a.d ? x[j][i] - mean : 0.f;
        q += v * v;
      }
    }
    rstd = 1.f / sqrtf(sum(q) * inv_d + a.eps);
  };
  stat(f, a.post);
  if (t == 0) {
    a.stats[row] = mean;
    a.stats[(size_t)a.N + row] = rstd;
  }
  const float* gr = a.gate ? a.gate + gate_row(row, a.gate_rows) * a.d : nullptr;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int c = (t + j * nt) * 8;
    if (a.post) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[j][i] = (f[j][i] - mean) * rstd;
      float w[8];
      if (a.pw) {
        load8(a.pw, c, a.d, a.wvec, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[j][i] *= w[i];
      }
      if (a.pb) {
        load8(a.pb, c, a.d, a.wvec, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[j][i] += w[i];
      }
    }
    if (gr) {
      float w[8];
      load8(gr, c, a.d, a.wvec, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[j][i] *= w[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) h[j][i] = c + i < a.d ? a.alpha * h[j][i] + a.beta * f[j][i] : 0.f;
    store8((T*)a.ho + o, c, a.d, a.vec, h[j]);
  }
  stat(h, a.pre);
  if (t == 0) {
    a.stats[2 * (size_t)a.N + row] = mean;
    a.stats[3 * (size_t)a.N + row] = rstd;
  }
  if (!a.pre) return;
#pragma unroll
  for (int j = 0; j < VPT; ++j) {
    const int c = (t + j * nt) * 8;
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) h[j][i] = (h[j][i] - mean) * rstd;
    if (a.nw) {
      load8(a.nw, c, a.d, a.wvec, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[j][i] *= w[i];
    }
    if (a.nb) {
      load8(a.nb, c, a.d, a.wvec, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) h[j][i] += w[i];
    }
    store8((T*)a.no + o, c, a.d, a.vec, h[j]);
    if (a.nq) {   // of n as it is stored
#pragma unroll
      for (int i = 0; i < 8; ++i) h[j][i] = c + i < a.d ? to_f(from_f<T>(h[j][i])) : 0.f;
      put_codes(a.fmt, h[j], a.nq, a.ne, (size_t)row * a.D + c, c < a.D);
    }
  }
}

// Rows of any width: a block per row that reads it again for every sum.
template <typename T>
__global__ void __launch_bounds__(512) fwd_any_k(const Fwd a) {
  pdl_wait();
  pdl_trigger();
  __shared__ float sh[32];
  const int row = blockIdx.x;
  const size_t o = (size_t)row * a.d;
  const float inv_d = 1.f / a.d;
  const float* gr = a.gate ? a.gate + gate_row(row, a.gate_rows) * a.d : nullptr;
  float pm = 0.f, pr = 1.f, m = 0.f, r = 1.f;
  auto fval = [&](int c, float* x) { load8((const T*)a.f + o, c, a.d, a.vec, x); };
  auto hval = [&](int c, float* x) {   // h' before its rounding
    float f[8], w[8];
    fval(c, f);
    load8((const T*)a.h + o, c, a.d, a.vec, x);
    if (a.post) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = (f[i] - pm) * pr;
      if (a.pw) {
        load8(a.pw, c, a.d, a.wvec, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] *= w[i];
      }
      if (a.pb) {
        load8(a.pb, c, a.d, a.wvec, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] += w[i];
      }
    }
    if (gr) {
      load8(gr, c, a.d, a.wvec, w);
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
      put_codes(a.fmt, x, a.fq, a.fe, (size_t)row * a.D + c, c < a.D);
    }
    hval(c, x);
    store8((T*)a.ho + o, c, a.d, a.vec, x);
    if (!a.pre) continue;
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (x[i] - m) * r;
    if (a.nw) {
      load8(a.nw, c, a.d, a.wvec, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] *= w[i];
    }
    if (a.nb) {
      load8(a.nb, c, a.d, a.wvec, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] += w[i];
    }
    store8((T*)a.no + o, c, a.d, a.vec, x);
    if (a.nq) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = c + i < a.d ? to_f(from_f<T>(x[i])) : 0.f;
      put_codes(a.fmt, x, a.nq, a.ne, (size_t)row * a.D + c, c < a.D);
    }
  }
}

template <typename T>
void forward(const Fwd& a, cudaStream_t s) {
  const int nvec = a.D / 8;
  note_launch(1);
  if (nvec <= 128) {
    const int blocks = (a.N + 7) / 8;
    if (nvec <= 32) launch_pdl(fwd_reg_k<T, true, 1>, blocks, 256, 0, s, a);
    else if (nvec <= 64) launch_pdl(fwd_reg_k<T, true, 2>, blocks, 256, 0, s, a);
    else launch_pdl(fwd_reg_k<T, true, 4>, blocks, 256, 0, s, a);
  } else if (nvec <= 2048) {
    int vpt = 1;
    while (vpt < 4 && (nvec + vpt - 1) / vpt > 128) vpt *= 2;
    const int th = ((nvec + vpt - 1) / vpt + 31) / 32 * 32;
    if (vpt == 1) launch_pdl(fwd_reg_k<T, false, 1>, a.N, th, 0, s, a);
    else if (vpt == 2) launch_pdl(fwd_reg_k<T, false, 2>, a.N, th, 0, s, a);
    else launch_pdl(fwd_reg_k<T, false, 4>, a.N, th, 0, s, a);
  } else {
    launch_pdl(fwd_any_k<T>, a.N, 512, 0, s, a);
  }
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
  float* part;               // [chunks, 5, d] partial sums: dw_pre, db_pre, dw_post, db_post, dgate
  float* out[5];
  int N, d, D;
  int post, pre, gate_rows;
  float alpha, beta;
  int fmt, accumulate;
  bool vec, wvec;
  int rows, per_group, chunks;   // the chunks of rows that partial sums are of
};

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
template <typename T>
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
    load8((const T*)a.f + (size_t)n * a.d, c, a.d, a.vec, x);
  }
}

// G of row n, columns c .. (0 past d).
template <typename T>
__device__ __forceinline__ void grad8(const Bwd& a, int n, int c, float s1, float s2, float* G) {
  const size_t o = (size_t)n * a.d;
#pragma unroll
  for (int i = 0; i < 8; ++i) G[i] = 0.f;
  if (a.dho) load8((const T*)a.dho + o, c, a.d, a.vec, G);
  if (a.pre) {
    const float m = a.stats[2 * (size_t)a.N + n], r = a.stats[3 * (size_t)a.N + n];
    float u[8], x[8], w[8];
    load8((const T*)a.dn + o, c, a.d, a.vec, u);
    load8((const T*)a.ho + o, c, a.d, a.vec, x);
    if (a.nw) {
      load8(a.nw, c, a.d, a.wvec, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) u[i] *= w[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) G[i] += c + i < a.d ? r * (u[i] - s1 - (x[i] - m) * r * s2) : 0.f;
  }
}

// mean(u) (LayerNorm) and mean(u xh) of every row.
template <typename T>
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
    load8((const T*)a.dn + o, c, a.d, a.vec, u);
    load8((const T*)a.ho + o, c, a.d, a.vec, x);
    if (a.nw) {
      load8(a.nw, c, a.d, a.wvec, w);
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
template <typename T>
__global__ void __launch_bounds__(256) bwd_cols_k(const Bwd a) {
  pdl_wait();
  pdl_trigger();
  __shared__ float sh[8][256];
  const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5, c = (blockIdx.y * 32 + tx) * 8;
  int r0, r1;
  chunk_rows(blockIdx.x, a.N, a.gate_rows ? a.gate_rows : a.N, a.rows, a.per_group, r0, r1);
  float acc[5][8];
#pragma unroll
  for (int k = 0; k < 5; ++k)
#pragma unroll
    for (int i = 0; i < 8; ++i) acc[k][i] = 0.f;
  // the sum over the row lanes of acc[k] at this thread's column blockIdx.y * 256 + threadIdx.x
  auto join = [&](int k) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) sh[ty][tx * 8 + i] = acc[k][i];
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
      grad8<T>(a, n, c, a.pre ? a.s12[n] : 0.f, a.pre ? a.s12[(size_t)a.N + n] : 0.f, G);
      if (a.pre) {
        const float m = a.stats[2 * (size_t)a.N + n], r = a.stats[3 * (size_t)a.N + n];
        load8((const T*)a.dn + (size_t)n * a.d, c, a.d, a.vec, w);
        load8((const T*)a.ho + (size_t)n * a.d, c, a.d, a.vec, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          acc[0][i] += w[i] * ((x[i] - m) * r);
          acc[1][i] += w[i];
        }
      }
      f8<T>(a, n, c, x);
      const float pm = a.stats[n], pr = a.stats[(size_t)a.N + n];
      float gt[8], b[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) { gt[i] = 1.f; w[i] = 1.f; b[i] = 0.f; }
      if (a.gate) load8(a.gate + gate_row(n, a.gate_rows) * a.d, c, a.d, a.wvec, gt);
      if (a.pw) load8(a.pw, c, a.d, a.wvec, w);
      if (a.pb) load8(a.pb, c, a.d, a.wvec, b);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float fh = a.post ? (x[i] - pm) * pr : x[i], q = a.beta * G[i];
        acc[2][i] += gt[i] * q * fh;
        acc[3][i] += gt[i] * q;
        acc[4][i] += q * (fh * w[i] + b[i]);
      }
    }
    if (a.out[4] && !a.per_group) {
      const float s = join(4);
      if (col < a.d) {
        float* p = a.out[4] + gate_row(g0, a.gate_rows) * a.d + col;
        *p = a.accumulate ? *p + s : s;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) acc[4][i] = 0.f;
    }
  }
#pragma unroll
  for (int k = 0; k < 5; ++k) {
    if (!a.out[k] || (k == 4 && !a.per_group)) continue;
    const float s = join(k);
    if (col < a.d) a.part[((size_t)blockIdx.x * 5 + k) * a.d + col] = s;
  }
}

// The chunks' partial sums in order: blockIdx.y 0..3 the parameters, 4 + g gate group g.
__global__ void __launch_bounds__(256) bwd_join_k(const Bwd a) {
  pdl_wait();
  pdl_trigger();
  const int c = blockIdx.x * 256 + threadIdx.x;
  if (c >= a.d) return;
  for (int y = blockIdx.y; y < 4 + (a.per_group ? a.chunks / a.per_group : 0); y += gridDim.y) {
    const int k = min(y, 4);
    if (!a.out[k]) continue;
    const int b0 = k < 4 ? 0 : (y - 4) * a.per_group, b1 = k < 4 ? a.chunks : b0 + a.per_group;
    float s = 0.f;
    for (int b = b0; b < b1; ++b) s += a.part[((size_t)b * 5 + k) * a.d + c];
    float* p = a.out[k] + (k < 4 ? 0 : (size_t)(y - 4) * a.d) + c;
    *p = a.accumulate ? *p + s : s;
  }
}

// dh and df of every row.
template <typename T>
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
    grad8<T>(a, n, c, s1, s2, G);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = a.beta * G[i];
    if (gr) {
      load8(gr, c, a.d, a.wvec, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= w[i];
    }
    if (!a.post) return;
    if (a.pw) {
      load8(a.pw, c, a.d, a.wvec, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] *= w[i];
    }
    f8<T>(a, n, c, fh);
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
    if (a.dh) store8((T*)a.dh + o, c, a.d, a.vec, G);
    store8((T*)a.df + o, c, a.d, a.vec, v);
  }
}

constexpr int kChunkRows = 64;

void plan_chunks(const zl_block_norm& p, int& rows, int& per_group, int& chunks) {
  const int gr = p.gate_rows && p.gate_rows < p.N ? p.gate_rows : std::max(p.N, 1);
  if (gr > kChunkRows) {
    per_group = (gr + kChunkRows - 1) / kChunkRows;
    rows = (gr + per_group - 1) / per_group;
    chunks = (p.N + gr - 1) / gr * per_group;
  } else {
    per_group = 0;
    rows = kChunkRows / gr * gr;
    chunks = (p.N + rows - 1) / rows;
  }
}

template <typename T>
void backward(const Bwd& a, cudaStream_t s) {
  if (a.pre) {
    note_launch(1);
    launch_pdl(bwd_sums_k<T>, a.N, 256, 0, s, a);
  }
  bool sums = false;
  for (float* o : a.out) sums |= o != nullptr;
  if (sums) {   // before dh, which may overwrite dh_out
    note_launch(2);
    launch_pdl(bwd_cols_k<T>, dim3(a.chunks, (a.d + 255) / 256), 256, 0, s, a);
    const int ys = 4 + (a.per_group ? a.chunks / a.per_group : 0);
    launch_pdl(bwd_join_k, dim3((a.d + 255) / 256, std::min(ys, 65535)), 256, 0, s, a);
  }
  note_launch(1);
  launch_pdl(bwd_rows_k<T>, a.N, 256, 0, s, a);
}

size_t up256(size_t b) { return (b + 255) / 256 * 256; }

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
bool al16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

}  // namespace
}  // namespace zl

using namespace zl;
using zl::act8::entry;
using zl::act8::launched;
using zl::act8::rows_aligned;

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
    Fwd a = {};
    a.h = h; a.f = f; a.pw = post_w; a.pb = post_b; a.gate = gate; a.nw = pre_w; a.nb = pre_b;
    a.ho = h_out; a.no = n_out; a.stats = stats; a.fq = f_q; a.fe = f_e; a.nq = n_q; a.ne = n_e;
    a.N = p->N; a.d = p->d; a.D = act8::pitch(p->d); a.post = p->post_norm; a.pre = p->pre_norm; a.gate_rows = p->gate_rows;
    a.eps = p->eps; a.alpha = p->res_scale; a.beta = p->branch_scale; a.fmt = p->fmt;
    a.vec = true;
    for (const void* t : {h, f, (const void*)h_out, (const void*)n_out}) a.vec &= !t || rows_aligned(t, p->d, p->dtype);
    a.wvec = al16(post_w) && al16(post_b) && al16(pre_w) && al16(pre_b) && (!gate || rows_aligned(gate, p->d, ZL_DTYPE_F32));
    if (p->dtype == ZL_DTYPE_BF16) forward<bf16>(a, (cudaStream_t)stream);
    else forward<float>(a, (cudaStream_t)stream);
    return launched("zl_op_block_norm");
  });
}

zl_status zl_op_block_norm_bwd_bytes(const zl_block_norm* p, size_t* bytes) {
  return entry([&]() -> zl_status {
    if (!dims_ok(p) || !bytes) return act8::fail(ZL_ERR_ARG, kDimsMsg);
    int rows, per_group, chunks;
    plan_chunks(*p, rows, per_group, chunks);
    *bytes = p->N ? up256((size_t)p->N * 8) + up256((size_t)chunks * 5 * p->d * 4) : 0;
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
      return act8::fail(ZL_ERR_ARG, "a weight or its gradient without its norm, a bias gradient without a LayerNorm, or dgate without gate");
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
    size_t need = 0;
    zl_op_block_norm_bwd_bytes(p, &need);
    if (!ws || ((uintptr_t)ws & 255u) || ws_bytes < need)
      return act8::fail(ZL_ERR_ARG, "the workspace must be 256-byte aligned and hold zl_op_block_norm_bwd_bytes() bytes");
    Bwd a = {};
    a.ho = h_out; a.f = f; a.fq = f_q; a.fe = f_e; a.pw = post_w; a.pb = post_b; a.gate = gate; a.nw = pre_w; a.stats = stats;
    a.dn = dn; a.dho = dh_out; a.dh = dh; a.df = df;
    a.s12 = (float*)ws;
    a.part = (float*)((char*)ws + up256((size_t)p->N * 8));
    a.out[0] = dpre_w; a.out[1] = dpre_b; a.out[2] = dpost_w; a.out[3] = dpost_b; a.out[4] = dgate;
    a.N = p->N; a.d = p->d; a.D = act8::pitch(p->d); a.post = p->post_norm; a.pre = p->pre_norm;
    a.gate_rows = p->gate_rows < p->N ? p->gate_rows : 0;   // one group holds every row
    a.alpha = p->res_scale; a.beta = p->branch_scale; a.fmt = p->fmt; a.accumulate = p->accumulate;
    plan_chunks(*p, a.rows, a.per_group, a.chunks);
    a.vec = true;
    for (const void* t : {h_out, f, dn, dh_out, (const void*)dh, (const void*)df}) a.vec &= !t || rows_aligned(t, d, p->dtype);
    a.wvec = al16(post_w) && al16(post_b) && al16(pre_w) && (!gate || rows_aligned(gate, d, ZL_DTYPE_F32));
    if (p->dtype == ZL_DTYPE_BF16) backward<bf16>(a, s);
    else backward<float>(a, s);
    return launched("zl_op_block_norm_bwd");
  });
}

}  // extern "C"
