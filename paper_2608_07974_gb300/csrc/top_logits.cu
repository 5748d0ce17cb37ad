// A teacher of whom only the top of its logits is kept: the record of a row (zl_op_top_logits) and the local objective
// against such records (zl_op_top_loss). Rows start anywhere: the values before a row's first 16-byte word and behind its
// last whole one are read and written one at a time, all others 16 bytes at a time.
#include <algorithm>
#include <cmath>

#include "act8.cuh"
#include "common.cuh"
#include "ops.h"
#include "per_device.h"
#include "tcgen05.cuh"
#include "vocab.cuh"

namespace zl {
namespace top {

using vocab::ex2;
using vocab::kL2e;
using vocab::kLn2;
using vocab::Lse;

constexpr int kThreads = 256, kBlocks = 4;   // of a CTA; CTAs an SM
constexpr int kWarps = kThreads / 32;
constexpr int kMaxSplit = 8;              // CTAs of a cluster that share a row

// A row of n values from p: `head` values before its first 16-byte word, `words` whole words, then the rest.
template <typename T>
struct Span {
  static constexpr int W = 16 / (int)sizeof(T);
  int head, words, tail;
  __device__ Span(const T* p, int n) {
    head = min(n, (int)((0u - (uint32_t)(uintptr_t)p) & 15u) / (int)sizeof(T));
    words = (n - head) / W;
    tail = head + words * W;
  }
  // Column of word i; of the i-th value outside the words (fewer than 2 W of them).
  __device__ int word_at(int i) const { return head + i * W; }
  __device__ int single_at(int i) const { return i < head ? i : tail + i - head; }
  __device__ int singles(int n) const { return n - words * W; }
};

// A row's words are shared by the CTAs of a cluster; each takes a slice of neighbouring words, which it reads twice, the second time
// from L2. (Kept in shared memory instead, filled by bulk copies or by the threads, a row of 100 KB leaves room for two CTAs an SM,
// whose steps between the passes then show: 4096 x 50257 bf16, top 64, 148 to 172 us against 122 with four CTAs and no copy.)
struct Slice {
  int first, n;   // the slice's first word in the row, its words
  const uint4* src;
  __device__ Slice(const uint4* row, int words, int rank, int split) {
    const int per = split > 1 ? (words + split - 1) / split : words;
    first = min(rank * per, words);
    n = min(per, words - first);
    src = row + first;
  }
  // Has the slice brought to L2, while other things are done before the first pass.
  __device__ __forceinline__ void prefetch() const {
#pragma unroll 1
    for (int i = (int)threadIdx.x * 8; i < n; i += kThreads * 8) asm volatile("prefetch.global.L2 [%0];" ::"l"(src + i));
  }
  // fn(word, its number in the slice, 0 or 1 in turn) for this thread's words.
  template <typename F>
  __device__ __forceinline__ void pass(F&& fn) const {
    constexpr int U = 6;   // words under way (4: 128 and 182 us where 6 takes 121 and 173; 8 spills)
    int i = (int)threadIdx.x;
#pragma unroll 1
    for (; i + (U - 1) * kThreads < n; i += U * kThreads) {
      uint4 r[U];
#pragma unroll
      for (int u = 0; u < U; ++u) r[u] = src[i + u * kThreads];
#pragma unroll
      for (int u = 0; u < U; ++u) fn(r[u], i + u * kThreads, u & 1);
    }
#pragma unroll 1
    for (; i < n; i += kThreads) fn(src[i], i, 0);
  }
};
// Has a row of `bytes` brought to L2 by the CTAs that share one.
__device__ __forceinline__ void prefetch_row(const void* p, int bytes, int rank, int split) {
#pragma unroll 1
  for (int at = (rank * kThreads + (int)threadIdx.x) * 128; at < bytes; at += split * kThreads * 128)
    asm volatile("prefetch.global.L2 [%0];" ::"l"((const char*)p + at));
}
// The same variable in CTA `rank` of the cluster.
template <typename U>
__device__ __forceinline__ U* peer(U* p, int rank) {
  U* r;
  asm("mapa.u64 %0, %1, %2;" : "=l"(r) : "l"(p), "r"(rank));
  return r;
}
// The two halves of a barrier over the cluster: other CTAs' shared memory may be used once all have arrived.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// The values of a 16-byte word.
__device__ __forceinline__ void word_floats(const uint4& u, float (&x)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void word_floats(const uint4& u, float (&x)[4]) {
  x[0] = __uint_as_float(u.x); x[1] = __uint_as_float(u.y); x[2] = __uint_as_float(u.z); x[3] = __uint_as_float(u.w);
}
__device__ __forceinline__ uint32_t max_nan_bf2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// The largest of a word's values (a NaN if one is among them).
template <typename T>
__device__ __forceinline__ float word_max(const uint4& u) {
  if (sizeof(T) == 2) {
    const uint32_t m = max_nan_bf2(max_nan_bf2(u.x, u.y), max_nan_bf2(u.z, u.w));
    return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u));
  }
  return max_nan(max_nan(__uint_as_float(u.x), __uint_as_float(u.y)), max_nan(__uint_as_float(u.z), __uint_as_float(u.w)));
}

// A word's values whose bits are set in m become -inf.
template <typename T>
__device__ __forceinline__ void mask_word(uint4& u, uint32_t m) {
  if (sizeof(T) == 2) {
    auto one = [](uint32_t w, uint32_t two) {
      const uint32_t k = (two & 1u) * 0xFFFFu | (two >> 1) * 0xFFFF0000u;
      return (w & ~k) | (0xFF80FF80u & k);
    };
    u.x = one(u.x, m & 3u); u.y = one(u.y, m >> 2 & 3u); u.z = one(u.z, m >> 4 & 3u); u.w = one(u.w, m >> 6);
  } else {
    u.x = m & 1u ? 0xFF800000u : u.x; u.y = m & 2u ? 0xFF800000u : u.y;
    u.z = m & 4u ? 0xFF800000u : u.z; u.w = m & 8u ? 0xFF800000u : u.w;
  }
}

// The order of logits as whole numbers: larger value, larger key; -0 is 0, every NaN above +inf.
__device__ __forceinline__ uint32_t key_of(float x) {
  if (x != x) return 0xFFFFFFFFu;
  const uint32_t u = __float_as_uint(x + 0.f);   // (-0 + 0 = 0)
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return key == 0xFFFFFFFFu ? __uint_as_float(0x7FC00000u) : __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key);
}
// The value at or below every T whose key has this upper half, and above all whose upper half is smaller.
template <typename T>
__device__ __forceinline__ float floor_of_half(uint32_t half) {
  const uint32_t k = half << 16;
  const uint32_t u = k & 0x80000000u ? k & 0x7FFFFFFFu : sizeof(T) == 2 ? ~k & 0xFFFF0000u : ~k;
  const float x = __uint_as_float(u);
  return x == x ? x : (k & 0x80000000u ? __uint_as_float(0x7FC00000u) : -INFINITY);
}
// Whether all of a word's values are below a bound (a NaN is not; bf16: the bound twice in `pair`, it is a bf16).
template <typename T>
__device__ __forceinline__ bool word_below(const uint4& u, float bound, uint32_t pair) {
  if (sizeof(T) == 2) {
    const uint32_t m = max_nan_bf2(max_nan_bf2(u.x, u.y), max_nan_bf2(u.z, u.w));
    uint32_t r;
    asm("{\n .reg .pred p, q;\n setp.lt.bf16x2 p|q, %1, %2;\n and.pred p, p, q;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(r) : "r"(m), "r"(pair));
    return r != 0u;
  }
  return word_max<T>(u) < bound;
}

// ------------------------------------------------------------------------------------------------
// The record of a row: the k largest logits in falling order (of equal ones the lower column first), and
// rest = log sum_{others} e^{z / T}.
//
// Two passes over the row. The first keeps 8 running maxima a thread, joined to 2 k "bins" or somewhat more. The k-th largest bin is a
// bound that at least k logits reach, and (the k largest lie in n bins like so many balls) about n log(n / (n - k)) of them, 1.4 k for
// n = 2 k. It is found to the upper 16 bits of its key by a search of 8 rounds of three counts: of up to 512 bins by one warp, without
// a barrier, of more by all. The second pass notes the words that reach the bound and sums the rest relative to it. Each candidate's
// place is the number of candidates before it. Rows with too many candidates (many equal logits) find the k-th key exactly, byte by
// byte.
// A row is shared by a cluster where it is long or rows are few: its CTAs exchange their bins, all find the same bound, and the
// first one takes their candidates and sums.
// 4096 x 50257 bf16, k 64: 106 us, 3.9 TB/s of the one reading (57% of the copy rate): the search and what follows the second pass are
// latency (warps wait for loads and at barriers, 0.6 instructions a cycle). 509 x 32000 fp32, k 256: 28 us, as a call among others 34.
// ------------------------------------------------------------------------------------------------
struct TopArgs {
  int N, V, ld, k, split, bins, cap;   // CTAs a row, bins of one, room for candidates
  int ahead;                           // see rows_ahead()
  float scale, T;                   // log2 e / T
  int32_t* idx;
  float* val;
  float* rest;
};

// 8 running maxima.
template <typename T>
struct Bins;
template <>
struct Bins<bf16> {
  static constexpr int N = 8;
  uint32_t b[4];
  __device__ void clear() { b[0] = b[1] = b[2] = b[3] = 0xFF80FF80u; }
  __device__ void add(const uint4& u, int) {
    b[0] = max_nan_bf2(b[0], u.x); b[1] = max_nan_bf2(b[1], u.y); b[2] = max_nan_bf2(b[2], u.z); b[3] = max_nan_bf2(b[3], u.w);
  }
  __device__ void add(float x) { b[0] = max_nan_bf2(b[0], __float_as_uint(x) >> 16 | 0xFF800000u); }
  // The upper half of the key of maximum i, and of the largest of all.
  __device__ uint32_t key(int i) const {
    uint32_t w = b[0];
#pragma unroll
    for (int e = 1; e < 4; ++e) w = (i >> 1) == e ? b[e] : w;
    return key_of(__uint_as_float(i & 1 ? w & 0xffff0000u : w << 16)) >> 16;
  }
  __device__ uint32_t top_key() const {
    const uint32_t m = max_nan_bf2(max_nan_bf2(b[0], b[1]), max_nan_bf2(b[2], b[3]));
    return key_of(max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u))) >> 16;
  }
};
template <>
struct Bins<float> {
  static constexpr int N = 8;
  float b[8];
  __device__ void clear() {
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = -INFINITY;
  }
  __device__ void add(const uint4& u, int turn) {
    float* const c = b + 4 * turn;
    c[0] = max_nan(c[0], __uint_as_float(u.x)); c[1] = max_nan(c[1], __uint_as_float(u.y));
    c[2] = max_nan(c[2], __uint_as_float(u.z)); c[3] = max_nan(c[3], __uint_as_float(u.w));
  }
  __device__ void add(float x) { b[0] = max_nan(b[0], x); }
  __device__ uint32_t key(int i) const {
    float x = b[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) x = e == i ? b[e] : x;
    return key_of(x) >> 16;
  }
  __device__ uint32_t top_key() const {
    float x = b[0];
#pragma unroll
    for (int e = 1; e < 8; ++e) x = max_nan(x, b[e]);
    return key_of(x) >> 16;
  }
};

struct TopShared {
  uint32_t count[8][2];
  uint32_t hist[256];
  Lse part[kWarps], sum;
  uint32_t lo;
  int n, words;
};
// Dynamic shared memory: the candidates (key, then the column's complement: the record's order is their falling order) and the
// words that hold them, before them in the same place the bins of every CTA, then the candidates behind the record.
__host__ __device__ inline int top_lists(int split, int bins, int cap) {
  const int c = cap * 12 + 16, b = split * bins * 2;
  return ((c > b ? c : b) + 15) / 16 * 16;
}
int top_dyn(int split, int bins, int cap) { return top_lists(split, bins, cap) + cap * 4; }

// The next two bits of the search from the counts of bins at or above lo + 1, 2 and 3 << shift.
__device__ __forceinline__ uint32_t narrow(uint32_t lo, int shift, int c1, int c2, int c3, int k) {
  return lo + ((c3 >= k ? 3u : c2 >= k ? 2u : c1 >= k ? 1u : 0u) << shift);
}
// The largest t (upper half of a key) that at least k of 32 M bins reach, by one warp.
template <int M>
__device__ __forceinline__ uint32_t search_warp(const uint16_t* bins, int k) {
  uint32_t h[M];
#pragma unroll
  for (int i = 0; i < M; ++i) h[i] = bins[32 * i + (threadIdx.x & 31)];
  uint32_t lo = 0;
#pragma unroll 1
  for (int shift = 14; shift >= 0; shift -= 2) {
    const uint32_t t1 = lo + (1u << shift), t2 = t1 + (1u << shift), t3 = t2 + (1u << shift);
    uint32_t c = 0;
#pragma unroll
    for (int i = 0; i < M; ++i) c += (h[i] >= t1 ? 1u : 0u) + (h[i] >= t2 ? 1u << 10 : 0u) + (h[i] >= t3 ? 1u << 20 : 0u);
    c = __reduce_add_sync(0xffffffffu, c);   // (at most 512 each)
    lo = narrow(lo, shift, (int)(c & 1023u), (int)(c >> 10 & 1023u), (int)(c >> 20), k);
  }
  return lo;
}
// The same of kThreads N bins, by the block; sh.count is 0 before it.
template <int N>
__device__ __forceinline__ uint32_t search_block(const uint16_t* bins, int k, TopShared& sh) {
  uint32_t h[N];
#pragma unroll
  for (int i = 0; i < N; ++i) h[i] = bins[i * kThreads + threadIdx.x];
  uint32_t lo = 0;
#pragma unroll 1
  for (int round = 0; round < 8; ++round) {
    const int shift = 14 - 2 * round;
    const uint32_t t1 = lo + (1u << shift), t2 = t1 + (1u << shift), t3 = t2 + (1u << shift);
    uint32_t c12 = 0, c3 = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      c12 += (h[i] >= t1 ? 1u : 0u) + (h[i] >= t2 ? 1u << 16 : 0u);
      c3 += h[i] >= t3 ? 1u : 0u;
    }
    c12 = __reduce_add_sync(0xffffffffu, c12);
    c3 = __reduce_add_sync(0xffffffffu, c3);
    if ((threadIdx.x & 31) == 0) {
      atomicAdd(&sh.count[round][0], c12);
      atomicAdd(&sh.count[round][1], c3);
    }
    __syncthreads();
    c12 = sh.count[round][0];
    lo = narrow(lo, shift, (int)(c12 & 0xffffu), (int)(c12 >> 16), (int)sh.count[round][1], k);
  }
  return lo;
}

// The k-th largest key of a row and how many keys are above it, byte by byte from the top.
template <typename T>
__device__ uint32_t kth_key(const T* z, int V, int k, TopShared& sh, int& above) {
  uint32_t prefix = 0, mask = 0;
  int left = k;
#pragma unroll 1
  for (int shift = 24; shift >= 0; shift -= 8) {
    __syncthreads();
    if (threadIdx.x < 256) sh.hist[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll 1
    for (int c = threadIdx.x; c < V; c += kThreads) {
      const uint32_t key = key_of(to_f(z[c]));
      if ((key & mask) == prefix) atomicAdd(&sh.hist[key >> shift & 255u], 1u);
    }
    __syncthreads();
    int b = 255;   // (every thread the same walk)
#pragma unroll 1
    for (; b > 0 && (int)sh.hist[b] < left; --b) left -= (int)sh.hist[b];
    prefix |= (uint32_t)b << shift;
    mask |= 255u << shift;
  }
  above = k - left;
  return prefix;
}

// This thread's share of the sum over the values below a bound, whatever their size. (The rare ways through the kernel are functions
// of their own: what is hardly ever run should not stand between what always is.)
template <typename T>
__device__ __noinline__ Lse sum_below(const T* p, int n, float bound, float scale) {
  Lse A = vocab::lse_empty();
#pragma unroll 1
  for (int i = threadIdx.x; i < n; i += kThreads) {
    const float x = to_f(p[i]);
    if (x < bound) vocab::lse_add1(A, x, scale);
  }
  return A;
}
// The k largest of a row of any values into cand, the warps' sums over the others into sh.part.
template <typename T>
__device__ __noinline__ void exact_record(const T* z, int V, int k, float scale, uint64_t* cand, TopShared& sh) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int above;
  const uint32_t key = kth_key(z, V, k, sh, above);
  __syncthreads();
  if (tid == 0) sh.n = 0;
  Lse A = vocab::lse_empty();
  int taken = 0;
  __syncthreads();
  // of those at the k-th key the first k - above columns, in order
#pragma unroll 1
  for (int c0 = 0; c0 < V; c0 += kThreads) {
    const int c = c0 + tid;
    const float x = c < V ? to_f(z[c]) : 0.f;
    const uint32_t kc = c < V ? key_of(x) : 0u;
    const bool eq = c < V && kc == key;
    const uint32_t ball = __ballot_sync(0xffffffffu, eq);
    if (lane == 0) sh.hist[warp] = __popc(ball);
    __syncthreads();
    int before = taken + __popc(ball & ((1u << lane) - 1u));
#pragma unroll 1
    for (int w = 0; w < kWarps; ++w) {
      const int m = (int)sh.hist[w];
      before += w < warp ? m : 0;
      taken += m;
    }
    if (c < V) {
      if (kc > key || (eq && before < k - above)) cand[atomicAdd(&sh.n, 1)] = (uint64_t)kc << 32 | (uint32_t)~c;
      else vocab::lse_add1(A, x, scale);
    }
    __syncthreads();
  }
  A = vocab::warp_merge(A, scale);
  if (lane == 0) sh.part[warp] = A;
  __syncthreads();
}

// Sorts n keys in falling order, by the block: a bitonic network over the next power of two, whose keys past n are 0 and lie behind
// every other.
__device__ __noinline__ void sort_falling(uint64_t* c, int n) {
  int size = 32;
  while (size < n) size *= 2;
  for (int i = n + (int)threadIdx.x; i < size; i += kThreads) c[i] = 0ull;
  __syncthreads();
#pragma unroll 1
  for (int len = 2; len <= size; len *= 2) {
#pragma unroll 1
    for (int step = len / 2; step > 0; step /= 2) {
#pragma unroll 1
      for (int t = threadIdx.x; t < size / 2; t += kThreads) {
        const int i = 2 * t - (t & (step - 1)), j = i + step;
        const uint64_t x = c[i], y = c[j];
        if ((x < y) == ((i & len) == 0)) {
          c[i] = y;
          c[j] = x;
        }
      }
      __syncthreads();
    }
  }
}

template <typename T>
__global__ void __launch_bounds__(kThreads, kBlocks) top_logits_k(const T* __restrict__ z0, const TopArgs a) {
  pdl_wait();
  pdl_trigger();
  __shared__ TopShared sh;
  extern __shared__ __align__(16) uint8_t dyn[];
  constexpr int W = Span<T>::W;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int split = a.split, rank = split > 1 ? (int)tc::cluster_rank() : 0;
  const size_t row = split > 1 ? blockIdx.x / split : blockIdx.x;
  const int cap = a.cap, k = a.k;
  uint64_t* const cand = reinterpret_cast<uint64_t*>(dyn);
  int* const noted = reinterpret_cast<int*>(cand + cap + 2);
  uint16_t* const bins = reinterpret_cast<uint16_t*>(dyn);
  float* const left = reinterpret_cast<float*>(dyn + top_lists(split, a.bins, cap));
  const T* const z = z0 + row * a.ld;
  const Span<T> sp(z, a.V);
  const Slice sl(reinterpret_cast<const uint4*>(z + sp.head), sp.words, rank, split);
  if (tid == 0) sh.n = sh.words = 0;
  if (tid < 16) (&sh.count[0][0])[tid] = 0u;
  if (split > 1) cluster_arrive();
  const int ns = rank == 0 ? sp.singles(a.V) : 0;
  const float single = tid < ns ? to_f(z[sp.single_at(tid)]) : 0.f;
  Bins<T> mine;
  mine.clear();
  sl.pass([&](const uint4& u, int, int turn) { mine.add(u, turn); });
  if (tid < ns) mine.add(single);
  // This CTA's bins (an empty one counts as -inf): several of a thread, or one of several neighbouring threads; to every CTA.
  if (split > 1) cluster_wait();
  auto put = [&](int i, uint32_t key) {
    if (split == 1) {
      bins[i] = (uint16_t)key;
    } else {
#pragma unroll 1
      for (int r = 0; r < split; ++r) peer(bins, r)[rank * a.bins + i] = (uint16_t)key;
    }
  };
  if (a.bins <= kThreads) {
    uint32_t key = mine.top_key();
    for (int o = 1; o * a.bins < kThreads; o *= 2) key = max(key, __shfl_xor_sync(0xffffffffu, key, o));
    const int share = kThreads / a.bins;
    if (tid % share == 0) put(tid / share, key);
  } else {
#pragma unroll 1
    for (int i = 0; i < a.bins / kThreads; ++i) {   // (kThreads of them at a time; 2: of each four maxima)
      uint32_t key = mine.key(i);
#pragma unroll 1
      for (int e = i + a.bins / kThreads; e < Bins<T>::N; e += a.bins / kThreads) key = max(key, mine.key(e));
      put(i * kThreads + tid, key);
    }
  }
  if (split > 1) tc::cluster_sync();
  else __syncthreads();
  const int all = split * a.bins;
  if (all <= 512) {
    if (warp == 0) {
      const uint32_t lo = all == 512   ? search_warp<16>(bins, k)
                          : all == 256 ? search_warp<8>(bins, k)
                          : all == 128 ? search_warp<4>(bins, k)
                                       : search_warp<2>(bins, k);
      if (lane == 0) sh.lo = lo;
    }
  } else {
    const uint32_t lo = all == 1024 ? search_block<1024 / kThreads>(bins, k, sh) : search_block<2048 / kThreads>(bins, k, sh);
    if (tid == 0) sh.lo = lo;
  }
  __syncthreads();   // (the candidates take the bins' place)
  const float bound = floor_of_half<T>(sh.lo);
  const uint32_t pair = __float_as_uint(bound) >> 16 | (__float_as_uint(bound) & 0xFFFF0000u);
  // note the words with values not below the bound (a NaN is not), sum all that is: relative to the bound, which none exceeds
  const bool fixed = fabsf(bound) < INFINITY;
  const float ref = fixed ? bound : 0.f;
  const uint64_t s2 = f2(a.scale, a.scale), nr = f2(-ref, -ref);
  uint64_t sum2 = 0ull;
  sl.pass([&](const uint4& u, int i, int) {
    float x[W];
    word_floats(u, x);
    if (!word_below<T>(u, bound, pair)) {
      const int at = atomicAdd(&sh.words, 1);
      if (at < cap) noted[at] = i;
#pragma unroll
      for (int e = 0; e < W; ++e) x[e] = x[e] < bound ? x[e] : -INFINITY;
    }
    uint64_t t = 0ull;
#pragma unroll
    for (int e = 0; e < W; e += 2) {
      const float2 v = uf2(mul2(add2(f2(x[e], x[e + 1]), nr), s2));
      const uint64_t p = f2(ex2(v.x), ex2(v.y));
      t = e == 0 ? p : add2(t, p);
    }
    sum2 = add2(sum2, t);
  });
  if ((size_t)a.N - row > (size_t)a.ahead) prefetch_row(z + (size_t)a.ahead * a.ld, a.V * (int)sizeof(T), rank, split);
  const float2 lanes = uf2(sum2);
  float sum = lanes.x + lanes.y;
  const bool single_in = tid < ns && !(single < bound);
  if (tid < ns && single < bound) sum += ex2((single - ref) * a.scale);
  // (a bound that is not finite is no reference; and where every thread's sum is tiny, its terms lie so far below the bound that
  // they lost digits)
  const bool good = __syncthreads_or(fixed && sum >= 0x1p-60f);
  sum = warp_sum(sum);
  if (lane == 0) sh.part[warp] = Lse{bound, sum};
  if (!good) {
    Lse A = sum_below<T>(reinterpret_cast<const T*>(sl.src), sl.n * W, bound, a.scale);
    if (tid < ns && single < bound) vocab::lse_add1(A, single, a.scale);
    A = vocab::warp_merge(A, a.scale);
    if (lane == 0) sh.part[warp] = A;
  }
  // the noted words' candidates, two values a thread at a time
  const bool over = sh.words > cap;
  const int values = over ? 0 : sh.words * W;
  auto push = [&](bool is, float x, int c) {
    const uint32_t ball = __ballot_sync(0xffffffffu, is);
    if (ball == 0u) return;
    int at = 0;
    if (lane == 0) at = atomicAdd(&sh.n, __popc(ball));
    at = __shfl_sync(0xffffffffu, at, 0) + __popc(ball & ((1u << lane) - 1u));
    if (is && at < cap) cand[at] = (uint64_t)key_of(x) << 32 | (uint32_t)~c;
  };
  if (warp == 0) push(single_in, single, sp.single_at(tid));
#pragma unroll 1
  for (int i0 = tid - lane; i0 < values; i0 += 2 * kThreads) {
    int wd[2];
    T x[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int i = i0 + lane + u * kThreads;
      wd[u] = i < values ? noted[i / W] : -1;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
      if (wd[u] >= 0) x[u] = reinterpret_cast<const T*>(sl.src)[(size_t)wd[u] * W + (lane & (W - 1))];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const bool in = wd[u] >= 0;
      const float f = in ? to_f(x[u]) : 0.f;
      push(in && !(f < bound), f, sp.word_at(sl.first + wd[u]) + (lane & (W - 1)));
    }
  }
  __syncthreads();
  int n = over ? cap + 1 : sh.n;
  Lse A = vocab::lse_empty();   // (the first warp's)
  if (warp == 0) A = vocab::warp_merge(lane < kWarps ? sh.part[lane] : vocab::lse_empty(), a.scale);
  if (split > 1) {   // to the first CTA
    if (tid == 0) {
      sh.sum = A;
      sh.n = n;
    }
    tc::cluster_sync();
    if (rank != 0) {
      tc::cluster_sync();   // it has read this one's
      return;
    }
#pragma unroll 1
    for (int r = 1; r < split; ++r) {
      const TopShared* const p = peer(&sh, r);
      const int m = p->n;
      if (n + m <= cap) {
        const uint64_t* const from = peer(cand, r);
#pragma unroll 1
        for (int i = tid; i < m; i += kThreads) cand[n + i] = from[i];
        n += m;
      } else {
        n = cap + 1;
      }
      if (warp == 0) A = vocab::lse_merge(A, *(const Lse*)&p->sum, a.scale);
    }
    tc::cluster_sync();
  }
  if (n > cap) {   // many equal logits
    exact_record(z, a.V, k, a.scale, cand, sh);
    n = k;
    if (warp == 0) A = vocab::warp_merge(lane < kWarps ? sh.part[lane] : vocab::lse_empty(), a.scale);
  }
  if (tid == 0) cand[n] = 0ull;   // (behind every key: two are read at a time)
  __syncthreads();
  auto give = [&](int p, uint64_t c) {   // candidate c has place p
    const float x = value_of((uint32_t)(c >> 32));
    if (p < k) {
      a.idx[row * k + p] = (int)~(uint32_t)c;
      a.val[row * k + p] = x;
    } else {
      left[p - k] = x;   // (collected in any order, summed in this one)
    }
  };
  // A candidate's place is the number of candidates before it: g lanes count for one. Many are sorted instead, since counting grows with
  // their square. 1216 x 32000 bf16, counted / sorted: 64 in the record (90 candidates) 28 / 32 us, 110 (150) 33.5 / 37.5, 160 (220) 40.5 / 42,
  // 256 (355) 53 / 54: level beyond some 200.
  if (n <= 160) {
    int g = 1;
    while (g < 8 && n * g * 2 <= kThreads) g *= 2;
    const int sub = tid & (g - 1), i = tid / g;
    if ((tid & ~31) / g < n) {   // (whole warps)
      const uint64_t own = i < n ? cand[i] : ~0ull;
      int p = 0;
      const ulonglong2* const c2 = reinterpret_cast<const ulonglong2*>(cand);
#pragma unroll 4
      for (int j = sub; j < (n + 1) / 2; j += g) {
        const ulonglong2 c = c2[j];
        p += (c.x > own ? 1 : 0) + (c.y > own ? 1 : 0);
      }
      for (int o = g >> 1; o > 0; o >>= 1) p += __shfl_xor_sync(0xffffffffu, p, o);
      if (i < n && sub == 0) give(p, own);
    }
  } else {
    sort_falling(cand, n);
#pragma unroll 1
    for (int i = tid; i < n; i += kThreads) give(i, cand[i]);
  }
  __syncthreads();
  if (warp == 0) {   // those behind the record lie between the bound and its last logit: relative to their first, the largest
    Lse B = vocab::lse_empty();
    if (n > k && left[0] != -INFINITY) {
      float t = 0.f;
#pragma unroll 1
      for (int i = lane; i < n - k; i += 32) t += ex2((left[i] - left[0]) * a.scale);
      B = Lse{left[0], warp_sum(t)};
    }
    A = vocab::lse_merge(A, B, a.scale);
    if (lane == 0) a.rest[row] = vocab::lse_value(A, 1.f / a.T);
  }
}

// ------------------------------------------------------------------------------------------------
// The local objective against records. Student classes c: the record's columns, and with `rest` one class of all others.
// With x = z / T, lse = log sum_v e^{x_v}, lp_c = x_c - lse (others: log sum_others e^{x} - lse), the teacher's
// lq_c = val_c / T (others: rest) less their log-sum-exp:
//   dir 0   KL(p || q) = sum_c p_c (lp_c - lq_c),   T dKL/dz_v = p_v (lp_c - lq_c - KL), c the class of v
//   dir 1   KL(q || p) = sum_c q_c (lq_c - lp_c),   T dKL/dz_v = p_v - q_v in the record, p_v (1 - q_r / p_r) else (p_v
//                                                    without `rest`: q lies in the record alone)
//   loss_i = alpha (log sum e^z - z_y) + (1 - alpha) T^2 KL
// The slice's columns in the record are marked in a bitmap in shared memory, a byte (fp32: half of one) for each 16-byte word,
// so that the first pass sums the other columns by themselves: their mass is no difference of sums. The second pass writes the
// gradient of the others, after which the record's columns and the label's are written over. The CTAs that share a row exchange
// their sums over the others, and each forms what goes by the record alone.
// 0 log 0 = 0 throughout; a record without any mass adds nothing, one with a NaN or +inf makes the row NaN.
// Bound by HBM (the row in, its gradient out): 4096 x 50257 bf16 165 us, 5.0 TB/s (74% of the copy rate). Where dz and z lie differently against
// 16 bytes the gradient leaves in single values, a word's neighbours in one thread: 520 us (fp32 327 against 287).
// ------------------------------------------------------------------------------------------------
// Up to so many rows every row counts |Omega| itself (2 KB of labels in L2 against a launch).
constexpr int kCountHere = 2 * kThreads;

struct LossArgs {
  const int32_t* idx;
  const float* val;
  const float* rest;
  const int32_t* labels;
  int N, V, ld, k, dir, count_here, split;
  float alpha, T;
  float* row_loss;
  float* loss;
};

// What a row's log-sum-exps and the teacher's come to, formed by one warp.
struct RowTerms {
  float lpr, lqr, omega;           // the rest's log probabilities; |Omega|
  // Sums s e^{m / T} as m, 1 / s and log s: of the others, all, all at T = 1 (those at T but for TWO), the teacher's. Probabilities and
  // their logarithms go by x - m, which is exact or nearly so, and not by x - log sum, whose rounding (2^-24 of 20 or 40, and of as many
  // over T) would be in all of a row's.
  float om, oi, pr, am, ai, al, cm, ci, cl, qm, qi, ql;   // pr: the others' probability
  int held;                        // the record holds something
  float bad;                       // NaN where the row or its record has no softmax (a NaN, +inf; a row of nothing but -inf), else 0
};
struct LossShared {
  Lse p[kWarps], c[kWarps], r[kWarps], q[kWarps];   // the warps' sums: others, all (TWO), record, teacher
  Lse others[kMaxSplit], all[kMaxSplit];            // of the row's CTAs
  int twice[kMaxSplit];
  float kl[kWarps];
  int n[kWarps];
  uint32_t singles;   // marks of the values outside the words
  RowTerms t;
};

// Bytes of a slice's bitmap.
int mark_bytes(int V, int W, int split) { return (((V / W + split) / split * W + 31) / 32 + 1) * 4; }
constexpr float kMasked = 1e38f;   // logits below -kMasked are masks
constexpr int kEntries = (ZL_TOP_MAX + kThreads - 1) / kThreads;   // of a record, a thread

// TWO: the task term's softmax is another one than the divergence's (T != 1, both terms).
template <typename T, bool TWO>
__global__ void __launch_bounds__(kThreads, kBlocks) top_loss_k(const T* z0, T* dz0, const LossArgs a) {
  pdl_wait();
  pdl_trigger();
  __shared__ LossShared sh;
  extern __shared__ uint32_t bits[];   // the slice's marks
  constexpr int W = Span<T>::W;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int split = a.split, rank = split > 1 ? (int)tc::cluster_rank() : 0;
  const size_t row = split > 1 ? blockIdx.x / split : blockIdx.x;
  const T* const z = z0 + row * a.ld;
  T* const dz = dz0 + row * a.ld;
  const bool kl_on = a.alpha < 1.f;
  const int k = kl_on ? a.k : 0;
  const int y = a.labels[row];
  int col[kEntries];   // this thread's entries of the record
  float lq[kEntries], zt[kEntries];
#pragma unroll
  for (int e = 0; e < kEntries; ++e) {
    const int j = tid + e * kThreads;
    col[e] = j < k ? a.idx[row * a.k + j] : -1;
    lq[e] = j < k ? a.val[row * a.k + j] : 0.f;
  }
  if (!(y >= 0 && y < a.V)) {   // outside Omega
    const Span<T> so(dz, a.ld);
    const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
#pragma unroll 1
    for (int i = rank * kThreads + tid; i < so.words; i += split * kThreads) *reinterpret_cast<uint4*>(dz + so.word_at(i)) = zero;
    if (rank == 0 && tid < so.singles(a.ld)) dz[so.single_at(tid)] = from_f<T>(0.f);
    if (rank == 0 && tid == 0) a.row_loss[row] = 0.f;
    return;
  }
  const Span<T> sp(z, a.V);
  const Slice sl(reinterpret_cast<const uint4*>(z + sp.head), sp.words, rank, split);
  sl.prefetch();
  if (split > 1) cluster_arrive();
  const int lo = sp.word_at(sl.first), hi = lo + sl.n * W;   // the slice's columns; the first CTA has the values outside the words too
  const int ns = rank == 0 ? sp.singles(a.V) : 0;
  auto place_of_single = [&](int c) { return c < sp.head ? c : c - sp.tail + sp.head; };
  auto here = [&](int c) { return (c >= lo && c < hi) || (rank == 0 && (c < sp.head || c >= sp.tail)); };
  auto marked = [&](int c) {
    return c >= lo && c < hi ? (bits[(c - lo) >> 5] >> ((c - lo) & 31) & 1u) != 0u : (sh.singles >> place_of_single(c) & 1u) != 0u;
  };
#pragma unroll 1
  for (int i = tid; i < (sl.n * W + 31) / 32; i += kThreads) bits[i] = 0u;
  if (tid == 0) sh.singles = 0u;
  int cnt = 0;   // (count_here: N is at most kCountHere, two labels a thread)
#pragma unroll 1
  for (int i = tid; a.count_here && i < a.N; i += kThreads) {
    const int l = a.labels[i];
    cnt += l >= 0 && l < a.V;
  }
  const float T1 = kl_on ? a.T : 1.f, inv_T = 1.f / T1, s = kL2e / T1;
  const bool has_rest = kl_on && a.rest != nullptr;
  const float rest = has_rest ? a.rest[row] : -INFINITY;
  const float zy = to_f(z[y]);
  const float single = tid < ns ? to_f(z[sp.single_at(tid)]) : 0.f;
  __syncthreads();
  bool twice = false;
#pragma unroll
  for (int e = 0; e < kEntries; ++e) {
    const int c = col[e] = col[e] >= 0 && col[e] < a.V ? col[e] : -1;
    lq[e] *= inv_T;
    zt[e] = c >= 0 ? to_f(z[c]) : 0.f;
    if (c >= 0 && here(c)) {
      uint32_t* const w = c >= lo && c < hi ? &bits[(c - lo) >> 5] : &sh.singles;
      const uint32_t b = c >= lo && c < hi ? 1u << ((c - lo) & 31) : 1u << place_of_single(c);
      twice |= (atomicOr(w, b) & b) != 0u;
    }
  }
  if (a.count_here) {
    const int n = __popc(__ballot_sync(0xffffffffu, cnt & 1)) + 2 * __popc(__ballot_sync(0xffffffffu, cnt & 2));
    if (lane == 0) sh.n[warp] = n;
  }
  twice = __syncthreads_or(twice);
  // pass 1: the columns outside the record
  vocab::LseRun Pr = vocab::run_empty(s), Cr = vocab::run_empty(kL2e);   // e^{z / T} (alpha 1: e^z); TWO: e^z
  sl.pass([&](const uint4& v, int i, int) {
    const uint32_t m = bits[i * W >> 5] >> (i * W & 31) & ((1u << W) - 1u);
    uint4 u = v;
    if (m != 0u) mask_word<T>(u, m);
    float x[W];
    word_floats(u, x);
    const float mx = word_max<T>(u);
    vocab::run_add(Pr, x, mx, s);
    if (TWO) vocab::run_add(Cr, x, mx, kL2e);
  });
  Lse P = vocab::run_sum(Pr), C = vocab::run_sum(Cr);
  if (tid < ns && !marked(sp.single_at(tid))) {
    vocab::lse_add1(P, single, s);
    if (TWO) vocab::lse_add1(C, single, kL2e);
  }
  P = vocab::warp_merge(P, s);
  if (TWO) C = vocab::warp_merge(C, kL2e);
  if (lane == 0) {
    sh.p[warp] = P;
    sh.c[warp] = C;
  }
  // one warp joins the block's sums
  auto joined = [&](const Lse* from, int n, float scale) {
    return vocab::warp_merge(lane < n ? from[lane] : vocab::lse_empty(), scale);
  };
  if (split > 1) {
    __syncthreads();
    cluster_wait();
    if (warp == 0) {
      P = joined(sh.p, kWarps, s);
      if (TWO) C = joined(sh.c, kWarps, kL2e);
      if (lane < split) {
        LossShared* const p = peer(&sh, lane);
        p->others[rank] = P;
        p->all[rank] = C;
        p->twice[rank] = twice;
      }
    }
    tc::cluster_sync();   // (every CTA has read the record's logits and its slice as well: dz may be z)
#pragma unroll 1
    for (int r = 0; r < split; ++r) twice |= sh.twice[r] != 0;
  }
  if (twice) {   // a column more than once: its first entry counts
#pragma unroll
    for (int e = 0; e < kEntries; ++e) {
      const int j = tid + e * kThreads;
      bool again = false;
#pragma unroll 1
      for (int i = 0; i < j && j < k; ++i) again |= a.idx[row * a.k + i] == col[e];
      if (again) col[e] = -1;
    }
  }
  // the record's own columns and the teacher's, by the warps that have entries
  const int kw = min(kWarps, (k + 31) / 32);
  if (warp < kw) {
    Lse R = vocab::lse_empty(), Q = vocab::lse_empty(), C1 = vocab::lse_empty();
#pragma unroll
    for (int e = 0; e < kEntries; ++e) {
      if (col[e] < 0) continue;
      vocab::lse_add1(R, zt[e], s);
      if (TWO) vocab::lse_add1(C1, zt[e], kL2e);
      vocab::lse_add1(Q, lq[e], kL2e);
    }
    if (has_rest && tid == 0) vocab::lse_add1(Q, rest, kL2e);
    R = vocab::warp_merge(R, s);
    Q = vocab::warp_merge(Q, kL2e);
    if (TWO) C1 = vocab::warp_merge(C1, kL2e);
    if (lane == 0) {
      sh.r[warp] = R;
      sh.q[warp] = Q;
      if (TWO && split == 1) sh.c[warp] = vocab::lse_merge(sh.c[warp], C1, kL2e);
      if (TWO && split > 1) sh.c[warp] = C1;
    }
  }
  __syncthreads();
  if (warp == 0) {
    P = split > 1 ? joined(sh.others, split, s) : joined(sh.p, kWarps, s);
    const Lse R = joined(sh.r, kw, s), Q = joined(sh.q, kw, kL2e);
    if (TWO) C = split > 1 ? vocab::lse_merge(joined(sh.all, split, kL2e), joined(sh.c, kw, kL2e), kL2e) : joined(sh.c, kWarps, kL2e);
    int n = a.count_here && lane < kWarps ? sh.n[lane] : 0;
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) {
      RowTerms t;
      t.omega = a.count_here ? (float)n : a.loss[1];
      const Lse A = vocab::lse_merge(P, R, s);
      t.al = log2f(A.s) * kLn2;
      t.ql = log2f(Q.s) * kLn2;
      t.lpr = (P.m - A.m) * inv_T + (log2f(P.s) * kLn2 - t.al);
      t.lqr = (rest - Q.m) - t.ql;
      t.held = !(Q.m == -INFINITY && Q.s == 0.f);
      t.bad = A.m == -INFINITY ? __uint_as_float(0x7FC00000u) : (A.s + Q.s) * 0.f;
      // no others, or only masks beside the record's logits: e_v 0 (a row of nothing but masks has their softmax)
      const bool none = P.m == -INFINITY || (P.m <= -kMasked && A.m > -kMasked);
      t.om = none ? 0.f : P.m;
      t.oi = none ? 0.f : 1.f / P.s;
      t.pr = none ? 0.f : P.s * ex2((P.m - A.m) * s) / A.s;
      t.am = A.m;
      t.ai = 1.f / A.s;
      t.cm = TWO ? C.m : A.m;
      t.ci = TWO ? 1.f / C.s : t.ai;
      t.cl = TWO ? log2f(C.s) * kLn2 : t.al;
      t.qm = Q.m;
      t.qi = 1.f / Q.s;
      sh.t = t;
    }
  }
  __syncthreads();
  const RowTerms& t = sh.t;
  const bool mass = kl_on && t.held;
  auto p_of = [&](float x) { return ex2((x - t.am) * s) * t.ai; };
  auto q_of = [&](float x) { return ex2((x - t.qm) * kL2e) * t.qi; };
  auto logp = [&](float x) { return (x - t.am) * inv_T - t.al; };
  auto logq = [&](float x) { return (x - t.qm) - t.ql; };
  // the divergence
  auto xlog = [](float p, float d) { return p == 0.f ? 0.f : p * d; };   // (a p of NaN stays)
  float kl = 0.f;
  if (mass) {
    if (warp < kw) {
#pragma unroll
      for (int e = 0; e < kEntries; ++e) {
        if (col[e] < 0) continue;
        const float lp = logp(zt[e]), q = logq(lq[e]);
        kl += a.dir == 1 ? xlog(q_of(lq[e]), q - lp) : xlog(p_of(zt[e]), lp - q);
      }
      if (has_rest && tid == 0) kl += a.dir == 1 ? xlog(q_of(rest), t.lqr - t.lpr) : xlog(t.pr, t.lpr - t.lqr);
      kl = warp_sum(kl);
      if (lane == 0) sh.kl[warp] = kl;
    }
    __syncthreads();
    kl = 0.f;
#pragma unroll 1
    for (int w = 0; w < kw; ++w) kl += sh.kl[w];
  }
  // Pass 2, of a column v outside the record: with e_v = e^{x_v - others} (its share of the others' mass) p_v = p_r e_v, and
  // T dKL/dz_v = e_v (p_r - q_r) (dir 1) or e_v p_r (lp_r - lq_r - KL) (dir 0): no quotient of probabilities near 0.
  // dz_v = wa p1_v + wk other e_v; without a second softmax p1_v = p_r e_v.
  const float w = 1.f / t.omega, wa = w * a.alpha, wk = (mass ? w * (1.f - a.alpha) * a.T : 0.f) + t.bad;
  float other = t.pr;
  if (has_rest) other = a.dir == 1 ? t.pr - q_of(rest) : xlog(t.pr, t.lpr - t.lqr - kl);
  const float ck = (wk == 0.f ? 0.f : wk * other) * t.oi, cs = fmaf(wa, t.pr * t.oi, ck), c1 = wa * t.ci;
  if (rank == 0 && tid == 0)
    a.row_loss[row] = (a.alpha > 0.f ? a.alpha * ((t.cm - zy) + t.cl) : 0.f) + (kl_on ? (1.f - a.alpha) * a.T * (a.T * kl) : 0.f) + t.bad;
  const uint64_t s2 = f2(s, s), cs2 = f2(TWO ? ck : cs, TWO ? ck : cs), c12 = f2(c1, c1), L2 = f2(kL2e, kL2e);
  const uint64_t om2 = f2(-t.om, -t.om), cm2 = f2(-t.cm, -t.cm);
  auto grad = [&](float x) {
    if (TWO) return fmaf(c1, ex2((x - t.cm) * kL2e), ck * ex2((x - t.om) * s));
    return cs * ex2((x - t.om) * s);
  };
  const bool same = ((uintptr_t)z & 15u) == ((uintptr_t)dz & 15u);
  uint4* const dw = reinterpret_cast<uint4*>(dz + lo);
  sl.pass([&](const uint4& u, int i, int) {
    float x[W];
    word_floats(u, x);
#pragma unroll
    for (int e = 0; e < W; e += 2) {
      const float2 v = uf2(mul2(add2(f2(x[e], x[e + 1]), om2), s2));
      uint64_t g = mul2(cs2, f2(ex2(v.x), ex2(v.y)));
      if (TWO) {
        const float2 v1 = uf2(mul2(add2(f2(x[e], x[e + 1]), cm2), L2));
        g = fma2(c12, f2(ex2(v1.x), ex2(v1.y)), g);
      }
      const float2 o = uf2(g);
      x[e] = o.x;
      x[e + 1] = o.y;
    }
    if (same) {
      __stcs(dw + i, vocab::pack_word(x));
    } else {
#pragma unroll
      for (int e = 0; e < W; ++e) dz[lo + i * W + e] = from_f<T>(x[e]);
    }
  });
  if (tid < ns) dz[sp.single_at(tid)] = from_f<T>(grad(single));
  if (rank == 0)
    for (int c = a.V + tid; c < a.ld; c += kThreads) dz[c] = from_f<T>(0.f);
  __syncthreads();
  // the record's columns and the label's
  if (warp < kw) {
#pragma unroll
    for (int e = 0; e < kEntries; ++e) {
      if (col[e] < 0 || !here(col[e])) continue;
      const float lp = logp(zt[e]), q = logq(lq[e]), p = p_of(zt[e]);
      float g = 0.f;
      if (mass) g = a.dir == 1 ? p - q_of(lq[e]) : xlog(p, lp - q - kl);
      const float v = (wa != 0.f ? wa * ((TWO ? ex2((zt[e] - t.cm) * kL2e) * t.ci : p) - (col[e] == y ? 1.f : 0.f)) : 0.f) + wk * g;
      dz[col[e]] = from_f<T>(v);
    }
  }
  if (tid == 0 && wa != 0.f && here(y) && !(k > 0 && marked(y))) dz[y] = from_f<T>(grad(zy) - wa);
}

// loss[0] = sum(row_loss) / |Omega|, loss[1] = |Omega|, in a fixed order; `part` 1 forms loss[1] alone (before the rows), 2
// loss[0] from it.
__global__ void __launch_bounds__(1024) top_finish_k(const float* __restrict__ row_loss, const int32_t* __restrict__ labels,
                                                     int N, int V, float* loss, int part) {
  pdl_wait();
  pdl_trigger();
  vocab::finish_loss(row_loss, labels, N, V, loss, part);
}

// CTAs that share a row: one, but for rows so long that those being worked on would not stay in L2 between their passes (140 KB
// a CTA, four an SM: 85 MB), and for few rows as many as fill the SMs with slices of 8 KB or more.
int split_of(int N, int V, size_t es) {
  const size_t bytes = (size_t)V * es;
  int s = 1;
  while (s < kMaxSplit && bytes / s > 140 * 1024) s *= 2;
  while (s < kMaxSplit && (size_t)N * s <= 152 && bytes / (2 * s) >= 8192) s *= 2;
  return s;
}

// How many rows further down the one lies that takes a row's place on the SMs. It is brought to L2 once the row at hand is no longer
// read (sooner, both would have to stay there), while what remains to be done waits for itself: 116 -> 106 us at 4096 x 50257. (The
// loss, whose gradient fills L2 as well, takes 174 us with it and 161 without; its gradient passes L2 by.)
int rows_ahead(int split) { return std::max(1, kBlocks * 152 / split); }

template <typename... KArgs, typename... Args>
bool launch_split(void (*kern)(KArgs...), int N, int split, int dyn, cudaStream_t s, Args&&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)N * (unsigned)split);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = (size_t)dyn;
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = (unsigned)split;
  at[1].val.clusterDim.y = 1;
  at[1].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = split > 1 ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, std::forward<Args>(args)...) == cudaSuccess;
}
// Lets a kernel have all the shared memory there is, once a device.
template <typename K>
bool allow(K* kern, PerDevice<bool>& devices) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  return devices.get(dev, [&](bool&) {
           cudaFuncAttributes fa;
           if (cudaFuncGetAttributes(&fa, kern) != cudaSuccess) return false;
           return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 232448 - (int)fa.sharedSizeBytes) == cudaSuccess;
         }) != nullptr;
}

bool shape_ok(int dtype, int N, int V, int ld, int k, float T) {
  return (dtype == ZL_DTYPE_F32 || dtype == ZL_DTYPE_BF16) && N >= 0 && N <= ZL_VOCAB_MAX_ROWS && V >= 2 && V <= ZL_VOCAB_MAX &&
         ld >= V && k >= 1 && k <= V && k <= ZL_TOP_MAX && T > 0.f && std::isfinite(T) && std::isfinite(kL2e / T);
}
const char* const kShapeMsg =
    "bad dtype or size (0 <= N <= 2^24, 2 <= V <= 2^20, ld >= V, 1 <= k <= min(V, 1024)), or a temperature that is not positive "
    "and finite, or so low that log2(e) / T is not";
const char* const kPtrMsg = "NULL pointer, or a tensor off the alignment of its elements";

template <typename T>
bool launch_top(const void* z, int N, TopArgs a, cudaStream_t s) {
  static PerDevice<bool> devices;
  auto kern = top_logits_k<T>;
  if (!allow(kern, devices)) return false;
  int all = std::max(64, 16 * a.split);
  while (all < 2 * a.k) all *= 2;
  a.bins = all / a.split;
  a.ahead = rows_ahead(a.split);
  a.cap = 512;   // a power of two (see sort_falling), twice the record or more
  while (a.cap < 2 * a.k) a.cap *= 2;
  return launch_split(kern, N, a.split, top_dyn(a.split, a.bins, a.cap), s, (const T*)z, a);
}

template <typename T, bool TWO>
bool launch_loss(const void* z, void* dz, const LossArgs& a, cudaStream_t s) {
  static PerDevice<bool> devices;
  auto kern = top_loss_k<T, TWO>;
  if (!allow(kern, devices)) return false;
  return launch_split(kern, a.N, a.split, mark_bytes(a.V, Span<T>::W, a.split), s, (const T*)z, (T*)dz, a);
}

}  // namespace top
}  // namespace zl

using namespace zl;
using zl::act8::entry;
using zl::act8::fail;
using zl::act8::launched;
using zl::act8::on_elements;

extern "C" {

zl_status zl_op_top_logits(int dtype, const void* z, int N, int V, int ld, int k, float T, int32_t* idx, float* val, float* rest,
                           void* stream) {
  return entry([&]() -> zl_status {
    if (!top::shape_ok(dtype, N, V, ld, k, T)) return fail(ZL_ERR_ARG, top::kShapeMsg);
    if (N == 0) return ZL_OK;
    if (!z || !idx || !val || !rest || !on_elements({z}, dt_size(dtype)) || !on_elements({idx, val, rest}, 4))
      return fail(ZL_ERR_ARG, top::kPtrMsg);
    const top::TopArgs a{N, V, ld, k, top::split_of(N, V, dt_size(dtype)), 0, 0, 0, vocab::kL2e / T, T, idx, val, rest};
    cudaStream_t s = (cudaStream_t)stream;
    note_launch(1);
    const bool ok = dtype == ZL_DTYPE_BF16 ? top::launch_top<bf16>(z, N, a, s) : top::launch_top<float>(z, N, a, s);
    const zl_status st = launched("zl_op_top_logits");
    return st != ZL_OK || ok ? st : fail(ZL_ERR_CUDA, "zl_op_top_logits: the kernel could not be launched on this device");
  });
}

zl_status zl_op_top_loss(int dtype, const void* z, const int32_t* idx, const float* val, const float* rest, const int32_t* labels,
                         int N, int V, int ld, int k, float alpha, float T, int kl_dir, void* dz, float* row_loss, float* loss,
                         void* stream) {
  return entry([&]() -> zl_status {
    if (!top::shape_ok(dtype, N, V, ld, k, T)) return fail(ZL_ERR_ARG, top::kShapeMsg);
    if (!(alpha >= 0.f && alpha <= 1.f) || (kl_dir != 0 && kl_dir != 1) || (N > 0 && alpha < 1.f && kl_dir == 0 && !rest))
      return fail(ZL_ERR_ARG, "alpha in [0, 1], kl_dir 0 or 1, kl_dir 0 needs rest (else it is infinite)");
    cudaStream_t s = (cudaStream_t)stream;
    if (N == 0) {
      if (!loss || !on_elements({loss}, 4)) return fail(ZL_ERR_ARG, top::kPtrMsg);
      cudaMemsetAsync(loss, 0, 8, s);
      return launched("zl_op_top_loss");
    }
    if (!z || !labels || !dz || !row_loss || !loss || (alpha < 1.f && (!idx || !val)) || !on_elements({z, dz}, dt_size(dtype)) ||
        !on_elements({idx, val, rest, labels, row_loss, loss}, 4))
      return fail(ZL_ERR_ARG, top::kPtrMsg);
    const int here = N <= top::kCountHere;
    const int split = top::split_of(N, V, dt_size(dtype));
    const top::LossArgs a{idx, val, rest, labels, N, V, ld, k, kl_dir, here, split, alpha, T, row_loss, loss};
    const bool two = T != 1.f && alpha > 0.f && alpha < 1.f;
    note_launch(here ? 2 : 3);
    if (!here) launch_pdl(top::top_finish_k, 1, 1024, 0, s, (const float*)row_loss, labels, N, V, loss, 1);
    const bool ok = dtype == ZL_DTYPE_BF16 ? (two ? top::launch_loss<bf16, true>(z, dz, a, s) : top::launch_loss<bf16, false>(z, dz, a, s))
                                           : (two ? top::launch_loss<float, true>(z, dz, a, s) : top::launch_loss<float, false>(z, dz, a, s));
    if (ok) launch_pdl(top::top_finish_k, 1, N <= 1024 ? 256 : 1024, 0, s, (const float*)row_loss, labels, N, V, loss, here ? 3 : 2);
    const zl_status st = launched("zl_op_top_loss");
    return st != ZL_OK || ok ? st : fail(ZL_ERR_CUDA, "zl_op_top_loss: the kernel could not be launched on this device");
  });
}

}  // extern "C"
