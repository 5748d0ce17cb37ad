// The products of the losses over a large vocabulary (host side; vocab_gemm.cu).
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace zl {
namespace vocab {

// An fp32 matrix takes part as three bf16 terms, x = h + m + l, each the leading 8 bits of what is left: exact, and every value by
// itself. (Fixed-point digits under a scale for each row add up without an error in the tensor cores, and the same products took 10%
// less time; but a row with a column 300 times the others holds those in 16 bits, and a gradient times a small row's scale falls below
// the smallest bf16.) Of the nine products of two such matrices the six largest are formed, smallest first. What is left out, m l
// twice and l l, is below 2^-21 of |a| |b| (|m| < 2^-7 |x|, |l| < 2^-15 |x|), with the product's sign.
constexpr int kTerms = 3, kPairs = 6;

// C [M, N] = A B^T (b_mn 0: B [N, K]) or A B (b_mn 1: B [K, N]), A [M, K] or with a_mn its transpose [K, M]; fp32 sums in
// TMEM. terms 1 or 3: term t of an operand starts t * a_term (b_term) rows further down, its rows lda (ldb) values apart.
struct Operands {
  const void *A, *B;
  int a_mn, b_mn;
  int a_rows, b_rows;          // rows that exist in memory, over all terms (rows past them read as zeros)
  int lda, ldb;                // multiples of 8
  int a_term, b_term, terms;
  int b_first;                 // first row of B (its columns in the product where b_mn is 0)
  int direct;                  // B is fp32 as it is, its terms are formed in the product; bn is 128
};

// How a product is cut: tiles of 128 (pair: 256) x bn, `splits` cuts of K, each of several accumulations in TMEM of at most
// kb_per_seg blocks of 64 (the largest pair of terms; the others share one), summed in fp32 registers.
struct Tiles {
  int bn, pair, splits, kb_per_split, kb_per_seg;
  double us;   // predicted
};
enum Kind { kLse, kGradZ, kOut16, kOut32 };
// out_step: what bn is a multiple of. seg: k blocks of one accumulation. max_splits 1: none. runs: products into the same slices.
Tiles plan(Kind kind, int M, int N, int K, int terms, int out_step, int seg, int max_splits, int runs = 1);

// The same for direct products.
Tiles plan_direct(int M, int N, int K, int seg, int max_splits, int runs = 1);

// (m, s) of every row of z = A B^T over each half tile: part [M][2 * tiles_n]; zl [M]: z at the row's label; *counter = 0.
bool gemm_lse(int M, int V, int K, const Operands& o, const Tiles& t, const int32_t* labels, float2* part, float* zl,
              unsigned* counter, cudaStream_t s);
inline int lse_parts(int V, const Tiles& t) { return 2 * ((V + t.bn - 1) / t.bn); }
// dz = e^{z - lse} - [label] in the rows of Omega, 0 else, for the columns first .. first + n of a vocabulary of V (0 past it): bf16
// terms [o.terms][rows_p][ldz], rows M .. rows_p zeros. Without the rows' common weight, whose rounding would be in every value:
// where p is small, dz is exactly -1 at the label.
bool gemm_grad_z(int M, int n, int K, const Operands& o, const Tiles& t, const int32_t* labels, const float* lse, int first, int V,
                 void* dz, int rows_p, int ldz, cudaStream_t s);
// C = A B: bf16 C [M, N] (a_mn), or fp32 slices [splits][M, N], one for each split, overwritten or (add) added to.
// C times loss_weight(omega, dloss) (omega NULL: 1).
bool gemm_out(int M, int N, int K, const Operands& o, const Tiles& t, int out_f32, void* C, int add, const float* omega,
              const float* dloss, cudaStream_t s);

}  // namespace vocab
}  // namespace zl
