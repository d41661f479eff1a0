// The products of a Newton-Schulz iteration, as muon_gemm.cu runs them.  Not part of the public ABI.
#pragma once

#include <cuda.h>
#include <cuda_fp16.h>

#include "internal.h"

namespace ffsp {
namespace muon {

// X, S = X X^T and P = a I + b S + c S^2 are held as fp16 times 256, which keeps values from 2.4e-7 to 200 normal: singular
// values of X stay below 1.5, so its elements do, S's below 2.3, and P is checked to stay below 200.  A second plane holds
// what the first one rounds off, times 2048: 22 bits together.
constexpr float HELD = 256.f, LOW = 2048.f;

// `count` matrices [rows, cols] with pitch ld (a multiple of 64), one after the other.  The second plane: the same, count * each
// elements on, where the tensor cores take it too (precise); else only epilogues read and write it, a lane to a row, and it lies
// in blocks of 32 rows x 16 columns, which is what a warp handles at once: 8 columns of 32 rows, then the other 8.
struct Matrices {
  __half *p, *low;
  int rows, cols, ld, count;
  long long each, low_each;
};
inline long long block_rows(int rows) { return (rows + 31) / 32 * 32; }

// What the last product's epilogue needs of a matrix; lies in the workspace.
struct Target {
  const void* W;
  void* out;
  float keep, step;       // out = keep W - step X; without W: out = -step X
  int f32, even;          // even: rows of W and out start on 4 bytes
};

// C = alpha A B + beta D + diagonal I for every matrix of a group.
struct Product {
  Matrices a, b, c;       // a: [M, K], or [K, M] with a_mn; b: [N, K], or [K, N] with b_mn
  int a_mn, b_mn;
  int M, N, K;
  float alpha, beta, diagonal;
  const Matrices* d;      // nullptr: no second term
  int d_high, d_low;      // which of its planes (both: precise; the second alone: in blocks)
  int symmetric;          // C = C^T: tiles above the diagonal only, and mirrored
  int c_low;              // the second plane of C is written
  const Target* target;   // the last product: the matrices are updated, nothing is written to c
};

constexpr int MAX_GROUPS = 4;
// precise: operands count with both planes (three products of planes), sums leave the tensor cores every few k-blocks.
ffsplit_status launch_products(ffsplit_ctx* ctx, bool precise, const Product* products, int n, cudaStream_t st);

// P = a I + b S + c S S with S = X X^T (X^T X) in one launch, for matrices with p <= SQUARE_MOST: a pair of CTAs to a matrix.
constexpr int SQUARE_MOST = 256;
struct Gram {
  Matrices X, P;
  int mn, K;              // mn: S = X^T X
  float a, b, c;
};
ffsplit_status launch_squares(ffsplit_ctx* ctx, const Gram* squares, int n, cudaStream_t st);

#ifdef __CUDACC__
// Where 8 columns (octet of them) of one row lie in a second plane of blocks.
__device__ __forceinline__ long long block_at(int row, int octet, int ld) {
  return (static_cast<long long>(row >> 5) * (ld >> 4) + (octet >> 1)) * 512 + (octet & 1) * 256 + (row & 31) * 8;
}
// One value's two planes.
__device__ __forceinline__ void split_half(float x, __half* hi, __half* lo) {
  *hi = __float2half_rn(x);
  *lo = __float2half_rn((x - __half2float(*hi)) * LOW);
}
#endif

}  // namespace muon
}  // namespace ffsp
