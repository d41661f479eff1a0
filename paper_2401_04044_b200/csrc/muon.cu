// The update of a list of matrices by orthogonalised momentum.
//
//   M' = beta M + G,  U = G + beta M' or M',  X = U / (|U| + 1e-7)
//   X <- a X + (b S + c S^2) X, S = X X^T   (rows <= cols; else X (b S + c S^2), S = X^T X),  once per (a, b, c)
//   W' = (1 - decay) W - step X
//
// Two passes over the gradients (the norm, then X and M'; both read G and M), then three products per iteration on the tensor
// cores (muon_gemm.cu), the last of which updates the matrices.  Matrices of one shape are one launch, up to four shapes
// share it.
#include <cmath>
#include <cstring>

#include "epilogue.cuh"
#include "muon.h"
#include "ptx.cuh"

namespace ffsp {
namespace muon {

constexpr int MAX_TENSORS = 128;        // of one launch's table
constexpr int THREADS = 256;
constexpr int MAX_PARTS = 1024;         // partial sums of one matrix's squares (256 of them read 90 MB at 1.2 TB/s: too few blocks)

struct Entry {
  const void* G;
  const float* M;
  float* Mo;
  const void* W;
  void* out;
  __half *X, *X_low;      // [rows][ld], and the second plane: likewise, or in blocks
  int blocks;
  int rows, cols, octets; // octets of columns in a row
  int g_f32, w_f32;
  int wide, wide_w;       // every octet of G, M, Mo (of W, out) starts on 16 bytes
  int ld;
  int parts;
  int place;              // in the caller's list
  float step, decay;
};
// (The argument block is copied with every launch and read through the constant cache: a short list gets a short one.)
template <int CAP>
struct Table {
  Entry t[CAP];
  int n;
  float beta;
  int nesterov;
  double* partial;        // [n][MAX_PARTS]
  Target* target;         // [n]
  int* status;
};

// Eight columns of M' and U.
__device__ __forceinline__ void load_u8(const Entry& e, float beta, int nesterov, int row, int octet, float* m, float* u) {
  const int c = octet * 8;
  const long long at = static_cast<long long>(row) * e.cols + c;
  float g[8];
  if (e.wide) {
    if (e.g_f32) {
      const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(e.G) + at);
      const float4 x = __ldg(p), y = __ldg(p + 1);
      g[0] = x.x; g[1] = x.y; g[2] = x.z; g[3] = x.w; g[4] = y.x; g[5] = y.y; g[6] = y.z; g[7] = y.w;
    } else {
      const uint4 q = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(e.G) + at));
      const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        g[2 * i] = __uint_as_float(w[i] << 16);
        g[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    }
    if (e.M) {
      const float4* p = reinterpret_cast<const float4*>(e.M + at);
      const float4 x = p[0], y = p[1];
      m[0] = x.x; m[1] = x.y; m[2] = x.z; m[3] = x.w; m[4] = y.x; m[5] = y.y; m[6] = y.z; m[7] = y.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const bool in = c + i < e.cols;
      g[i] = !in ? 0.f : e.g_f32 ? static_cast<const float*>(e.G)[at + i] : __bfloat162float(static_cast<const __nv_bfloat16*>(e.G)[at + i]);
      m[i] = in && e.M ? e.M[at + i] : 0.f;
    }
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (e.M) {
      m[i] = fmaf(beta, m[i], g[i]);
      u[i] = nesterov ? fmaf(beta, m[i], g[i]) : m[i];
    } else {
      u[i] = g[i];
    }
  }
}
// A matrix is gone through in pieces of 16 rows x 128 columns, eight columns to a thread: a warp reads 256 bytes of each of two
// rows of G, and what it leaves in a second plane of blocks is whole sectors.  Pieces begin .. end of block `part`.
constexpr int PIECE_ROWS = 16, PIECE_OCTETS = 16;
__host__ __device__ __forceinline__ int pieces_across(int octets) { return (octets + PIECE_OCTETS - 1) / PIECE_OCTETS; }
__device__ __forceinline__ void range_of(const Entry& e, int part, int* begin, int* end) {
  const int all = (e.rows + PIECE_ROWS - 1) / PIECE_ROWS * pieces_across(e.octets), per = (all + e.parts - 1) / e.parts;
  *begin = part * per;
  *end = *begin + per < all ? *begin + per : all;
}
// This thread's columns of a piece; false: there are none.
__device__ __forceinline__ bool place(const Entry& e, int piece, int* row, int* octet) {
  const int across = pieces_across(e.octets), r = piece / across;
  *row = r * PIECE_ROWS + (threadIdx.x >> 4);
  *octet = (piece - r * across) * PIECE_OCTETS + (threadIdx.x & 15);
  return *row < e.rows && *octet < e.octets;
}
__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_down_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  double t = 0.0;
  for (int i = 0; i < THREADS / 32; ++i) t += red[i];
  return t;
}

// A row of blocks to a matrix; those behind its parts have nothing to do.
template <int CAP>
__global__ void __launch_bounds__(THREADS) norm_kernel(const __grid_constant__ Table<CAP> t) {
  __shared__ double red[THREADS / 32];
  pdl_wait();
  const int which = blockIdx.y, part = blockIdx.x;
  const Entry& e = t.t[which];
  if (part >= e.parts) return;
  int begin, end;
  range_of(e, part, &begin, &end);
  double acc = 0.0;
#pragma unroll 2
  for (int i = begin; i < end; ++i) {
    int row, octet;
    if (!place(e, i, &row, &octet)) continue;
    float m[8], u[8];
    load_u8(e, t.beta, t.nesterov, row, octet, m, u);
#pragma unroll
    for (int k = 0; k < 8; ++k) acc += static_cast<double>(u[k]) * static_cast<double>(u[k]);
  }
  const double s = block_sum(acc, red);
  if (threadIdx.x == 0) t.partial[which * MAX_PARTS + part] = s;
}

// X = U / (norm + 1e-7), M', and what the last product does with the matrix.
template <int CAP>
__global__ void __launch_bounds__(THREADS) prepare_kernel(const __grid_constant__ Table<CAP> t) {
  __shared__ double red[THREADS / 32];
  pdl_wait();
  const int which = blockIdx.y, part = blockIdx.x;
  const Entry& e = t.t[which];
  if (part >= e.parts) return;
  double mine = 0.0;
#pragma unroll
  for (int k = 0; k < MAX_PARTS / THREADS; ++k)
    if (k * THREADS + static_cast<int>(threadIdx.x) < e.parts) mine += __ldcg(t.partial + which * MAX_PARTS + k * THREADS + threadIdx.x);
  const double squares = block_sum(mine, red);
  const float norm = static_cast<float>(sqrt(squares));
  const bool finite = isfinite(norm);
  const float inv = finite ? HELD / (norm + 1e-7f) : 0.f;      // (with the factor X is held with: 1 / norm may be below the normal numbers)
  if (part == 0 && threadIdx.x == 0) {
    Target o;
    o.W = e.W; o.out = e.out; o.f32 = e.w_f32;
    o.even = e.cols % 2 == 0 && ((reinterpret_cast<uintptr_t>(e.W) | reinterpret_cast<uintptr_t>(e.out)) & 3u) == 0;
    o.keep = finite ? 1.0f - e.decay : 1.0f;
    o.step = e.W ? (finite ? e.step : 0.f) : finite ? -1.0f : __int_as_float(0x7fffffff);
    t.target[which] = o;
    if (!finite) record_status(t.status, FFSPLIT_ERR_NONFINITE, e.place, KID_MUON);
  }
  int begin, end;
  range_of(e, part, &begin, &end);
#pragma unroll 2
  for (int i = begin; i < end; ++i) {
    int row, octet;
    if (!place(e, i, &row, &octet)) continue;
    float m[8], u[8];
    load_u8(e, t.beta, t.nesterov, row, octet, m, u);
    const int c = octet * 8;
    const long long at = static_cast<long long>(row) * e.cols + c;
    if (e.M) {
      if (!finite) {
#pragma unroll
        for (int k = 0; k < 8; ++k) if (e.Mo != e.M && c + k < e.cols) e.Mo[at + k] = e.M[at + k];
      } else if (e.wide) {
        float4* p = reinterpret_cast<float4*>(e.Mo + at);
        p[0] = make_float4(m[0], m[1], m[2], m[3]);
        p[1] = make_float4(m[4], m[5], m[6], m[7]);
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) if (c + k < e.cols) e.Mo[at + k] = m[k];
      }
    }
    __align__(16) __half hi[8], lo[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) split_half(finite ? u[k] * inv : 0.f, &hi[k], &lo[k]);
    __half* x = e.X + static_cast<long long>(row) * e.ld + c;
    *reinterpret_cast<uint4*>(x) = *reinterpret_cast<const uint4*>(hi);
    __half* x_low = e.X_low + (e.blocks ? block_at(row, octet, e.ld) : static_cast<long long>(row) * e.ld + c);
    *reinterpret_cast<uint4*>(x_low) = *reinterpret_cast<const uint4*>(lo);
  }
}

// ------------------------------------------------------------------------------------------------ thin matrices
// p = min(rows, cols) <= 64 (an adapter's factors): the tensor cores' tiles would be nearly empty, and 15 launches are what
// the work is not.  X stays in the row space of U, so X_n = Q U with Q a polynomial in S = U U^T: one pass over U for S, the
// iteration on p x p matrices (S <- A S A, Q <- A Q, A = a I + b S + c S S), one pass for Q U.  S has the squares of U's
// singular values and Q their inverses: all of that is held in fp64, so that nothing is lost over the direct form.
// The products are fp64 matrix instructions of 8 x 8 x 4 (with scalar ones the loads from shared memory were the bound: 100 us
// for 32 factors of rank 16).
constexpr int THIN = 64, THIN_PARTS = 64;
constexpr int SQUARE_PITCH = THIN + 4;      // doubles: the 4 rows x 4 columns of half a fragment fall into 32 banks
constexpr int WARPS = THREADS / 32;
// p in tiles of 8, 1, 2, 4 or 8 of them; a block takes so many of U's columns at a time that every thread has two octets.
__host__ __device__ __forceinline__ int thin_tiles(int p) { return p <= 8 ? 1 : p <= 16 ? 2 : p <= 32 ? 4 : 8; }
__host__ __device__ __forceinline__ int thin_chunk(int tiles) { return 512 / tiles; }
constexpr size_t THIN_U_BYTES = (8 * 512 + 8 * 4 * 8) * sizeof(double);      // the most that 8 tiles (chunk + 4) takes
inline size_t square_bytes(int tiles) { return static_cast<size_t>(tiles) * 8 * SQUARE_PITCH * sizeof(double); }
template <int CAP>
struct ThinTable {
  Entry t[CAP];
  double* S[CAP];      // [parts][p][p]
  double* Q[CAP];      // [p][p], for U itself (not divided by its norm)
  int n;
  int tiles;           // thin_tiles() of the largest p
  float beta;
  int nesterov, iterations;
  float coefficients[48];
  int* status;
};
typedef double (*Square)[SQUARE_PITCH];

// c (8 x 8) += a (8 x 4) b (4 x 8): lane l holds a[l / 4][l % 4], b[l % 4][l / 4], c[l / 4][2 (l % 4) + {0, 1}].
__device__ __forceinline__ void mma8(double* c, double a, double b) {
  asm volatile("mma.sync.aligned.m8n8k4.row.col.f64.f64.f64.f64 {%0, %1}, {%2}, {%3}, {%0, %1};" : "+d"(c[0]), "+d"(c[1]) : "d"(a), "d"(b));
}
// `chunk` columns (rows, where the matrix is tall) of U from `begin` on as u[i * pitch + k], i < p, zeros behind the last; M' is
// written.
template <bool WRITE>
__device__ __forceinline__ void load_thin(const Entry& e, float beta, int nesterov, int begin, int chunk, bool write_m, double* u) {
  const bool tall = e.rows > e.cols;
  const int p = tall ? e.cols : e.rows, pitch = chunk + 4;
  const int across = tall ? e.octets : chunk / 8, octets = (tall ? chunk : p) * across;
#pragma unroll 2
  for (int o = threadIdx.x; o < octets; o += THREADS) {
    const int r = o / across, row = tall ? begin + r : r, octet = (tall ? 0 : begin / 8) + o - r * across;
    float m[8], x[8];
    const bool in = row < e.rows && octet < e.octets;
    if (in) {
      load_u8(e, beta, nesterov, row, octet, m, x);
    } else {
#pragma unroll
      for (int k = 0; k < 8; ++k) x[k] = 0.f;
    }
    if (!tall) {      // (zero behind the last column)
      double* to = u + row * pitch + octet * 8 - begin;
#pragma unroll
      for (int k = 0; k < 8; ++k) to[k] = x[k];
    } else {
      double* to = u + octet * 8 * pitch + r;
#pragma unroll
      for (int k = 0; k < 8; ++k) if (octet * 8 + k < p) to[k * pitch] = x[k];
    }
    if constexpr (WRITE) {
      if (e.M && in) {
        const long long at = static_cast<long long>(row) * e.cols + octet * 8;
        if (!write_m) {
#pragma unroll
          for (int k = 0; k < 8; ++k) if (e.Mo != e.M && octet * 8 + k < e.cols) e.Mo[at + k] = e.M[at + k];
        } else if (e.wide) {
          float4* q = reinterpret_cast<float4*>(e.Mo + at);
          q[0] = make_float4(m[0], m[1], m[2], m[3]);
          q[1] = make_float4(m[4], m[5], m[6], m[7]);
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) if (octet * 8 + k < e.cols) e.Mo[at + k] = m[k];
        }
      }
    }
  }
}
// Columns of part `part` of a matrix: whole chunks.
__device__ __forceinline__ void thin_range(const Entry& e, int part, int chunk, int* begin, int* end) {
  const int q = e.rows > e.cols ? e.rows : e.cols, chunks = (q + chunk - 1) / chunk, per = (chunks + e.parts - 1) / e.parts;
  *begin = part * per * chunk;
  *end = *begin + per * chunk < q ? *begin + per * chunk : q;
}

// Partial sums of S: a warp to a row of tiles; where there are fewer than eight, the warps share the columns of a chunk.
template <int CAP>
__global__ void __launch_bounds__(THREADS) thin_gram_kernel(const __grid_constant__ ThinTable<CAP> t) {
  extern __shared__ double thin_smem[];
  double* u = thin_smem;
  pdl_wait();
  const int which = blockIdx.y, part = blockIdx.x;
  const Entry& e = t.t[which];
  if (part >= e.parts) return;
  const int p = e.rows > e.cols ? e.cols : e.rows, tiles = thin_tiles(p), chunk = thin_chunk(tiles), pitch = chunk + 4, groups = WARPS / tiles;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, ti = warp % tiles, group = warp / tiles;
  int begin, end;
  thin_range(e, part, chunk, &begin, &end);
  double c[8][2] = {};
  const double* mine = u + (lane >> 2) * pitch + (lane & 3);
  for (int k0 = begin; k0 < end; k0 += chunk) {
    __syncthreads();
    load_thin<false>(e, t.beta, t.nesterov, k0, chunk, false, u);
    __syncthreads();
    // (rows behind p hold anything: their sums are not written)
#pragma unroll 2
    for (int k = group * 4; k < chunk; k += 4 * groups) {
      const double a = mine[8 * ti * pitch + k];
#pragma unroll
      for (int tj = 0; tj < 8; ++tj) {
        if (tj >= tiles) break;
        mma8(c[tj], a, mine[8 * tj * pitch + k]);
      }
    }
  }
  // the groups' sums, one after the other
  const Square sum = reinterpret_cast<Square>(thin_smem);
  for (int g = 0; g < groups; ++g) {
    __syncthreads();
    if (group == g) {
#pragma unroll
      for (int tj = 0; tj < 8; ++tj) {
        if (tj >= tiles) break;
        double* to = &sum[8 * ti + (lane >> 2)][8 * tj + 2 * (lane & 3)];
        to[0] = g == 0 ? c[tj][0] : to[0] + c[tj][0];
        to[1] = g == 0 ? c[tj][1] : to[1] + c[tj][1];
      }
    }
  }
  __syncthreads();
  double* S = t.S[which] + static_cast<long long>(part) * p * p;
  for (int i = threadIdx.x; i < p * p; i += THREADS) S[i] = sum[i / p][i % p];
}

// C = A B of tiles x tiles tiles: f(row, column, value) for every element of C.  Everything is symmetric up to rounding (all are
// polynomials in S), so B is read along its rows like A, and tiles below the diagonal are those above it, turned: 36 of 64 for
// p = 64, which the fp64 instructions are busy with for 1.2 us instead of 2.1.
template <typename F>
__device__ __forceinline__ void thin_product(const Square A, const Square B, int tiles, F f) {
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int i = warp; i < tiles * (tiles + 1) / 2; i += blockDim.x / 32) {
    int ti = 0, tj = i;
    while (tj >= tiles - ti) tj -= tiles - ti++;
    tj += ti;
    double c[2][2] = {};
#pragma unroll 4
    for (int k = 0; k < 8 * tiles; k += 8) {
      mma8(c[0], A[8 * ti + (lane >> 2)][k + (lane & 3)], B[8 * tj + (lane >> 2)][k + (lane & 3)]);
      mma8(c[1], A[8 * ti + (lane >> 2)][k + 4 + (lane & 3)], B[8 * tj + (lane >> 2)][k + 4 + (lane & 3)]);
    }
    const int row = 8 * ti + (lane >> 2), col = 8 * tj + 2 * (lane & 3);
#pragma unroll
    for (int v = 0; v < 2; ++v) {
      const double x = c[0][v] + c[1][v];
      f(row, col + v, x);
      if (ti != tj) f(col + v, row, x);
    }
  }
}
constexpr int SOLVE_THREADS = 512;
// A block to a matrix, or a cluster whose blocks share the adding up of the parts (2 MB for 64 parts of p = 64: 100 of 200 us alone).
template <int CAP>
__global__ void __launch_bounds__(SOLVE_THREADS) thin_solve_kernel(const __grid_constant__ ThinTable<CAP> t) {
  extern __shared__ double thin_smem[];
  __shared__ double norm;
  const int rows = t.tiles * 8;
  // S and Q move between two buffers each
  const Square S0 = reinterpret_cast<Square>(thin_smem), S1 = S0 + rows, Q0 = S1 + rows, Q1 = Q0 + rows, A = Q1 + rows;
  if (gridDim.x > 1) ptx::cluster_sync_all();      // (the first block is known to run before the others write to it; under the tail of the kernel before)
  pdl_wait();
  const int which = blockIdx.y;
  const Entry& e = t.t[which];
  const int p = e.rows > e.cols ? e.cols : e.rows, tiles = (p + 7) / 8;
  const double* partial = t.S[which];
  for (int i = blockIdx.x * SOLVE_THREADS + threadIdx.x; i < 64 * tiles * tiles; i += gridDim.x * SOLVE_THREADS) {
    const int r = i / (8 * tiles), c = i % (8 * tiles);
    double s = 0.0;
    if (r < p && c < p) {
#pragma unroll 16
      for (int k = 0; k < e.parts; ++k) s += __ldcg(partial + static_cast<long long>(k) * p * p + r * p + c);
    }
    asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(ptx::map_to_cta(ptx::smem_u32(&S0[r][c]), 0)), "d"(s) : "memory");
  }
  if (gridDim.x > 1) ptx::cluster_sync_all();
  else __syncthreads();
  if (blockIdx.x > 0) return;
  if (threadIdx.x < 32) {
    double trace = 0.0;
    for (int i = threadIdx.x; i < p; i += 32) trace += S0[i][i];
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) trace += __shfl_xor_sync(0xffffffffu, trace, o);
    if (threadIdx.x == 0) norm = sqrt(trace);
  }
  __syncthreads();
  const bool finite = isfinite(static_cast<float>(norm));
  const double inv = finite ? 1.0 / (norm + 1e-7) : 0.0;
  for (int i = threadIdx.x; i < 64 * tiles * tiles; i += SOLVE_THREADS) S0[i / (8 * tiles)][i % (8 * tiles)] *= inv * inv;
  __syncthreads();
  Square S = S0, S_next = S1, Q = Q0, Q_next = Q1;
  for (int it = 0; it < t.iterations && finite; ++it) {
    const double a = t.coefficients[3 * it], b = t.coefficients[3 * it + 1], c = t.coefficients[3 * it + 2];
    // (Q is the identity before the first iteration, and nobody asks for S after the last one)
    thin_product(S, S, tiles, [&](int r, int k, double x) {
      A[r][k] = fma(c, x, fma(b, S[r][k], r == k ? a : 0.0));
      if (it == 0) Q_next[r][k] = A[r][k];
    });
    __syncthreads();
    if (it > 0) thin_product(A, Q, tiles, [&](int r, int k, double x) { Q_next[r][k] = x; });
    if (it + 1 < t.iterations) {
      thin_product(A, S, tiles, [&](int r, int k, double x) { S_next[r][k] = x; });
      __syncthreads();
      thin_product(S_next, A, tiles, [&](int r, int k, double x) { S[r][k] = x; });
    }
    __syncthreads();
    const Square q = Q;
    Q = Q_next;
    Q_next = q;
  }
  // what is not finite leaves here as NaN: the last kernel leaves such a matrix alone
  for (int i = threadIdx.x; i < p * p; i += SOLVE_THREADS)
    t.Q[which][i] = finite ? Q[i / p][i % p] * inv : __longlong_as_double(0x7fffffffffffffffll);
  if (threadIdx.x == 0 && !finite) record_status(t.status, FFSPLIT_ERR_NONFINITE, e.place, KID_MUON);
}

// W' = keep W - step Q U for every chunk, and M'.  A warp to every eighth eight columns.
template <int CAP>
__global__ void __launch_bounds__(THREADS) thin_apply_kernel(const __grid_constant__ ThinTable<CAP> t) {
  extern __shared__ double thin_smem[];
  pdl_wait();
  const int which = blockIdx.y, part = blockIdx.x;
  const Entry& e = t.t[which];
  if (part >= e.parts) return;
  const bool tall = e.rows > e.cols;
  const int p = tall ? e.cols : e.rows, tiles = thin_tiles(p), chunk = thin_chunk(tiles), pitch = chunk + 4;
  double* u = thin_smem + THIN_U_BYTES / sizeof(double);
  const Square Q = reinterpret_cast<Square>(u);
  u = thin_smem;
  for (int i = threadIdx.x; i < 64 * tiles * tiles; i += THREADS) {
    const int r = i / (8 * tiles), c = i % (8 * tiles);
    Q[r][c] = r < p && c < p ? __ldcg(t.Q[which] + r * p + c) : 0.0;
  }
  for (int i = p * pitch + threadIdx.x; i < 8 * tiles * pitch; i += THREADS) u[i] = 0.0;      // (rows behind p count with a zero of Q: no NaN there)
  int begin, end;
  thin_range(e, part, chunk, &begin, &end);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  bool finite = true;
  for (int k0 = begin; k0 < end; k0 += chunk) {
    __syncthreads();
    if (k0 == begin) finite = Q[0][0] == Q[0][0];
    load_thin<true>(e, t.beta, t.nesterov, k0, chunk, finite, u);
    __syncthreads();
    for (int n0 = 8 * warp; n0 < chunk; n0 += 8 * WARPS) {
      double c[8][2] = {};
      for (int k = 0; k < 8 * tiles; k += 4) {
        const double b = u[(k + (lane & 3)) * pitch + n0 + (lane >> 2)];
#pragma unroll
        for (int ti = 0; ti < 8; ++ti) {
          if (ti >= tiles) break;
          mma8(c[ti], Q[8 * ti + (lane >> 2)][k + (lane & 3)], b);
        }
      }
      __syncwarp();
      // (a warp reads and writes its own columns only)
#pragma unroll
      for (int ti = 0; ti < 8; ++ti) {
        const int r = 8 * ti + (lane >> 2);
        if (ti >= tiles || r >= p) break;
        u[r * pitch + n0 + 2 * (lane & 3)] = c[ti][0];
        u[r * pitch + n0 + 2 * (lane & 3) + 1] = c[ti][1];
      }
      __syncwarp();
    }
    __syncthreads();
    // as load_thin() went over U
    const int across = tall ? e.octets : chunk / 8, octets = (tall ? chunk : p) * across;
#pragma unroll 2
    for (int o = threadIdx.x; o < octets; o += THREADS) {
      const int r = o / across, row = tall ? k0 + r : r, octet = (tall ? 0 : k0 / 8) + o - r * across;
      if (row >= e.rows || octet >= e.octets) continue;
      const long long at = static_cast<long long>(row) * e.cols + octet * 8;
      const float keep = finite ? 1.0f - e.decay : 1.0f, step = finite ? e.step : 0.f;
      float x[8], w[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int col = octet * 8 + k;
        x[k] = static_cast<float>(tall ? (col < p ? u[col * pitch + r] : 0.0) : u[row * pitch + col - k0]);
        w[k] = 0.f;
      }
      if (e.W) {
        if (e.wide_w && e.w_f32) {
          const float4* q = reinterpret_cast<const float4*>(static_cast<const float*>(e.W) + at);
          const float4 f = q[0], g = q[1];
          w[0] = f.x; w[1] = f.y; w[2] = f.z; w[3] = f.w; w[4] = g.x; w[5] = g.y; w[6] = g.z; w[7] = g.w;
        } else if (e.wide_w) {
          const uint4 q = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(e.W) + at);
          const uint32_t v[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            w[2 * k] = __uint_as_float(v[k] << 16);
            w[2 * k + 1] = __uint_as_float(v[k] & 0xffff0000u);
          }
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k)
            if (octet * 8 + k < e.cols) w[k] = e.w_f32 ? static_cast<const float*>(e.W)[at + k] : __bfloat162float(static_cast<const __nv_bfloat16*>(e.W)[at + k]);
        }
        // (where nothing is to be updated Q U is NaN)
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = finite ? fmaf(keep, w[k], -step * x[k]) : w[k];
      }
      if (e.wide_w && e.w_f32) {
        float4* q = reinterpret_cast<float4*>(static_cast<float*>(e.out) + at);
        q[0] = make_float4(x[0], x[1], x[2], x[3]);
        q[1] = make_float4(x[4], x[5], x[6], x[7]);
      } else if (e.wide_w) {
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(e.out) + at) =
            make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (octet * 8 + k >= e.cols) break;
          if (e.w_f32) static_cast<float*>(e.out)[at + k] = x[k];
          else static_cast<__nv_bfloat16*>(e.out)[at + k] = __float2bfloat16_rn(x[k]);
        }
      }
    }
  }
}

}  // namespace muon

namespace {

constexpr float kStandard[3] = {3.4445f, -4.7750f, 2.0315f};

inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// Bytes of one matrix's buffers: X twice, S and P (in pairs of iterations two more of these), two planes each.
bool in_pairs(int rows, int cols, bool precise);
size_t x_bytes(int rows, int cols) { return static_cast<size_t>(rows + muon::block_rows(rows)) * round_up(cols, 64) * 2; }
int thin_parts(int rows, int cols) {      // (parts are whole chunks)
  const int p = rows < cols ? rows : cols, q = rows < cols ? cols : rows, chunk = muon::thin_chunk(muon::thin_tiles(p));
  const int chunks = (q + chunk - 1) / chunk, most = chunks < muon::THIN_PARTS ? chunks : muon::THIN_PARTS, per = (chunks + most - 1) / most;
  return (chunks + per - 1) / per;
}
// Whether products take both planes of their operands and sums leave tensor memory every few k-blocks: fp32 gradients, and matrices
// with a side above 2^18.  Tensor cores cut what they add at the last place of the running sum; the square's diagonal is a sum of
// terms of one sign, which loses n 2^-28 or so of n terms: with bf16 gradients 65 x 2^17 is 1.6e-3 off, 2^18 2.1e-3, 2^19 3.1e-3,
// 2^20 5.6e-3, 2^22 2.2e-2, and 2^25 terms no longer move the sum at all.
constexpr int LONG_SIDE = 1 << 18;
bool is_precise(const ffsplit_muon_tensor& t) { return t.grad_dtype == FFSPLIT_F32 || t.rows > LONG_SIDE || t.cols > LONG_SIDE; }
bool is_thin(int rows, int cols) { return (rows < cols ? rows : cols) <= muon::THIN; }
size_t matrix_bytes(int rows, int cols, bool precise) {
  const int p = rows < cols ? rows : cols;
  if (is_thin(rows, cols)) return up256(static_cast<size_t>(thin_parts(rows, cols) + 1) * p * p * sizeof(double));
  return 2 * x_bytes(rows, cols) + (in_pairs(rows, cols, precise) ? 4 : 2) * x_bytes(p, p);
}
constexpr size_t kTableBytes = muon::MAX_TENSORS * (muon::MAX_PARTS * sizeof(double) + sizeof(muon::Target));
// Matrices are worked on in runs: as many as fit the tables and three gigabytes, one at least.
constexpr size_t kRunBytes = static_cast<size_t>(3) << 30;
int run_length(const ffsplit_muon_tensor* t, int count, size_t* bytes) {
  size_t sum = 0;
  int n = 0;
  while (n < count && n < muon::MAX_TENSORS) {
    const size_t more = matrix_bytes(t[n].rows, t[n].cols, is_precise(t[n]));
    if (n > 0 && sum + more > kRunBytes) break;
    sum += more;
    ++n;
  }
  *bytes = sum;
  return n;
}

ffsplit_status check_list(ffsplit_ctx* ctx, const ffsplit_muon_tensor* t, int count) {
  if (count < 0 || (count > 0 && !t)) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "NULL list, or a negative count");
  for (int i = 0; i < count; ++i) {
    if (t[i].rows < 1 || t[i].cols < 1 || t[i].rows > (1 << 30) || t[i].cols > (1 << 30))
      return fail(ctx, FFSPLIT_ERR_SHAPE, "rows and columns must be in [1, 2^30]");
    if (static_cast<long long>(t[i].rows) * t[i].cols > (1ll << 36) || (t[i].rows < t[i].cols ? t[i].rows : t[i].cols) > (1 << 17))
      return fail(ctx, FFSPLIT_ERR_SHAPE, "a matrix of more than 2^36 elements, or both sides above 2^17");
    for (const int32_t d : {t[i].grad_dtype, t[i].weight_dtype})
      if (d != FFSPLIT_F32 && d != FFSPLIT_BF16) return fail(ctx, FFSPLIT_ERR_DTYPE, "unknown dtype in the list");
  }
  return FFSPLIT_OK;
}

// What a list of coefficients allows.
struct Coefficients {
  const float* k;                       // [iterations][3], or nullptr: the standard ones
  int iterations;
  bool pair[16];                        // iterations i and i + 1 may be taken as one
};

// Whether the iteration keeps singular values of [0, 1] below 1.5 and P = a I + b S + c S^2 below 200, and does not carry all of
// them below 2^-10 and on from there (X would leave what its two planes hold; zeros stay zeros); and which iterations keep
// P2 P below 200 together with the one after them (each may be steep where the other one shrinks).
bool coefficients_hold(Coefficients* list) {
  const auto polynomial = [](const float* c, double s) { return c[0] + s * s * (c[1] + s * s * c[2]); };
  const float* c = list->k;
  for (int i = 0; i < 3 * list->iterations; ++i) if (!(std::fabs(c[i]) <= 64.f)) return false;
  double top = 1.0;
  for (int i = 0; i < list->iterations; ++i, c += 3) {
    const bool followed = i + 1 < list->iterations;
    double most = 0.0, both = 0.0;
    for (int k = 0; k <= 4096; ++k) {
      const double s = top * k / 4096, p = polynomial(c, s), v = std::fabs(s * p);
      if (!(std::fabs(p) <= 200.0)) return false;
      if (v > most) most = v;
      if (followed) both = std::fmax(both, std::fabs(p * polynomial(c + 3, v)));
    }
    if (!(most <= 1.5) || (followed && most > 0.0 && most < 0x1p-10)) return false;
    list->pair[i] = followed && both <= 200.0;
    top = most;
  }
  return true;
}

// Matrices of one shape and precision.
struct Group {
  int first, count, rows, cols;
  bool precise, paired, fused;
  muon::Matrices X[2], S, P, T, R;      // T, R: paired only
  int at;                               // which X is the current one
};
// Two iterations at once, where P2 P stays below 200 (see coefficients_hold()).  The second one's S is P S P (all of these are
// polynomials in S), so X need not be formed between the two: X <- (P2 P) X with P2 = a I + b S2 + c S2 S2, S2 = (P S) P.
// 3 p^2 q + 5 p^3 operations instead of 6 p^2 q + 2 p^3, and X is read and written once instead of twice; for two roundings
// more, which leave up to 4e-3 of the result instead of 3e-3 (512 x 2000, all singular values alike: 3.8e-3).  Small matrices would pay for one launch more (256 x 1024: 50 us
// for a pair either way).
bool in_pairs(int rows, int cols, bool precise) {
  const int p = rows < cols ? rows : cols, q = rows < cols ? cols : rows;
  return !precise && p >= 512 && 2ll * q >= 3ll * p;
}

// S and P in one launch, which has a pair of SMs to a matrix whatever p and q are: not where the sum over q is long and there are
// few rows, which goes faster in tiles of 128 columns (an iteration on 65 x 4096: 27.9 us that way, 29.2 in one launch; 128 x 128:
// 14.4 and 11.3; 256 x 4096: 31.1 and 30.7, 64 of them 141 and 131).
bool in_squares(int rows, int cols, bool precise) {
  const int p = rows < cols ? rows : cols, q = rows < cols ? cols : rows;
  return !precise && p <= muon::SQUARE_MOST && q <= 16 * p;
}

// All iterations of up to MAX_GROUPS groups that go alike.
ffsplit_status iterate(ffsplit_ctx* ctx, Group* const* groups, int n, const muon::Target* targets, const Coefficients& list, cudaStream_t st) {
  const float* coefficients = list.k;
  const int iterations = list.iterations;
  const bool precise = groups[0]->precise;
  muon::Product q[muon::MAX_GROUPS];
  // one launch: `fill` says what it is for each group
  const auto launch = [&](auto fill) {
    std::memset(q, 0, sizeof(q));
    for (int i = 0; i < n; ++i) {
      q[i].alpha = 1.f / muon::HELD;
      fill(*groups[i], q[i]);
    }
    return muon::launch_products(ctx, precise, q, n, st);
  };
  // C = alpha A B of p x p matrices that commute
  const auto square = [&](muon::Product& p, const muon::Matrices& A, const muon::Matrices& B, const muon::Matrices& C) {
    p.a = A; p.b = B; p.c = C;
    p.M = p.N = p.K = A.rows;
    p.symmetric = 1;
    p.c_low = precise;
  };
  // P = a I + b S + c S S
  const auto polynomial = [&](muon::Product& p, const float* k, const muon::Matrices& S, const muon::Matrices* add, const muon::Matrices& P) {
    square(p, S, S, P);
    p.alpha *= k[2]; p.beta = k[1]; p.diagonal = k[0];
    p.d = add; p.d_high = 1; p.d_low = precise;
  };
  ffsplit_status s;
  for (int i = 0; i < n; ++i) groups[i]->at = 0;
  for (int it = 0; it < iterations;) {
    const float *k = coefficients ? coefficients + 3 * it : kStandard, *k2 = coefficients ? k + 3 : kStandard;
    const bool pair = groups[0]->paired && list.pair[it];
    if (groups[0]->fused) {                                            // S and P
      muon::Gram squares[muon::MAX_GROUPS];
      for (int i = 0; i < n; ++i) {
        const Group& g = *groups[i];
        const bool tall = g.rows > g.cols;
        squares[i] = {g.X[g.at], g.P, tall, tall ? g.rows : g.cols, k[0], k[1], k[2]};
      }
      if ((s = muon::launch_squares(ctx, squares, n, st)) != FFSPLIT_OK) return s;
    } else if ((s = launch([&](Group& g, muon::Product& p) {           // S = X X^T
           const bool tall = g.rows > g.cols;
           p.a = p.b = g.X[g.at]; p.c = g.S;
           p.a_mn = p.b_mn = tall;
           p.M = p.N = g.S.rows; p.K = tall ? g.rows : g.cols;
           p.symmetric = 1;
           p.c_low = precise;
         })) != FFSPLIT_OK) return s;
    if (!groups[0]->fused && (s = launch([&](Group& g, muon::Product& p) { polynomial(p, k, g.S, &g.S, g.P); })) != FFSPLIT_OK) return s;
    if (pair) {
      if ((s = launch([&](Group& g, muon::Product& p) { square(p, g.P, g.S, g.T); })) != FFSPLIT_OK) return s;            // T = P S
      if ((s = launch([&](Group& g, muon::Product& p) { square(p, g.T, g.P, g.S); })) != FFSPLIT_OK) return s;            // S2 = T P
      if ((s = launch([&](Group& g, muon::Product& p) { polynomial(p, k2, g.S, &g.S, g.T); })) != FFSPLIT_OK) return s;   // P2
      if ((s = launch([&](Group& g, muon::Product& p) { square(p, g.T, g.P, g.R); })) != FFSPLIT_OK) return s;            // R = P2 P
    }
    it += pair ? 2 : 1;
    if ((s = launch([&](Group& g, muon::Product& p) {                  // P X (R X), or X P
           const bool tall = g.rows > g.cols;
           const muon::Matrices &X = g.X[g.at], &P = pair ? g.R : g.P;
           p.a = tall ? X : P; p.b = tall ? P : X; p.c = g.X[1 - g.at];
           p.b_mn = !tall;
           p.M = g.rows; p.N = g.cols; p.K = P.rows;
           if (!precise) {            // (of the second plane only the term a X)
             p.beta = pair ? k[0] * k2[0] : k[0];
             p.d = &X; p.d_low = 1;
           }
           p.c_low = 1;
           if (it == iterations) p.target = targets + g.first;
         })) != FFSPLIT_OK) return s;
    for (int i = 0; i < n; ++i) groups[i]->at = 1 - groups[i]->at;
  }
  return FFSPLIT_OK;
}

// What every kernel needs of a matrix.
muon::Entry entry_for(const ffsplit_muon_tensor& s, int place) {
  muon::Entry e;
  std::memset(&e, 0, sizeof(e));
  e.G = s.grad; e.M = s.momentum; e.Mo = s.momentum_out; e.W = s.weight; e.out = s.out;
  e.rows = s.rows; e.cols = s.cols; e.octets = (s.cols + 7) / 8;
  e.g_f32 = s.grad_dtype == FFSPLIT_F32; e.w_f32 = s.weight_dtype == FFSPLIT_F32;
  e.wide = s.cols % 8 == 0 && aligned16(s.grad) && aligned16(s.momentum) && aligned16(s.momentum_out);
  e.wide_w = s.cols % 8 == 0 && aligned16(s.weight) && aligned16(s.out);
  e.place = place; e.step = s.step; e.decay = s.decay;
  return e;
}

// The thin matrices among t, which begins at place `first` of the caller's list: three launches.
template <int CAP>
ffsplit_status run_thin(ffsplit_ctx* ctx, const ffsplit_muon_tensor* t, int first, int n, float beta, int nesterov, const float* coefficients, int iterations,
                        char* at, cudaStream_t st) {
  muon::ThinTable<CAP> tab;
  std::memset(&tab, 0, sizeof(tab));
  tab.beta = beta; tab.nesterov = nesterov; tab.iterations = iterations;
  for (int i = 0; i < 3 * iterations; ++i) tab.coefficients[i] = coefficients ? coefficients[i] : kStandard[i % 3];
  tab.status = ctx->status();
  int blocks = 0, most = 1;
  for (int i = 0; i < n; ++i) {
    const ffsplit_muon_tensor& s = t[i];
    if (!is_thin(s.rows, s.cols)) continue;
    const int p = s.rows < s.cols ? s.rows : s.cols;
    muon::Entry& e = tab.t[tab.n];
    e = entry_for(s, first + i);
    e.parts = thin_parts(s.rows, s.cols);
    tab.S[tab.n] = reinterpret_cast<double*>(at);
    tab.Q[tab.n] = tab.S[tab.n] + static_cast<size_t>(e.parts) * p * p;
    at += matrix_bytes(s.rows, s.cols, is_precise(s));
    if (p > most) most = p;
    if (e.parts > blocks) blocks = e.parts;
    ++tab.n;
  }
  tab.tiles = muon::thin_tiles(most);
  const int apply_bytes = static_cast<int>(muon::THIN_U_BYTES + muon::square_bytes(tab.tiles));
  cudaError_t e = cudaFuncSetAttribute(muon::thin_solve_kernel<CAP>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(5 * muon::square_bytes(8)));
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(muon::thin_apply_kernel<CAP>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(muon::THIN_U_BYTES + muon::square_bytes(8)));
  if (e != cudaSuccess) return check_cuda(ctx, e, "cudaFuncSetAttribute(muon::thin kernels)");
  e = launch_pdl(muon::thin_gram_kernel<CAP>, dim3(blocks, tab.n), dim3(muon::THREADS), muon::THIN_U_BYTES, st, tab);
  if (e == cudaSuccess) {
    // (a block of the largest p takes an SM)
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(blocks >= 8 && 8 * tab.n <= ctx->num_sms ? 8 : 1, tab.n);
    cfg.blockDim = dim3(muon::SOLVE_THREADS);
    cfg.dynamicSmemBytes = 5 * muon::square_bytes(tab.tiles);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cfg.gridDim.x;
    attr[1].val.clusterDim.y = 1;
    attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, muon::thin_solve_kernel<CAP>, tab);
  }
  if (e == cudaSuccess) e = launch_pdl(muon::thin_apply_kernel<CAP>, dim3(blocks, tab.n), dim3(muon::THREADS), apply_bytes, st, tab);
  ctx->launches += 3;
  return check_cuda(ctx, e, "muon::thin kernels launch");
}

// The first two passes over the other matrices.
template <int CAP>
ffsplit_status run_first(ffsplit_ctx* ctx, const muon::Entry* entries, int n, int blocks, float beta, int nesterov, double* partial, muon::Target* target,
                         cudaStream_t st) {
  muon::Table<CAP> tab;
  std::memset(&tab, 0, sizeof(tab));
  std::memcpy(tab.t, entries, sizeof(muon::Entry) * n);
  tab.n = n; tab.beta = beta; tab.nesterov = nesterov;
  tab.partial = partial; tab.target = target; tab.status = ctx->status();
  cudaError_t e = launch_pdl(muon::norm_kernel<CAP>, dim3(blocks, n), dim3(muon::THREADS), 0, st, tab);
  if (e == cudaSuccess) e = launch_pdl(muon::prepare_kernel<CAP>, dim3(blocks, n), dim3(muon::THREADS), 0, st, tab);
  ctx->launches += 2;
  return check_cuda(ctx, e, "muon::prepare_kernel launch");
}

ffsplit_status run_matrices(ffsplit_ctx* ctx, const ffsplit_muon_tensor* t, int first, int n, float beta, int nesterov, const Coefficients& list, cudaStream_t st) {
  char* ws = ctx->ws + kCtrlBytes;
  double* partial = reinterpret_cast<double*>(ws);
  muon::Target* target = reinterpret_cast<muon::Target*>(ws + sizeof(double) * muon::MAX_TENSORS * muon::MAX_PARTS);
  char* at = ws + up256(kTableBytes);
  int thin = 0;
  for (int i = 0; i < n; ++i) thin += is_thin(t[i].rows, t[i].cols) ? 1 : 0;
  if (thin > 0) {
    const ffsplit_status s = thin <= 4    ? run_thin<4>(ctx, t, first, n, beta, nesterov, list.k, list.iterations, at, st)
                             : thin <= 32 ? run_thin<32>(ctx, t, first, n, beta, nesterov, list.k, list.iterations, at, st)
                                          : run_thin<muon::MAX_TENSORS>(ctx, t, first, n, beta, nesterov, list.k, list.iterations, at, st);
    if (s != FFSPLIT_OK) return s;
    for (int i = 0; i < n; ++i)
      if (is_thin(t[i].rows, t[i].cols)) at += matrix_bytes(t[i].rows, t[i].cols, is_precise(t[i]));
  }
  if (thin == n) return FFSPLIT_OK;
  // matrices of one shape lie one after the other, whatever their place in the list
  Group groups[muon::MAX_TENSORS];
  int order[muon::MAX_TENSORS], n_groups = 0, placed = 0;
  bool done[muon::MAX_TENSORS] = {};
  const auto matrices = [&](int rows, int cols, int count, bool precise) {
    muon::Matrices m;
    m.p = reinterpret_cast<__half*>(at);
    m.rows = rows; m.cols = cols; m.ld = round_up(cols, 64); m.count = count;
    m.each = static_cast<long long>(rows) * m.ld;
    m.low_each = precise ? m.each : muon::block_rows(rows) * m.ld;
    m.low = m.p + m.each * count;
    at += x_bytes(rows, cols) * count;
    return m;
  };
  for (int i = 0; i < n; ++i) {
    if (done[i] || is_thin(t[i].rows, t[i].cols)) continue;
    Group& g = groups[n_groups++];
    g.first = placed; g.count = 0; g.rows = t[i].rows; g.cols = t[i].cols;
    g.precise = is_precise(t[i]);
    for (int j = i; j < n; ++j)
      if (!done[j] && t[j].rows == g.rows && t[j].cols == g.cols && is_precise(t[j]) == g.precise) {
        done[j] = true;
        order[placed++] = j;
        ++g.count;
      }
    const int p = g.rows < g.cols ? g.rows : g.cols;
    g.X[0] = matrices(g.rows, g.cols, g.count, g.precise);
    g.X[1] = matrices(g.rows, g.cols, g.count, g.precise);
    g.S = matrices(p, p, g.count, g.precise);
    g.P = matrices(p, p, g.count, g.precise);
    g.paired = in_pairs(g.rows, g.cols, g.precise);
    g.fused = in_squares(g.rows, g.cols, g.precise);
    if (g.paired) {
      g.T = matrices(p, p, g.count, g.precise);
      g.R = matrices(p, p, g.count, g.precise);
    }
  }
  muon::Entry entries[muon::MAX_TENSORS];
  int blocks = 0;
  for (int gi = 0, k = 0; gi < n_groups; ++gi) {
    const Group& g = groups[gi];
    for (int j = 0; j < g.count; ++j, ++k) {
      const ffsplit_muon_tensor& s = t[order[k]];
      muon::Entry& e = entries[k];
      e = entry_for(s, first + order[k]);
      e.ld = g.X[0].ld;
      e.X = g.X[0].p + j * g.X[0].each;
      e.X_low = g.X[0].low + j * g.X[0].low_each;
      e.blocks = g.precise ? 0 : 1;
      const long long pieces = (s.rows + muon::PIECE_ROWS - 1ll) / muon::PIECE_ROWS * muon::pieces_across(e.octets);
      // (a block to a piece as long as they find room at once, four pieces to a block then)
      const long long few = pieces < 256 ? pieces : 256, many = (pieces + 3) / 4;
      e.parts = static_cast<int>(many < few ? few : many < muon::MAX_PARTS ? many : muon::MAX_PARTS);
      if (e.parts > blocks) blocks = e.parts;
    }
  }
  const ffsplit_status rc = placed <= 4    ? run_first<4>(ctx, entries, placed, blocks, beta, nesterov, partial, target, st)
                            : placed <= 32 ? run_first<32>(ctx, entries, placed, blocks, beta, nesterov, partial, target, st)
                                           : run_first<muon::MAX_TENSORS>(ctx, entries, placed, blocks, beta, nesterov, partial, target, st);
  if (rc != FFSPLIT_OK) return rc;
  for (int kind = 0; kind < 4; ++kind) {      // precise, in pairs, in squares, none of these: groups of one kind go together
    Group* some[muon::MAX_GROUPS];
    int m = 0;
    for (int gi = 0; gi <= n_groups; ++gi) {
      if (gi < n_groups && (groups[gi].precise ? 0 : groups[gi].paired ? 1 : groups[gi].fused ? 2 : 3) == kind) some[m++] = &groups[gi];
      if (m == muon::MAX_GROUPS || (gi == n_groups && m > 0)) {
        const ffsplit_status s = iterate(ctx, some, m, target, list, st);
        if (s != FFSPLIT_OK) return s;
        m = 0;
      }
    }
  }
  return FFSPLIT_OK;
}

}  // namespace
}  // namespace ffsp

extern "C" {

ffsplit_status ffsplit_muon_workspace_size(const ffsplit_muon_tensor* tensors, int32_t count, size_t* bytes) {
  using namespace ffsp;
  if (!bytes) return FFSPLIT_ERR_INVALID_ARG;
  const ffsplit_status s = check_list(nullptr, tensors, count);
  if (s != FFSPLIT_OK) return s;
  size_t most = 0;
  for (int at = 0; at < count;) {
    size_t mine;
    at += run_length(tensors + at, count - at, &mine);
    if (mine > most) most = mine;
  }
  *bytes = kCtrlBytes + up256(kTableBytes) + most;
  return FFSPLIT_OK;
}

ffsplit_status ffsplit_muon_step(ffsplit_ctx* ctx, const ffsplit_muon_tensor* tensors, int32_t count, float beta, int32_t nesterov,
                                 const float* coefficients, int32_t iterations, void* stream) {
  using namespace ffsp;
  ffsplit_status s = check_ctx(ctx, true);
  if (s != FFSPLIT_OK) return s;
  if ((s = check_list(ctx, tensors, count)) != FFSPLIT_OK) return s;
  if (iterations < 1 || iterations > 16) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "1 to 16 iterations");
  if (!std::isfinite(beta)) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "beta must be finite");
  Coefficients list = {coefficients, iterations, {}};
  if (!coefficients) {
    for (int i = 0; i + 1 < iterations; ++i) list.pair[i] = true;      // (P is 3.4445 at most)
  } else if (!coefficients_hold(&list)) {
    return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "coefficients that may carry a singular value above 1.5, or all of them below 2^-10 before the last iteration");
  }
  for (int i = 0; i < count; ++i) {
    const ffsplit_muon_tensor& t = tensors[i];
    if (!t.grad || !t.out) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "NULL tensor in the list");
    if (!t.momentum != !t.momentum_out) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "momentum and momentum_out go together");
    if (t.weight && (!std::isfinite(t.step) || !std::isfinite(t.decay))) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "step and decay must be finite");
    const uintptr_t mask_g = elem_size(t.grad_dtype) - 1, mask_w = elem_size(t.weight_dtype) - 1;
    if ((reinterpret_cast<uintptr_t>(t.grad) & mask_g) || (reinterpret_cast<uintptr_t>(t.momentum) & 3u) ||
        (reinterpret_cast<uintptr_t>(t.momentum_out) & 3u) || (reinterpret_cast<uintptr_t>(t.weight) & mask_w) ||
        (reinterpret_cast<uintptr_t>(t.out) & mask_w))
      return fail(ctx, FFSPLIT_ERR_ALIGN, "a tensor is not aligned to its element size");
  }
  size_t need = 0;
  ffsplit_muon_workspace_size(tensors, count, &need);
  if (need > ctx->ws_bytes) return fail(ctx, FFSPLIT_ERR_BUFFER_TOO_SMALL, "workspace too small for this list (ffsplit_muon_workspace_size)");
  ctx->score_prep.valid = false;   // the scoring buffers share the workspace
  for (int at = 0; at < count;) {
    size_t mine;
    const int n = run_length(tensors + at, count - at, &mine);
    if ((s = run_matrices(ctx, tensors + at, at, n, beta, nesterov, list, static_cast<cudaStream_t>(stream))) != FFSPLIT_OK) return s;
    at += n;
  }
  return FFSPLIT_OK;
}

}  // extern "C"
