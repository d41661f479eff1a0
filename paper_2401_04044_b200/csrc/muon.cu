// The update of a list of matrices by orthogonalised momentum.
//
//   M' = beta M + G,  U = G + beta M' or M',  X = U / (|U| + 1e-7)
//   X <- a X + (b S + c S^2) X, S = X X^T   (rows <= cols; else X (b S + c S^2), S = X^T X),  once per (a, b, c)
//   W' = (1 - decay) W - step X
//
// Two passes over the gradients (the norm, then X and M'; both read G and M), three products per iteration.  The first
// form of the products: 64 x 64 tiles in fp32 on the CUDA cores.
#include <cmath>
#include <cstring>

#include "epilogue.cuh"
#include "internal.h"

namespace ffsp {
namespace muon {

constexpr int MAX_TENSORS = 128;        // of one launch's table
constexpr int THREADS = 256;
constexpr int MAX_PARTS = 256;          // partial sums of one matrix's squares

// What the last product's epilogue needs of a matrix; lies in the workspace, written by prepare_kernel.
struct Target {
  const void* W;
  void* out;
  float keep, step;       // out = keep W - step X; without W: out = -step X
  int f32;
};
struct Entry {
  const void* G;
  const float* M;
  float* Mo;
  const void* W;
  void* out;
  float* X;               // [rows][ld]
  int rows, cols, octets; // octets of columns in a row
  int g_f32, w_f32, wide; // wide: every octet of G, M, Mo starts on 16 bytes
  int ld;
  int parts, block0;
  float step, decay;
};
struct Table {
  Entry t[MAX_TENSORS];
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
__device__ __forceinline__ const Entry& entry_of(const Table& t, int block, int* which) {
  int lo = 0, hi = t.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.t[mid].block0 <= block) lo = mid; else hi = mid - 1;
  }
  *which = lo;
  return t.t[lo];
}
// Octets begin .. end of block `part` of a matrix.
__device__ __forceinline__ void range_of(const Entry& e, int part, long long* begin, long long* end) {
  const long long all = static_cast<long long>(e.rows) * e.octets, per = (all + e.parts - 1) / e.parts;
  *begin = part * per;
  *end = *begin + per < all ? *begin + per : all;
}
__device__ __forceinline__ void place(const Entry& e, long long i, int* row, int* octet) {
  const long long all = static_cast<long long>(e.rows) * e.octets;
  const long long r = all <= 0xffffffffll ? static_cast<unsigned>(i) / static_cast<unsigned>(e.octets) : i / e.octets;
  *row = static_cast<int>(r);
  *octet = static_cast<int>(i - r * e.octets);
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

__global__ void __launch_bounds__(THREADS) norm_kernel(const __grid_constant__ Table t) {
  __shared__ double red[THREADS / 32];
  pdl_wait();
  int which;
  const Entry& e = entry_of(t, blockIdx.x, &which);
  const int part = blockIdx.x - e.block0;
  long long begin, end;
  range_of(e, part, &begin, &end);
  double acc = 0.0;
  for (long long i = begin + threadIdx.x; i < end; i += THREADS) {
    int row, octet;
    place(e, i, &row, &octet);
    float m[8], u[8];
    load_u8(e, t.beta, t.nesterov, row, octet, m, u);
#pragma unroll
    for (int k = 0; k < 8; ++k) acc += static_cast<double>(u[k]) * static_cast<double>(u[k]);
  }
  const double s = block_sum(acc, red);
  if (threadIdx.x == 0) t.partial[which * MAX_PARTS + part] = s;
}

// X = U / (norm + 1e-7), M', and what the last product does with the matrix.
__global__ void __launch_bounds__(THREADS) prepare_kernel(const __grid_constant__ Table t) {
  __shared__ double red[THREADS / 32];
  pdl_wait();
  int which;
  const Entry& e = entry_of(t, blockIdx.x, &which);
  const int part = blockIdx.x - e.block0;
  const double squares = block_sum(threadIdx.x < e.parts ? __ldcg(t.partial + which * MAX_PARTS + threadIdx.x) : 0.0, red);
  const float norm = static_cast<float>(sqrt(squares));
  const bool finite = isfinite(norm);
  const float inv = finite ? 1.0f / (norm + 1e-7f) : 0.f;
  if (part == 0 && threadIdx.x == 0) {
    Target o;
    o.W = e.W; o.out = e.out; o.f32 = e.w_f32;
    o.keep = finite ? 1.0f - e.decay : 1.0f;
    o.step = e.W ? (finite ? e.step : 0.f) : finite ? -1.0f : __int_as_float(0x7fffffff);
    t.target[which] = o;
    if (!finite) record_status(t.status, FFSPLIT_ERR_NONFINITE, which, KID_MUON);
  }
  long long begin, end;
  range_of(e, part, &begin, &end);
  for (long long i = begin + threadIdx.x; i < end; i += THREADS) {
    int row, octet;
    place(e, i, &row, &octet);
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
    float* x = e.X + static_cast<long long>(row) * e.ld + c;
#pragma unroll
    for (int k = 0; k < 8; ++k) x[k] = finite ? u[k] * inv : 0.f;
  }
}

// C = alpha A B + beta D; A [M, K] lies as [K, M] rows where a_t, B [K, N] as [N, K] where b_t.  With target: the result
// is X, and the matrix is updated instead.
struct ProductArgs {
  const float *A, *B, *D;
  float* C;
  long long batch;        // elements from one matrix of the operands to the next are as below
  long long sA, sB, sD, sC;
  int M, N, K, lda, ldb, ldd, ldc;
  int a_t, b_t;
  float alpha, beta;
  const Target* target;
  int cols;
};
__global__ void __launch_bounds__(256) product_kernel(const __grid_constant__ ProductArgs p) {
  __shared__ float As[16][65], Bs[16][65];
  pdl_wait();
  const int z = blockIdx.z, m0 = blockIdx.y * 64, n0 = blockIdx.x * 64, tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const float *A = p.A + z * p.sA, *B = p.B + z * p.sB;
  float acc[4][4] = {};
  for (int k0 = 0; k0 < p.K; k0 += 16) {
    for (int i = threadIdx.x; i < 1024; i += 256) {
      {
        const int m = p.a_t ? i & 63 : i >> 4, k = p.a_t ? i >> 6 : i & 15;
        const bool in = m0 + m < p.M && k0 + k < p.K;
        As[k][m] = !in ? 0.f : p.a_t ? A[static_cast<long long>(k0 + k) * p.lda + m0 + m] : A[static_cast<long long>(m0 + m) * p.lda + k0 + k];
      }
      {
        const int n = p.b_t ? i >> 4 : i & 63, k = p.b_t ? i & 15 : i >> 6;
        const bool in = n0 + n < p.N && k0 + k < p.K;
        Bs[k][n] = !in ? 0.f : p.b_t ? B[static_cast<long long>(n0 + n) * p.ldb + k0 + k] : B[static_cast<long long>(k0 + k) * p.ldb + n0 + n];
      }
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      float a[4], b[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) { a[i] = As[k][ty + 16 * i]; b[i] = Bs[k][tx + 16 * i]; }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = fmaf(a[i], b[j], acc[i][j]);
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int m = m0 + ty + 16 * i, n = n0 + tx + 16 * j;
      if (m >= p.M || n >= p.N) continue;
      float v = p.alpha * acc[i][j];
      if (p.D) v = fmaf(p.beta, p.D[z * p.sD + static_cast<long long>(m) * p.ldd + n], v);
      if (p.target) {
        const Target& t = p.target[z];
        const long long at = static_cast<long long>(m) * p.cols + n;
        if (t.f32) static_cast<float*>(t.out)[at] = (t.W ? t.keep * static_cast<const float*>(t.W)[at] : 0.f) - t.step * v;
        else static_cast<__nv_bfloat16*>(t.out)[at] = __float2bfloat16_rn((t.W ? t.keep * __bfloat162float(static_cast<const __nv_bfloat16*>(t.W)[at]) : 0.f) - t.step * v);
      } else {
        p.C[z * p.sC + static_cast<long long>(m) * p.ldc + n] = v;
      }
    }
}

}  // namespace muon

namespace {

constexpr float kStandard[3] = {3.4445f, -4.7750f, 2.0315f};

inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// Bytes of one matrix's buffers: X twice, S and b S + c S^2.
size_t matrix_bytes(int rows, int cols) {
  const int p = rows < cols ? rows : cols;
  const size_t x = up256(static_cast<size_t>(rows) * round_up(cols, 64) * 4), s = up256(static_cast<size_t>(p) * round_up(p, 64) * 4);
  return 2 * x + 2 * s;
}
constexpr size_t kTableBytes = muon::MAX_TENSORS * (muon::MAX_PARTS * sizeof(double) + sizeof(muon::Target));
// Matrices are worked on in runs: as many as fit the tables and half a gigabyte, one at least.
constexpr size_t kRunBytes = 512u << 20;
int run_length(const ffsplit_muon_tensor* t, int count, size_t* bytes) {
  size_t sum = 0;
  int n = 0;
  while (n < count && n < muon::MAX_TENSORS) {
    const size_t more = matrix_bytes(t[n].rows, t[n].cols);
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
    if (t[i].rows < 1 || t[i].cols < 1) return fail(ctx, FFSPLIT_ERR_SHAPE, "a matrix without rows or columns");
    if (static_cast<long long>(t[i].rows) * t[i].cols > (1ll << 36) || (t[i].rows < t[i].cols ? t[i].rows : t[i].cols) > (1 << 17))
      return fail(ctx, FFSPLIT_ERR_SHAPE, "a matrix of more than 2^36 elements, or both sides above 2^17");
    for (const int32_t d : {t[i].grad_dtype, t[i].weight_dtype})
      if (d != FFSPLIT_F32 && d != FFSPLIT_BF16) return fail(ctx, FFSPLIT_ERR_DTYPE, "unknown dtype in the list");
  }
  return FFSPLIT_OK;
}

// Whether the iteration keeps singular values of [0, 1] below 1.5.
bool coefficients_hold(const float* c, int iterations) {
  double top = 1.0;
  for (int i = 0; i < iterations; ++i, c += 3) {
    for (int k = 0; k < 3; ++k) if (!(std::fabs(c[k]) <= 64.f)) return false;
    double most = 0.0;
    for (int k = 0; k <= 4096; ++k) {
      const double s = top * k / 4096, v = std::fabs(s * (c[0] + s * s * (c[1] + s * s * c[2])));
      if (v > most) most = v;
    }
    if (!(most <= 1.5)) return false;
    top = most;
  }
  return true;
}

ffsplit_status run_products(ffsplit_ctx* ctx, muon::ProductArgs& p, int batch, cudaStream_t st) {
  const dim3 grid((p.N + 63) / 64, (p.M + 63) / 64, batch);
  const cudaError_t e = launch_pdl(muon::product_kernel, grid, dim3(256), 0, st, p);
  ctx->launches++;
  return check_cuda(ctx, e, "muon::product_kernel launch");
}

ffsplit_status run_matrices(ffsplit_ctx* ctx, const ffsplit_muon_tensor* t, int n, float beta, int nesterov, const float* coefficients,
                            int iterations, cudaStream_t st) {
  char* ws = ctx->ws + kCtrlBytes;
  muon::Table tab;
  std::memset(&tab, 0, sizeof(tab));
  tab.n = n; tab.beta = beta; tab.nesterov = nesterov;
  tab.partial = reinterpret_cast<double*>(ws);
  tab.target = reinterpret_cast<muon::Target*>(ws + sizeof(double) * muon::MAX_TENSORS * muon::MAX_PARTS);
  tab.status = ctx->status();
  char* at = ws + up256(kTableBytes);
  // matrices of one shape lie one after the other, whatever their place in the list
  struct Group { int first, count, rows, cols; char *X0, *X1, *S, *P; };
  Group groups[muon::MAX_TENSORS];
  int order[muon::MAX_TENSORS], n_groups = 0, placed = 0;
  bool done[muon::MAX_TENSORS] = {};
  for (int i = 0; i < n; ++i) {
    if (done[i]) continue;
    Group& g = groups[n_groups++];
    g.first = placed; g.count = 0; g.rows = t[i].rows; g.cols = t[i].cols;
    for (int j = i; j < n; ++j)
      if (!done[j] && t[j].rows == g.rows && t[j].cols == g.cols) {
        done[j] = true;
        order[placed++] = j;
        ++g.count;
      }
    const int p = g.rows < g.cols ? g.rows : g.cols;
    const size_t x = up256(static_cast<size_t>(g.rows) * round_up(g.cols, 64) * 4), s = up256(static_cast<size_t>(p) * round_up(p, 64) * 4);
    g.X0 = at; at += x * g.count;
    g.X1 = at; at += x * g.count;
    g.S = at; at += s * g.count;
    g.P = at; at += s * g.count;
  }
  int blocks = 0;
  for (int gi = 0, k = 0; gi < n_groups; ++gi) {
    const Group& g = groups[gi];
    for (int j = 0; j < g.count; ++j, ++k) {
      const ffsplit_muon_tensor& s = t[order[k]];
      muon::Entry& e = tab.t[k];
      e.G = s.grad; e.M = s.momentum; e.Mo = s.momentum_out; e.W = s.weight; e.out = s.out;
      e.rows = s.rows; e.cols = s.cols; e.octets = (s.cols + 7) / 8;
      e.g_f32 = s.grad_dtype == FFSPLIT_F32; e.w_f32 = s.weight_dtype == FFSPLIT_F32;
      e.ld = round_up(s.cols, 64);
      e.X = reinterpret_cast<float*>(g.X0 + j * up256(static_cast<size_t>(s.rows) * e.ld * 4));
      e.wide = s.cols % 8 == 0 && aligned16(s.grad) && aligned16(s.momentum) && aligned16(s.momentum_out);
      e.step = s.step; e.decay = s.decay;
      const long long octets = static_cast<long long>(s.rows) * e.octets;
      e.parts = static_cast<int>(octets < 512ll * muon::MAX_PARTS ? (octets + 511) / 512 : muon::MAX_PARTS);
      e.block0 = blocks;
      blocks += e.parts;
    }
  }
  cudaError_t e = launch_pdl(muon::norm_kernel, dim3(blocks), dim3(muon::THREADS), 0, st, tab);
  ctx->launches++;
  if (e != cudaSuccess) return check_cuda(ctx, e, "muon::norm_kernel launch");
  e = launch_pdl(muon::prepare_kernel, dim3(blocks), dim3(muon::THREADS), 0, st, tab);
  ctx->launches++;
  if (e != cudaSuccess) return check_cuda(ctx, e, "muon::prepare_kernel launch");
  for (int gi = 0; gi < n_groups; ++gi) {
    const Group& g = groups[gi];
    const bool tall = g.rows > g.cols;
    const int p = tall ? g.cols : g.rows, ldx = round_up(g.cols, 64), lds = round_up(p, 64);
    const long long sx = static_cast<long long>(up256(static_cast<size_t>(g.rows) * ldx * 4)) / 4, ss = static_cast<long long>(up256(static_cast<size_t>(p) * lds * 4)) / 4;
    float *X = reinterpret_cast<float*>(g.X0), *Y = reinterpret_cast<float*>(g.X1), *S = reinterpret_cast<float*>(g.S), *P = reinterpret_cast<float*>(g.P);
    for (int it = 0; it < iterations; ++it) {
      const float a = coefficients ? coefficients[3 * it] : kStandard[0], b = coefficients ? coefficients[3 * it + 1] : kStandard[1],
                  c = coefficients ? coefficients[3 * it + 2] : kStandard[2];
      muon::ProductArgs q;
      std::memset(&q, 0, sizeof(q));
      q.A = q.B = X; q.sA = q.sB = sx; q.lda = q.ldb = ldx;
      q.M = q.N = p; q.K = tall ? g.rows : g.cols;
      q.a_t = tall; q.b_t = !tall;
      q.C = S; q.sC = ss; q.ldc = lds; q.alpha = 1.f;
      ffsplit_status r = run_products(ctx, q, g.count, st);
      if (r != FFSPLIT_OK) return r;
      std::memset(&q, 0, sizeof(q));
      q.A = q.B = q.D = S; q.sA = q.sB = q.sD = ss; q.lda = q.ldb = q.ldd = lds;
      q.M = q.N = q.K = p;
      q.b_t = 1;
      q.C = P; q.sC = ss; q.ldc = lds; q.alpha = c; q.beta = b;
      if ((r = run_products(ctx, q, g.count, st)) != FFSPLIT_OK) return r;
      std::memset(&q, 0, sizeof(q));
      q.M = g.rows; q.N = g.cols; q.K = p;
      q.A = tall ? X : P; q.sA = tall ? sx : ss; q.lda = tall ? ldx : lds;
      q.B = tall ? P : X; q.sB = tall ? ss : sx; q.ldb = tall ? lds : ldx;
      q.D = X; q.sD = sx; q.ldd = ldx; q.alpha = 1.f; q.beta = a;
      q.C = Y; q.sC = sx; q.ldc = ldx;
      if (it + 1 == iterations) { q.target = tab.target + g.first; q.cols = g.cols; }
      if ((r = run_products(ctx, q, g.count, st)) != FFSPLIT_OK) return r;
      float* swap = X; X = Y; Y = swap;
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
  if (coefficients && !coefficients_hold(coefficients, iterations))
    return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "coefficients that may carry a singular value above 1.5");
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
    if ((s = run_matrices(ctx, tensors + at, n, beta, nesterov, coefficients, iterations, static_cast<cudaStream_t>(stream))) != FFSPLIT_OK) return s;
    at += n;
  }
  return FFSPLIT_OK;
}

}  // extern "C"
