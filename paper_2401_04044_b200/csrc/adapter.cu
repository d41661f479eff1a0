// Low-rank adapters of many requests beside a shared projection.
//
//   forward:   P[t] = s_i (X[t] A_i),  Y[t] = X[t] W + bias + P[t] B_i,             i = index[t]
//   backward:  D[t] = s_i (dY[t] B_i^T),  dX[t] = dY[t] W^T + D[t] A_i^T,  dA_i = sum_t X[t]^T D[t],  dB_i = sum_t P[t]^T dY[t]
//
// The shared product runs on the tensor cores (train_gemm.cu).  So do the adapters' products of bf16 batches of more than
// FEW tokens (adapter_tc.cu).  Those of few tokens and of fp32 layers are taken here, on the CUDA cores in fp32.
#include <cstring>
#include <type_traits>

#include "adapter.h"
#include "epilogue.cuh"

namespace ffsp {
namespace adapter {

constexpr int FEW = 64;
constexpr int THREADS = 256;
constexpr int CHUNK = 512;           // elements along a contraction that are staged at a time
constexpr int MAX_SPLITS = 32;
// Tokens of a block.  Tokens of one adapter share its elements; one token to a block where each may have its own.
constexpr int MANY = 8, SOME = 4;
template <bool F32> constexpr int VEC = F32 ? 4 : 8;      // elements of 16 bytes

template <bool F32>
__device__ __forceinline__ float load(const void* p, long long i) {
  return F32 ? __ldg(static_cast<const float*>(p) + i) : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}
template <bool F32>
__device__ __forceinline__ void load_vec(const void* p, long long i, float* v) {      // 16-byte aligned
  if constexpr (F32) {
    const float4 q = __ldg(reinterpret_cast<const float4*>(static_cast<const float*>(p) + i));
    v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
  } else {
    const uint4 q = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(p) + i));
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = __uint_as_float(w[k] << 16);
      v[2 * k + 1] = __uint_as_float(w[k] & 0xffff0000u);
    }
  }
}
template <bool F32>
__device__ __forceinline__ void store(void* p, long long i, float v) {
  if (F32) static_cast<float*>(p)[i] = v;
  else static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
}
__device__ __forceinline__ int adapter_of(const int* index, long long t, int n) {
  const int i = __ldg(index + t);
  return i < 0 || i >= n ? -1 : i;
}

// This block's tokens and their adapters (-1: none); how many there are.
template <int G>
__device__ __forceinline__ int tokens_of(const int* index, const int* order, long long T, int n, int* token, int* of) {
  const long long t0 = static_cast<long long>(blockIdx.x) * G;
  const int count = T - t0 < G ? static_cast<int>(T - t0) : G;
#pragma unroll
  for (int g = 0; g < G; ++g) token[g] = g >= count ? 0 : order ? __ldcg(order + t0 + g) : static_cast<int>(t0 + g);
#pragma unroll
  for (int g = 0; g < G; ++g) of[g] = g < count ? adapter_of(index, token[g], n) : -1;
  return count;
}

// P[t][j] = scale_i sum_k V[t][k] F_i(k, j).  F lies as [n][K][r] (k_minor = 0) or [n][r][K].  K is cut into ranges, so that
// few tokens occupy all SMs; the ranges' sums are added by whoever reads P.  Bound by reading each token's factor once.
struct ShrinkJob {
  const void *V, *F;
  float* P;               // [splits][T][r]
  int K, k_minor;
};
struct ShrinkArgs {
  ShrinkJob job[2];
  const int* index;
  const int* order;       // the tokens sorted by adapter, or nullptr: as they come
  const float* scale;
  long long T;
  int n, r, splits;
  int* status;
};
template <bool F32, int G>
__global__ void __launch_bounds__(THREADS) shrink_kernel(const __grid_constant__ ShrinkArgs a) {
  constexpr int V = VEC<F32>;
  __shared__ float x[G][CHUNK];
  __shared__ float part[THREADS * V * G < MAX_RANK * G * 8 ? MAX_RANK * G * 8 : THREADS * V * G];
  pdl_wait();
  const ShrinkJob& job = a.job[blockIdx.y];
  int token[G], of[G];
  const int count = tokens_of<G>(a.index, a.order, a.T, a.n, token, of);
  if (threadIdx.x == 0 && blockIdx.y == 0 && blockIdx.z == 0) {
#pragma unroll
    for (int g = 0; g < G; ++g)
      if (g < count && __ldg(a.index + token[g]) >= a.n) record_status(a.status, FFSPLIT_ERR_BAD_INDEX, token[g], KID_ADAPTER);
  }
  const int per = ((job.K + a.splits - 1) / a.splits + 63) / 64 * 64, begin = blockIdx.z * per, end = begin + per < job.K ? begin + per : job.K;
  float* P = job.P + blockIdx.z * a.T * a.r;
  const bool wide = (job.k_minor ? job.K : a.r) % V == 0;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // the rank along memory: a thread to `step` ranks of every slices-th k
  const int step = wide ? V : 1, across = (a.r + step - 1) / step, slices = THREADS / across;
  const int slice = threadIdx.x / across, j0 = (threadIdx.x - slice * across) * step;
  bool staged = false;
  for (int first = 0; first < count; ++first) {
    int i = -1;
    unsigned mask = 0;
#pragma unroll
    for (int g = 0; g < G; ++g) if (g == first) i = of[g];
#pragma unroll
    for (int g = 0; g < G; ++g) mask |= of[g] == i ? 1u << g : 0u;
    if (i < 0 || (mask & ((1u << first) - 1u))) continue;      // none, or taken with an earlier token
    const float scale = a.scale ? __ldg(a.scale + i) : 1.f;
    const long long f0 = static_cast<long long>(i) * job.K * a.r;
    float acc[V][G];
#pragma unroll
    for (int v = 0; v < V; ++v)
#pragma unroll
      for (int g = 0; g < G; ++g) acc[v][g] = 0.f;
    bool fresh = true;
    for (int k0 = begin; k0 < end; k0 += CHUNK) {
      const int m = end - k0 < CHUNK ? end - k0 : CHUNK;
      if (!staged) {
        __syncthreads();
#pragma unroll
        for (int g = 0; g < G; ++g)
          for (int k = threadIdx.x; k < CHUNK; k += THREADS) x[g][k] = g < count && k < m ? load<F32>(job.V, static_cast<long long>(token[g]) * job.K + k0 + k) : 0.f;
        __syncthreads();
        staged = end - begin <= CHUNK;      // (all of this block's range: the other adapters find it there)
      }
      if (!job.k_minor) {
        if (slice < slices) {
          if (wide) {
#pragma unroll 4
            for (int k = slice; k < m; k += slices) {
              float f[V];
              load_vec<F32>(job.F, f0 + static_cast<long long>(k0 + k) * a.r + j0, f);
#pragma unroll
              for (int g = 0; g < G; ++g) {
                const float y = x[g][k];
#pragma unroll
                for (int v = 0; v < V; ++v) acc[v][g] = fmaf(y, f[v], acc[v][g]);
              }
            }
          } else {
#pragma unroll 4
            for (int k = slice; k < m; k += slices) {
              const float f = load<F32>(job.F, f0 + static_cast<long long>(k0 + k) * a.r + j0);
#pragma unroll
              for (int g = 0; g < G; ++g) acc[0][g] = fmaf(x[g][k], f, acc[0][g]);
            }
          }
        }
      } else {
        // a warp to R ranks at a time, lanes along the contraction (one rank after the other waits for every load: 32 us instead of 19
        // for 27 tokens of rank 96, K = 8120)
        constexpr int R = G == 1 ? 4 : 2, STEP = THREADS / 32;
        for (int c = warp; c < a.r; c += R * STEP) {
          float sum[R][G] = {};
          const long long at = f0 + static_cast<long long>(c) * job.K + k0, next = static_cast<long long>(STEP) * job.K;
          if (wide) {
#pragma unroll 2
            for (int k = lane * V; k < m; k += 32 * V) {
              float f[R][V];
#pragma unroll
              for (int q = 0; q < R; ++q) {
                if (c + q * STEP < a.r) {
                  load_vec<F32>(job.F, at + q * next + k, f[q]);
                } else {
#pragma unroll
                  for (int v = 0; v < V; ++v) f[q][v] = 0.f;
                }
              }
#pragma unroll
              for (int g = 0; g < G; ++g)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                  const float y = x[g][k + v];
#pragma unroll
                  for (int q = 0; q < R; ++q) sum[q][g] = fmaf(y, f[q][v], sum[q][g]);
                }
            }
          } else {
#pragma unroll 4
            for (int k = lane; k < m; k += 32) {
              float f[R];
#pragma unroll
              for (int q = 0; q < R; ++q) f[q] = c + q * STEP < a.r ? load<F32>(job.F, at + q * next + k) : 0.f;
#pragma unroll
              for (int g = 0; g < G; ++g) {
                const float y = x[g][k];
#pragma unroll
                for (int q = 0; q < R; ++q) sum[q][g] = fmaf(y, f[q], sum[q][g]);
              }
            }
          }
#pragma unroll
          for (int q = 0; q < R; ++q)
#pragma unroll
            for (int g = 0; g < G; ++g) {
#pragma unroll
              for (int o = 16; o > 0; o >>= 1) sum[q][g] += __shfl_xor_sync(0xffffffffu, sum[q][g], o);
              float* to = part + (c + q * STEP) * G + g;
              if (lane == 0 && c + q * STEP < a.r) *to = fresh ? sum[q][g] : *to + sum[q][g];
            }
        }
      }
      fresh = false;
    }
    __syncthreads();
    int left = 1;
    if (!job.k_minor) {
      if (slice < slices) {
#pragma unroll
        for (int v = 0; v < V; ++v)
          if (v < step)
#pragma unroll
            for (int g = 0; g < G; ++g) part[(slice * a.r + j0 + v) * G + g] = acc[v][g];
      }
      __syncthreads();
      // halves of the slices onto each other, as long as there are many (one after the other, 85 of them took 1.3 us)
      for (left = slices; left > 4;) {
        const int half = (left + 1) / 2, size = a.r * G;
        for (int e = threadIdx.x; e < (left - half) * size; e += THREADS) part[e] += part[half * size + e];
        left = half;
        __syncthreads();
      }
    }
    // (sums of tokens that use another adapter were taken along; they are not written)
    for (int e = threadIdx.x; e < a.r * G; e += THREADS) {
      const int c = e / G, g = e - c * G;
      if (!(mask >> g & 1u)) continue;
      float s = 0.f;
      if (begin < end) {
        for (int k = 0; k < left; ++k) s += part[(k * a.r + c) * G + g];
      }
      int to = 0;
#pragma unroll
      for (int q = 0; q < G; ++q) if (q == g) to = token[q];
      P[static_cast<long long>(to) * a.r + c] = scale * s;
    }
    __syncthreads();
  }
}

// P = the ranges' sums of P, in order (where many blocks read it).
__global__ void __launch_bounds__(THREADS) add_ranges_kernel(float* P0, float* P1, long long count, int splits) {
  pdl_wait();
  float* P = blockIdx.y ? P1 : P0;
  const long long i = static_cast<long long>(blockIdx.x) * THREADS + threadIdx.x;
  if (i >= count) return;
  float s = 0.f;
#pragma unroll 8
  for (int k = 0; k < splits; ++k) s += __ldcg(P + k * count + i);
  P[i] = s;
}

// Y[t][c] = base[t][c] + sum_j P[t][j] F_i(j, c).  F lies as [n][r][N] (r_minor = 0) or [n][N][r].  Bound by reading the
// factors and, of many tokens, base and Y.  The four warps of a block share the ranks (one thread through all of 88: 26 us for
// three tokens).
struct ExpandArgs {
  const float* P;         // [splits][T][r]
  const void *F, *base;
  void* Y;
  const int *index, *order;
  long long T;
  int N, n, r, r_minor, splits;
  int late;               // the kernel before, which gives base, was launched behind all else that is read here: waited for before base
};
constexpr int EXPAND_THREADS = 128, SHARES = EXPAND_THREADS / 32;
template <bool F32, int G>
__global__ void __launch_bounds__(EXPAND_THREADS) expand_kernel(const __grid_constant__ ExpandArgs a) {
  constexpr int V = VEC<F32>;
  __shared__ float p[MAX_RANK][G], sums[SHARES][V][G][32];
  __shared__ int row[G];
  if (!a.late) pdl_wait();
  const bool wide = (a.r_minor ? a.r : a.N) % V == 0;
  const int step = wide && !a.r_minor ? V : 1;              // columns of a thread
  const int lane = threadIdx.x & 31, share = threadIdx.x >> 5, c = ((blockIdx.z * gridDim.y + blockIdx.y) * 32 + lane) * step;
  int token[G], of[G];
  const int count = tokens_of<G>(a.index, a.order, a.T, a.n, token, of);
  if (threadIdx.x == 0) {
#pragma unroll
    for (int g = 0; g < G; ++g) row[g] = of[g] >= 0 ? token[g] : -1;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.r * G; e += EXPAND_THREADS) {
    const int g = e / a.r, j = e - g * a.r;
    float s = 0.f;
    if (row[g] >= 0) {
#pragma unroll 8
      for (int k = 0; k < a.splits; ++k) s += __ldcg(a.P + (k * a.T + row[g]) * a.r + j);
    }
    p[j][g] = s;
  }
  __syncthreads();
  // this warp's ranks, whole vectors of them
  const int each = ((a.r + SHARES - 1) / SHARES + V - 1) / V * V, j0 = share * each, j1 = j0 + each < a.r ? j0 + each : a.r;
  float acc[V][G];
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int g = 0; g < G; ++g) acc[v][g] = 0.f;
  for (int first = 0; first < count && c < a.N; ++first) {
    int i = -1;
    unsigned mask = 0;
#pragma unroll
    for (int g = 0; g < G; ++g) if (g == first) i = of[g];
#pragma unroll
    for (int g = 0; g < G; ++g) mask |= of[g] == i ? 1u << g : 0u;
    if (i < 0 || (mask & ((1u << first) - 1u))) continue;
    const long long f0 = static_cast<long long>(i) * a.N * a.r;
    if (a.r_minor) {
      const long long at = f0 + static_cast<long long>(c) * a.r;
      if (wide) {
#pragma unroll 2
        for (int j = j0; j < j1; j += V) {
          float f[V];
          load_vec<F32>(a.F, at + j, f);
#pragma unroll
          for (int g = 0; g < G; ++g)
            if (mask >> g & 1u)
#pragma unroll
              for (int v = 0; v < V; ++v) acc[0][g] = fmaf(p[j + v][g], f[v], acc[0][g]);
        }
      } else {
#pragma unroll 4
        for (int j = j0; j < j1; ++j) {
          const float f = load<F32>(a.F, at + j);
#pragma unroll
          for (int g = 0; g < G; ++g) if (mask >> g & 1u) acc[0][g] = fmaf(p[j][g], f, acc[0][g]);
        }
      }
    } else if (wide) {
#pragma unroll 4
      for (int j = j0; j < j1; ++j) {
        float f[V];
        load_vec<F32>(a.F, f0 + static_cast<long long>(j) * a.N + c, f);
#pragma unroll
        for (int g = 0; g < G; ++g)
          if (mask >> g & 1u)
#pragma unroll
            for (int v = 0; v < V; ++v) acc[v][g] = fmaf(p[j][g], f[v], acc[v][g]);
      }
    } else {
#pragma unroll 4
      for (int j = j0; j < j1; ++j) {
        const float f = load<F32>(a.F, f0 + static_cast<long long>(j) * a.N + c);
#pragma unroll
        for (int g = 0; g < G; ++g) if (mask >> g & 1u) acc[0][g] = fmaf(p[j][g], f, acc[0][g]);
      }
    }
  }
#pragma unroll
  for (int v = 0; v < V; ++v)
#pragma unroll
    for (int g = 0; g < G; ++g) sums[share][v][g][lane] = acc[v][g];
  __syncthreads();
  if (a.late) pdl_wait();
  if (c >= a.N) return;
  // the shares' sums in order; a warp to every fourth token
#pragma unroll
  for (int g = 0; g < G; ++g) {
    if (g >= count || g % SHARES != share || (of[g] < 0 && a.base == a.Y)) continue;
    const long long at = static_cast<long long>(token[g]) * a.N + c;
    float s[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      s[v] = sums[0][v][g][lane];
#pragma unroll
      for (int k = 1; k < SHARES; ++k) s[v] += sums[k][v][g][lane];
    }
    if (step > 1) {      // (then c + V <= N)
      if constexpr (F32) {
        float4 q = make_float4(0.f, 0.f, 0.f, 0.f);
        if (a.base) q = *reinterpret_cast<const float4*>(static_cast<const float*>(a.base) + at);
        *reinterpret_cast<float4*>(static_cast<float*>(a.Y) + at) = make_float4(q.x + s[0], q.y + s[1], q.z + s[2], q.w + s[3]);
      } else {
        uint32_t w[4] = {0u, 0u, 0u, 0u};
        if (a.base) {
          const uint4 q = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.base) + at);
          w[0] = q.x; w[1] = q.y; w[2] = q.z; w[3] = q.w;
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
          w[k] = pack_bf16x2(__uint_as_float(w[k] << 16) + s[V > 4 ? 2 * k : 0], __uint_as_float(w[k] & 0xffff0000u) + s[V > 4 ? 2 * k + 1 : 0]);
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.Y) + at) = make_uint4(w[0], w[1], w[2], w[3]);
      }
    } else {
      const float b = !a.base ? 0.f : F32 ? static_cast<const float*>(a.base)[at] : __bfloat162float(static_cast<const __nv_bfloat16*>(a.base)[at]);
      store<F32>(a.Y, at, b + s[0]);
    }
  }
}

// out_i(j, c) = sum over the tokens of adapter i, in order, of P[t][j] V[t][c]; lies as [n][r][N], or [n][N][r] (r_minor).
struct GradJob {
  const float* P;
  const void* V;
  void* out;
  int N, r_minor, blocks;
};
struct GradArgs {
  GradJob job[2];
  const int* index;
  const int *count, *offset, *order;      // the tokens sorted by adapter, or nullptr: there are no more than THREADS
  long long T;
  int n, r;
  int apart;                              // as in expand's launch, but waited for at the end
};
// A block takes 64 columns, two to a thread, and all ranks.  Bound by writing the gradients, most of them zeros where a few tokens
// meet many adapters (57 of rank 88 and 10256 columns, 10 tokens: 92 us with 32 columns and 2 bytes to a store, 41 us so).
constexpr int GRAD_COLS = 64, GRAD_TOKENS = 32;
// U: ranks of a thread, at least r / 8.
template <bool F32, int U>
__global__ void __launch_bounds__(THREADS) gradient_kernel(const __grid_constant__ GradArgs a) {
  using Value = std::conditional_t<F32, float, __nv_bfloat16>;
  constexpr int RANKS = 8 * U;
  constexpr size_t P_BYTES = GRAD_TOKENS * RANKS * 4, OUT_BYTES = GRAD_COLS * RANKS * sizeof(Value);
  __shared__ __align__(16) char area[P_BYTES > OUT_BYTES ? P_BYTES : OUT_BYTES];
  __shared__ __align__(16) float v[GRAD_TOKENS][GRAD_COLS];
  __shared__ int list[THREADS], found[THREADS / 32];
  float(*p)[RANKS] = reinterpret_cast<float(*)[RANKS]>(area);
  if (!a.apart) pdl_wait();
  const int which = static_cast<int>(blockIdx.x) >= a.job[0].blocks ? 1 : 0, i = blockIdx.y;
  const GradJob& job = a.job[which];
  const int c0 = (blockIdx.x - (which ? a.job[0].blocks : 0)) * GRAD_COLS;
  const int lane = threadIdx.x & 31, jg = threadIdx.x >> 5;
  float acc[U][2] = {};
  const int mine = a.order ? __ldcg(a.count + i) : static_cast<int>(a.T), from = a.order ? __ldcg(a.offset + i) : 0;
  for (int t0 = 0; t0 < mine; t0 += THREADS) {
    int all;
    if (a.order) {
      all = mine - t0 < THREADS ? mine - t0 : THREADS;
      if (static_cast<int>(threadIdx.x) < all) list[threadIdx.x] = __ldcg(a.order + from + t0 + threadIdx.x);
    } else {
      const bool hit = static_cast<int>(threadIdx.x) < mine && __ldg(a.index + threadIdx.x) == i;
      const unsigned votes = __ballot_sync(0xffffffffu, hit);
      if (lane == 0) found[jg] = __popc(votes);
      __syncthreads();
      int before = 0;
      all = 0;
#pragma unroll
      for (int w = 0; w < THREADS / 32; ++w) {
        if (w < jg) before += found[w];
        all += found[w];
      }
      if (hit) list[before + __popc(votes & ((1u << lane) - 1u))] = threadIdx.x;
    }
    __syncthreads();
    for (int b = 0; b < all; b += GRAD_TOKENS) {
      const int m = all - b < GRAD_TOKENS ? all - b : GRAD_TOKENS;
      for (int e = threadIdx.x; e < m * a.r; e += THREADS) {
        const int q = e / a.r, j = e - q * a.r;
        p[q][j] = __ldcg(job.P + static_cast<long long>(list[b + q]) * a.r + j);
      }
      for (int e = threadIdx.x; e < m * GRAD_COLS; e += THREADS) {
        const int q = e / GRAD_COLS, c = e % GRAD_COLS;
        v[q][c] = c0 + c < job.N ? load<F32>(job.V, static_cast<long long>(list[b + q]) * job.N + c0 + c) : 0.f;
      }
      __syncthreads();
      for (int q = 0; q < m; ++q) {
        const float2 x = *reinterpret_cast<const float2*>(&v[q][2 * lane]);
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (jg + 8 * u < a.r) {
            acc[u][0] = fmaf(p[q][jg + 8 * u], x.x, acc[u][0]);
            acc[u][1] = fmaf(p[q][jg + 8 * u], x.y, acc[u][1]);
          }
      }
      __syncthreads();
    }
  }
  const long long first = static_cast<long long>(i) * job.N * a.r;
  if (job.r_minor) {
    // these columns' ranks are one run of memory
    Value* turn = reinterpret_cast<Value*>(area);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (jg + 8 * u < a.r) {
        store<F32>(turn, 2 * lane * a.r + jg + 8 * u, acc[u][0]);
        store<F32>(turn, (2 * lane + 1) * a.r + jg + 8 * u, acc[u][1]);
      }
    __syncthreads();
    const int n = (job.N - c0 < GRAD_COLS ? job.N - c0 : GRAD_COLS) * a.r;
    Value* out = static_cast<Value*>(job.out) + first + static_cast<long long>(c0) * a.r;
    constexpr int V = VEC<F32>;
    const int whole = (reinterpret_cast<uintptr_t>(out) & 15u) == 0 ? n / V : 0;
    for (int e = threadIdx.x; e < whole; e += THREADS) reinterpret_cast<uint4*>(out)[e] = reinterpret_cast<const uint4*>(turn)[e];
    for (int e = whole * V + threadIdx.x; e < n; e += THREADS) out[e] = turn[e];
  } else {
    const int c = c0 + 2 * lane;
    const bool even = job.N % 2 == 0;      // (then every row starts on two elements)
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = jg + 8 * u;
      if (j >= a.r || c >= job.N) break;
      const long long at = first + static_cast<long long>(j) * job.N + c;
      if (even) {
        if constexpr (F32) *reinterpret_cast<float2*>(static_cast<float*>(job.out) + at) = make_float2(acc[u][0], acc[u][1]);
        else *reinterpret_cast<uint32_t*>(static_cast<__nv_bfloat16*>(job.out) + at) = pack_bf16x2(acc[u][0], acc[u][1]);
      } else {
        store<F32>(job.out, at, acc[u][0]);
        if (c + 1 < job.N) store<F32>(job.out, at + 1, acc[u][1]);
      }
    }
  }
  if (a.apart) pdl_wait();
}

}  // namespace adapter

namespace {

inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// Batches whose adapters' products run on the tensor cores.
bool on_tensor_cores(const ffsplit_projection& p, int n, long long T) {
  return p.dtype == FFSPLIT_BF16 && T > adapter::FEW && adapter::tile_bound(T, n) <= 65535;
}

// Batches whose tokens are sorted by adapter first (few tokens are not: that is a launch more).
bool is_sorted(long long T) { return T > adapter::FEW; }

// Ranges of K of the products on the CUDA cores: two blocks to an SM (as many as fit: a few more take twice as long), 64
// elements each at least.  (148 SMs: the size of the workspace goes by this, and is asked for without a context.)
int tokens_per_block(const ffsplit_projection& p, int n, long long T) {
  if (T > adapter::FEW) return p.dtype == FFSPLIT_F32 ? adapter::MANY : adapter::SOME;      // (bf16: 65000 adapters and more)
  return n == 1 ? adapter::SOME : 1;
}
int splits_of(const ffsplit_projection& p, int n, long long T) {
  const int group = tokens_per_block(p, n, T), K = p.in > p.out ? p.in : p.out;
  const long long blocks = (T + group - 1) / group;
  long long s = 2 * 148 / blocks;
  if (s > K / 64) s = K / 64;
  return static_cast<int>(s < 1 ? 1 : s > adapter::MAX_SPLITS ? adapter::MAX_SPLITS : s);
}

// The adapters' part inside the shared product, in a product of `width` columns over `sum`: entries to a tile of 256 rows.  An
// entry costs a tile as much as one or two k-blocks of its sum; where a tile has more adapters than half its k-blocks, or than
// 32, a second pass over Y is cheaper.  So it is where Y is small: the pass moves 2.7 TB/s (63 us of 335 for 4096 x 11008), while
// checking the factors and planning the entries take 15 us and the entries of 24 adapters 30 us in that product.  The entries
// take 32 KB (64 KB) each, 256 MB in all at most.
int extension_most(const ffsplit_projection& p, int n, int r, long long T, int sum, int width) {
  if (!on_tensor_cores(p, n, T) || T * width < (32ll << 20)) return 0;
  const long long blocks = (sum + 63) / 64, pitch = adapter::rank_pitch(r);
  long long most = blocks / (2 * (pitch / 64));
  if (most > 32) most = 32;
  if (most > n) most = n;
  const long long room = (256ll << 20) / (adapter::extension_tiles(T) * adapter::EXTENSION_ROWS * pitch * 2);
  return static_cast<int>(most < room ? most : room);
}

struct AdapterLayout {
  long long ldi, ldo, ldr;
  int most, most_back;      // entries to a tile forward, backward
  size_t slot, Q;
  size_t P, D, sorted, X, dY, W, A, B, parts, parts_bytes, end;
};
AdapterLayout adapter_layout(const ffsplit_projection& p, int n, int r, long long T) {
  AdapterLayout L;
  const bool f32 = p.dtype == FFSPLIT_F32, tc = on_tensor_cores(p, n, T);
  const size_t planes = f32 ? 3 : 1;
  L.ldi = round_up_ll(p.in, 64);
  L.ldo = round_up_ll(p.out, 64);
  L.ldr = round_up_ll(r, 8);
  size_t off = 0;
  const auto take = [&](size_t* at, size_t bytes) { *at = off; off = up256(off + bytes); };
  const size_t inner = tc ? static_cast<size_t>(adapter::tile_bound(T, n)) * adapter::TOKENS * adapter::rank_pitch(r) * 2 : static_cast<size_t>(splits_of(p, n, T)) * T * r * 4;
  take(&L.P, inner);
  take(&L.D, inner);
  take(&L.sorted, is_sorted(T) ? (static_cast<size_t>(T) + 2 * (static_cast<size_t>(n) + 1)) * 4 : 0);
  L.most = extension_most(p, n, r, T, p.in, p.out);
  L.most_back = extension_most(p, n, r, T, p.out, p.in);
  const size_t tiles = static_cast<size_t>(adapter::extension_tiles(T)), most = L.most > L.most_back ? L.most : L.most_back;
  take(&L.slot, most ? (static_cast<size_t>(T) + 2 * tiles * (most + 1) + n) * 4 : 0);
  take(&L.Q, tiles * most * adapter::EXTENSION_ROWS * adapter::rank_pitch(r) * 2);
  take(&L.X, f32 || p.in % 8 ? static_cast<size_t>(T) * L.ldi * 2 * planes : 0);
  take(&L.dY, f32 || p.out % 8 ? static_cast<size_t>(T) * L.ldo * 2 * planes : 0);
  take(&L.W, f32 || p.out % 8 ? static_cast<size_t>(p.in) * L.ldo * 2 * planes : 0);
  take(&L.A, tc && r % 8 ? static_cast<size_t>(n) * p.in * L.ldr * 2 : 0);
  take(&L.B, tc && p.out % 8 ? static_cast<size_t>(n) * r * L.ldo * 2 : 0);
  const size_t want = 64 * static_cast<size_t>(T) * (L.ldi > L.ldo ? L.ldi : L.ldo);
  L.parts_bytes = up256(want < (32u << 20) ? want : (32u << 20));
  take(&L.parts, L.parts_bytes);
  L.end = off;
  return L;
}

ffsplit_status check_projection(ffsplit_ctx* ctx, const ffsplit_projection* p, int n, int r, long long T) {
  if (!p) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "projection is NULL");
  if (p->dtype != FFSPLIT_F32 && p->dtype != FFSPLIT_BF16) return fail(ctx, FFSPLIT_ERR_DTYPE, "unknown dtype");
  if (p->in < 1 || p->out < 1 || p->in > (1 << 23) || p->out > (1 << 23)) return fail(ctx, FFSPLIT_ERR_SHAPE, "in and out must be in [1, 2^23]");
  if (n < 1 || n > 65535) return fail(ctx, FFSPLIT_ERR_SHAPE, "1 to 65535 adapters");
  if (r < 1 || r > adapter::MAX_RANK) return fail(ctx, FFSPLIT_ERR_SHAPE, "ranks of 1 to 128");
  if (T < 1 || T > 0x7fffff00ll) return fail(ctx, FFSPLIT_ERR_SHAPE, "T must be in [1, 2^31 - 256]");
  return FFSPLIT_OK;
}
ffsplit_status check_adapters(ffsplit_ctx* ctx, const ffsplit_projection* p, const ffsplit_adapters* a, const void* X, long long T) {
  ffsplit_status s = check_ctx(ctx, true);
  if (s != FFSPLIT_OK) return s;
  if (!a) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "adapters is NULL");
  if ((s = check_projection(ctx, p, a->n, a->r, T)) != FFSPLIT_OK) return s;
  if (!a->A || !a->B || !a->index || !X) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "NULL tensor");
  if (!aligned16(a->A) || !aligned16(a->B) || !aligned16(X)) return fail(ctx, FFSPLIT_ERR_ALIGN, "tensors must be 16-byte aligned");
  if ((reinterpret_cast<uintptr_t>(a->index) & 3u) || (reinterpret_cast<uintptr_t>(a->scale) & 3u))
    return fail(ctx, FFSPLIT_ERR_ALIGN, "index and scale must be 4-byte aligned");
  if (kCtrlBytes + adapter_layout(*p, a->n, a->r, T).end > ctx->ws_bytes)
    return fail(ctx, FFSPLIT_ERR_BUFFER_TOO_SMALL, "workspace too small for this call (ffsplit_adapter_workspace_size)");
  ctx->score_prep.valid = false;   // the scoring buffers share the workspace
  return FFSPLIT_OK;
}

// The operands of a call: the caller's tensors, or their planes (or padded copies) in the workspace.
struct Call {
  ffsplit_ctx* ctx;
  const ffsplit_projection& p;
  const ffsplit_adapters& a;
  long long T;
  AdapterLayout L;
  char* ws;
  cudaStream_t st;
  bool f32, tc;
  train::PrepArgs prep;
  int prep_blocks = 0;
  tg::Matrix X{}, dY{}, W{};
  adapter::Factor A{}, B{};
  adapter::Sorted sorted{};

  Call(ffsplit_ctx* c, const ffsplit_projection& projection, const ffsplit_adapters& adapters, long long tokens, void* stream)
      : ctx(c), p(projection), a(adapters), T(tokens), L(adapter_layout(projection, adapters.n, adapters.r, tokens)), ws(c->ws + kCtrlBytes),
        st(static_cast<cudaStream_t>(stream)), f32(projection.dtype == FFSPLIT_F32), tc(on_tensor_cores(projection, adapters.n, tokens)) {
    std::memset(&prep, 0, sizeof(prep));
  }
  float* inner(size_t at) const { return reinterpret_cast<float*>(ws + at); }
  __nv_bfloat16* tiles(size_t at) const { return reinterpret_cast<__nv_bfloat16*>(ws + at); }
  void use_X(const void* x) { X = train::operand(&prep, &prep_blocks, f32, x, T, p.in, L.ldi, ws + L.X); }
  void use_dY(const void* y) { dY = train::operand(&prep, &prep_blocks, f32, y, T, p.out, L.ldo, ws + L.dY); }
  void use_W(const void* w) { W = train::operand(&prep, &prep_blocks, f32, w, p.in, p.out, L.ldo, ws + L.W); }
  void use_A() { A = {train::operand(&prep, &prep_blocks, false, a.A, static_cast<long long>(a.n) * p.in, a.r, L.ldr, ws + L.A), p.in, a.r, 0}; }
  void use_B() { B = {train::operand(&prep, &prep_blocks, false, a.B, static_cast<long long>(a.n) * a.r, p.out, L.ldo, ws + L.B), a.r, p.out, 1}; }
  // most > 0: the adapters' part is taken along in the shared product, where `F` is the factor (as it came: `each` elements)
  ffsplit_status prepare(int most, const void* F, long long each) {
    if (is_sorted(T)) {
      sorted.count = reinterpret_cast<int*>(ws + L.sorted);
      sorted.offset = sorted.count + a.n + 1;
      sorted.order = sorted.offset + a.n + 1;
      sorted.n = a.n;
      sorted.T = T;
      if (most > 0) {
        const size_t tiles = static_cast<size_t>(adapter::extension_tiles(T));
        sorted.most = most;
        sorted.slot = reinterpret_cast<int*>(ws + L.slot);
        sorted.entries = sorted.slot + T;
        sorted.ids = sorted.entries + tiles;
        sorted.left = sorted.ids + tiles * most;
        sorted.list = sorted.left + tiles;
        sorted.broken = sorted.list + tiles * most;
        sorted.Q = reinterpret_cast<__nv_bfloat16*>(ws + L.Q);
        sorted.pitch = adapter::rank_pitch(a.r);
      }
      ffsplit_status s = adapter::launch_sort(ctx, a.index, sorted, st);
      if (s == FFSPLIT_OK && most > 0) s = adapter::launch_check(ctx, F, each, sorted, st);
      if (s != FFSPLIT_OK) return s;
    }
    prep.apart = is_sorted(T);      // (beside the sort)
    return train::launch_prepare(ctx, prep, prep_blocks, f32, st);
  }
  // C [T, N] = V [T, K] times W [in, out] (transposed: its transpose).
  ffsplit_status shared_product(const tg::Matrix& V, const void* bias, bool transposed, void* C, const adapter::Factor* F = nullptr) {
    tg::Product g;
    std::memset(&g, 0, sizeof(g));
    g.a[0] = V; g.b[0] = W;
    g.pairs = 1;
    g.b_mn = transposed ? 0 : 1;
    g.M = T; g.N = transposed ? p.in : p.out; g.K = transposed ? p.out : p.in;
    g.C = C; g.ldc = g.N; g.bias = bias;
    g.b_ready = 1;      // (the launch before is a shrink: W, or its copy, is complete)
    g.apart = F ? 0 : 1;
    tg::Extension e;
    std::memset(&e, 0, sizeof(e));
    if (F) {
      e.Q = sorted.Q;
      e.entries = adapter::extension_tiles(T) * sorted.most;
      e.pitch = sorted.pitch; e.most = sorted.most;
      e.F = {F->m.p, F->rows, F->cols, F->m.ld, F->rows * F->m.ld, a.n};
      e.rank = a.r;
      e.count = sorted.left; e.list = sorted.list;
    }
    return tg::launch(ctx, tg::PLAIN, 0, f32, &g, 1, tg::Hidden{}, ws + L.parts, L.parts_bytes, st, nullptr, F ? &e : nullptr);
  }
};

template <int G>
ffsplit_status launch_shrink_g(const Call& c, const adapter::ShrinkArgs& s, int jobs) {
  const dim3 grid(static_cast<unsigned>((c.T + G - 1) / G), jobs, s.splits);
  constexpr int G16 = G < adapter::MANY ? G : adapter::SOME;
  const cudaError_t e = c.f32 ? launch_pdl(adapter::shrink_kernel<true, G>, grid, dim3(adapter::THREADS), 0, c.st, s)
                              : launch_pdl(adapter::shrink_kernel<false, G16>, grid, dim3(adapter::THREADS), 0, c.st, s);
  c.ctx->launches++;
  return check_cuda(c.ctx, e, "adapter::shrink_kernel launch");
}
ffsplit_status launch_shrink(const Call& c, adapter::ShrinkArgs& s, int jobs) {
  s.index = c.a.index; s.order = c.sorted.order; s.scale = c.a.scale; s.T = c.T; s.n = c.a.n; s.r = c.a.r; s.status = c.ctx->status();
  s.splits = splits_of(c.p, c.a.n, c.T);
  switch (tokens_per_block(c.p, c.a.n, c.T)) {
    case adapter::MANY: return launch_shrink_g<adapter::MANY>(c, s, jobs);
    case adapter::SOME: return launch_shrink_g<adapter::SOME>(c, s, jobs);
    default: return launch_shrink_g<1>(c, s, jobs);
  }
}
template <int G>
ffsplit_status launch_expand_g(const Call& c, const adapter::ExpandArgs& x) {
  const int vec = c.f32 ? adapter::VEC<true> : adapter::VEC<false>, step = !x.r_minor && x.N % vec == 0 ? vec : 1;
  const unsigned across = (x.N + 32 * step - 1) / (32 * step), y = across < 32768 ? across : 32768;      // (a grid has 65535 rows at most)
  const dim3 grid(static_cast<unsigned>((x.T + G - 1) / G), y, (across + y - 1) / y);
  constexpr int G16 = G < adapter::MANY ? G : adapter::SOME;
  const cudaError_t e = c.f32 ? launch_pdl(adapter::expand_kernel<true, G>, grid, dim3(adapter::EXPAND_THREADS), 0, c.st, x)
                              : launch_pdl(adapter::expand_kernel<false, G16>, grid, dim3(adapter::EXPAND_THREADS), 0, c.st, x);
  c.ctx->launches++;
  return check_cuda(c.ctx, e, "adapter::expand_kernel launch");
}
ffsplit_status launch_expand(const Call& c, const float* P, int splits, const void* F, const void* base, void* Y, int N, int r_minor, bool late) {
  const adapter::ExpandArgs x = {P, F, base, Y, c.a.index, c.sorted.order, c.T, N, c.a.n, c.a.r, r_minor, splits, late};
  switch (tokens_per_block(c.p, c.a.n, c.T)) {
    case adapter::MANY: return launch_expand_g<adapter::MANY>(c, x);
    case adapter::SOME: return launch_expand_g<adapter::SOME>(c, x);
    default: return launch_expand_g<1>(c, x);
  }
}

}  // namespace
}  // namespace ffsp

extern "C" {

ffsplit_status ffsplit_adapter_workspace_size(const ffsplit_projection* projection, int32_t n, int32_t r, int64_t T, size_t* bytes) {
  using namespace ffsp;
  if (!bytes) return FFSPLIT_ERR_INVALID_ARG;
  const ffsplit_status s = check_projection(nullptr, projection, n, r, T);
  if (s != FFSPLIT_OK) return s;
  *bytes = kCtrlBytes + adapter_layout(*projection, n, r, T).end;
  return FFSPLIT_OK;
}

ffsplit_status ffsplit_adapter_forward(ffsplit_ctx* ctx, const ffsplit_projection* projection, const void* W, const void* bias,
                                       const void* base, const ffsplit_adapters* adapters, const void* X, int64_t T, void* Y,
                                       void* stream) {
  using namespace ffsp;
  ffsplit_status s = check_adapters(ctx, projection, adapters, X, T);
  if (s != FFSPLIT_OK) return s;
  if (!Y) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "NULL tensor");
  if ((W && base) || (bias && !W)) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "W (with or without bias), or base, or neither");
  if (!aligned16(W) || !aligned16(bias) || !aligned16(base) || !aligned16(Y)) return fail(ctx, FFSPLIT_ERR_ALIGN, "tensors must be 16-byte aligned");
  Call c(ctx, *projection, *adapters, T, stream);
  if (W || c.tc) c.use_X(X);
  if (W) c.use_W(W);
  if (c.tc) {
    c.use_A();
    c.use_B();
  }
  const bool extended = W && c.L.most > 0;
  if ((s = c.prepare(extended ? c.L.most : 0, adapters->B, static_cast<long long>(c.a.r) * c.p.out)) != FFSPLIT_OK) return s;
  if (c.tc) {
    const adapter::Shrink job = {c.X, c.A, c.tiles(c.L.P), c.p.in, extended ? 1 : 0};
    if ((s = adapter::launch_shrink_tc(ctx, &job, 1, 1, c.sorted, c.a.r, c.a.scale, c.st)) != FFSPLIT_OK) return s;
  } else {
    adapter::ShrinkArgs sh;
    std::memset(&sh, 0, sizeof(sh));
    sh.job[0] = {X, adapters->A, c.inner(c.L.P), c.p.in, 0};
    if ((s = launch_shrink(c, sh, 1)) != FFSPLIT_OK) return s;
  }
  if (W && (s = c.shared_product(c.X, bias, false, Y, extended ? &c.B : nullptr)) != FFSPLIT_OK) return s;
  if (c.tc) return adapter::launch_expand_tc(ctx, c.tiles(c.L.P), c.B, c.p.out, W ? Y : base, Y, c.sorted, c.a.r, extended, W != nullptr, c.st);
  return launch_expand(c, c.inner(c.L.P), splits_of(c.p, c.a.n, T), adapters->B, W ? Y : base, Y, c.p.out, 0, W != nullptr);
}

ffsplit_status ffsplit_adapter_backward(ffsplit_ctx* ctx, const ffsplit_projection* projection, const void* W, const void* base,
                                        const ffsplit_adapters* adapters, const void* X, int64_t T, const void* dY,
                                        const ffsplit_adapter_grads* grads, void* stream) {
  using namespace ffsp;
  ffsplit_status s = check_adapters(ctx, projection, adapters, X, T);
  if (s != FFSPLIT_OK) return s;
  if (!dY || !grads) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "NULL tensor");
  if (!grads->dX && !grads->dA && !grads->dB) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "no gradient asked for");
  if (grads->dX && W && base) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "W, or base, or neither");
  if (!grads->dX) W = base = nullptr;
  for (const void* q : {dY, W, base, static_cast<const void*>(grads->dX), static_cast<const void*>(grads->dA), static_cast<const void*>(grads->dB)})
    if (!aligned16(q)) return fail(ctx, FFSPLIT_ERR_ALIGN, "tensors must be 16-byte aligned");
  Call c(ctx, *projection, *adapters, T, stream);
  const bool dX = grads->dX != nullptr, dA = grads->dA != nullptr, dB = grads->dB != nullptr;
  if (c.tc && (dA || dB)) c.use_X(X);
  if ((dX && W) || c.tc) c.use_dY(dY);
  if (dX && W) c.use_W(W);
  if (c.tc) {
    c.use_A();
    if (dX || dA) c.use_B();
  }
  const bool extended = dX && W && c.L.most_back > 0;
  if ((s = c.prepare(extended ? c.L.most_back : 0, adapters->A, static_cast<long long>(c.p.in) * c.a.r)) != FFSPLIT_OK) return s;
  int n = 0, splits = splits_of(c.p, c.a.n, T);
  if (c.tc) {
    adapter::Shrink jobs[2];
    if (dX || dA) jobs[n++] = {c.dY, c.B, c.tiles(c.L.D), c.p.out, extended ? 1 : 0};
    if (dB) jobs[n++] = {c.X, c.A, c.tiles(c.L.P), c.p.in, 0};
    if ((s = adapter::launch_shrink_tc(ctx, jobs, n, 2, c.sorted, c.a.r, c.a.scale, c.st)) != FFSPLIT_OK) return s;
  } else {
    adapter::ShrinkArgs sh;
    std::memset(&sh, 0, sizeof(sh));
    if (dX || dA) sh.job[n++] = {dY, adapters->B, c.inner(c.L.D), c.p.out, 1};
    if (dB) sh.job[n++] = {X, adapters->A, c.inner(c.L.P), c.p.in, 0};
    if ((s = launch_shrink(c, sh, n)) != FFSPLIT_OK) return s;
    if (splits > 1 && (dA || dB)) {
      const long long count = T * c.a.r;
      const cudaError_t e = launch_pdl(adapter::add_ranges_kernel, dim3(static_cast<unsigned>((count + adapter::THREADS - 1) / adapter::THREADS), n),
                                       dim3(adapter::THREADS), 0, c.st, sh.job[0].P, sh.job[1].P, count, splits);
      ctx->launches++;
      if (e != cudaSuccess) return check_cuda(ctx, e, "adapter::add_ranges_kernel launch");
      splits = 1;
    }
  }
  if (dX) {
    if (W && (s = c.shared_product(c.dY, nullptr, true, grads->dX, extended ? &c.A : nullptr)) != FFSPLIT_OK) return s;
    const void* add = W ? grads->dX : base;
    s = c.tc ? adapter::launch_expand_tc(ctx, c.tiles(c.L.D), c.A, c.p.in, add, grads->dX, c.sorted, c.a.r, extended, W != nullptr, c.st)
             : launch_expand(c, c.inner(c.L.D), splits, adapters->A, add, grads->dX, c.p.in, 1, W != nullptr);
    if (s != FFSPLIT_OK) return s;
  }
  if (!dA && !dB) return FFSPLIT_OK;
  if (c.tc) {
    adapter::Gradient jobs[2];
    n = 0;
    if (dA) jobs[n++] = {c.X, c.tiles(c.L.D), grads->dA, c.p.in, 0};
    if (dB) jobs[n++] = {c.dY, c.tiles(c.L.P), grads->dB, c.p.out, 1};
    return adapter::launch_gradients_tc(ctx, jobs, n, c.sorted, c.a.r, dX, c.st);
  }
  adapter::GradArgs g;
  std::memset(&g, 0, sizeof(g));
  n = 0;
  if (dA) g.job[n++] = {c.inner(c.L.D), X, grads->dA, c.p.in, 1, (c.p.in + adapter::GRAD_COLS - 1) / adapter::GRAD_COLS};
  if (dB) g.job[n++] = {c.inner(c.L.P), dY, grads->dB, c.p.out, 0, (c.p.out + adapter::GRAD_COLS - 1) / adapter::GRAD_COLS};
  g.index = adapters->index; g.T = T; g.n = c.a.n; g.r = c.a.r; g.apart = dX;
  g.count = c.sorted.count; g.offset = c.sorted.offset; g.order = c.sorted.order;
  const dim3 grid(g.job[0].blocks + g.job[1].blocks, c.a.n);
  const auto kernel = c.a.r <= 16 ? (c.f32 ? adapter::gradient_kernel<true, 2> : adapter::gradient_kernel<false, 2>)
                      : c.a.r <= 64 ? (c.f32 ? adapter::gradient_kernel<true, 8> : adapter::gradient_kernel<false, 8>)
                                    : (c.f32 ? adapter::gradient_kernel<true, 16> : adapter::gradient_kernel<false, 16>);
  const cudaError_t e = launch_pdl(kernel, grid, dim3(adapter::THREADS), 0, c.st, g);
  ctx->launches++;
  return check_cuda(ctx, e, "adapter::gradient_kernel launch");
}

}  // extern "C"
