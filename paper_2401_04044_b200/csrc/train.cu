// Training a feed-forward layer: forward and backward from the row-major weights.
//
//   gated:  G = X W1, U = X W1u, H = silu(G) U, Y = H W2 + b2
//           dH = dY W2^T, dU = dH silu(G), dG = dH U silu'(G), dX = dG W1^T + dU W1u^T,
//           dW1 = X^T dG, dW1u = X^T dU, dW2 = H^T dY, db2 = sum_t dY
//   GELU:   Z = X W1 + b1, H = act(Z), Y = H W2 + b2; dZ = (dY W2^T) act'(Z), the rest likewise, db1 = sum_t dZ
//
// First form: one plain fp32 kernel for all products (64 x 64 tiles, any strides), with the activation or its
// derivative in its epilogue.
#include <cstring>

#include "epilogue.cuh"
#include "internal.h"

namespace ffsp {
namespace train {

__device__ __forceinline__ void act_and_slope(float z, int act, float* value, float* slope) {
  if (act == FFSPLIT_SWIGLU) {
    const float s = 1.0f / (1.0f + expf(-z));
    *value = z * s;
    *slope = s * (1.0f + z * (1.0f - s));
  } else if (act == FFSPLIT_GELU_ERF) {
    const float phi = 0.5f * erfcf(-z * 0.70710678118654752f);
    *value = z * phi;
    *slope = phi + z * (0.3989422804014327f * expf(-0.5f * z * z));
  } else {
    const float c = 0.79788456080286536f, a = 0.044715f;
    const float t = tanhf(c * (z + a * z * z * z));
    *value = 0.5f * z * (1.0f + t);
    *slope = 0.5f * (1.0f + t) + 0.5f * z * (1.0f - t * t) * (c * (1.0f + 3.0f * a * z * z));
  }
}

// An operand element (i, k) at p[i * si + k * sk].
template <typename E> struct Operand { const E* p; long long si, sk; };

enum Mode : int { PLAIN = 0, FORWARD = 1, BACKWARD = 2 };

template <typename E>
struct SimpleArgs {
  Operand<E> a[2], b[2];
  int pairs;            // PLAIN: products added up
  int gated, act, mode;
  long long M; int N; long long K;
  const E* bias;        // [N] or nullptr
  E* C;                 // PLAIN: output, FORWARD: H; BACKWARD: H
  E *dG, *dU;           // BACKWARD
  float *G, *U;         // FORWARD: written when not nullptr, BACKWARD: read
  long long ldc, ldm;
};

constexpr int TM = 64, TN = 64, TK = 16;

template <typename E>
__global__ void __launch_bounds__(256) simple_kernel(const SimpleArgs<E> p) {
  __shared__ float As[TK][TM + 1], Bs[2][TK][TN + 1];
  pdl_wait();
  const int tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
  const long long row0 = static_cast<long long>(blockIdx.y) * TM;
  const int col0 = blockIdx.x * TN;
  const bool two = p.mode == FORWARD && p.gated;
  float acc[2][4][4] = {};
  for (int pair = 0; pair < p.pairs; ++pair)
    for (long long k0 = 0; k0 < p.K; k0 += TK) {
      for (int i = tid; i < TM * TK; i += 256) {
        const Operand<E>& a = p.a[pair];
        const bool along_k = a.sk == 1;
        const int kk = along_k ? i % TK : i / TM, r = along_k ? i / TK : i % TM;
        const bool in = row0 + r < p.M && k0 + kk < p.K;
        As[kk][r] = in ? to_float<E>(a.p[(row0 + r) * a.si + (k0 + kk) * a.sk]) : 0.f;
      }
      for (int w = 0; w < (two ? 2 : 1); ++w)
        for (int i = tid; i < TN * TK; i += 256) {
          const Operand<E>& b = p.b[two ? w : pair];
          const bool along_k = b.sk == 1;
          const int kk = along_k ? i % TK : i / TN, c = along_k ? i / TK : i % TN;
          const bool in = col0 + c < p.N && k0 + kk < p.K;
          Bs[w][kk][c] = in ? to_float<E>(b.p[(col0 + c) * b.si + (k0 + kk) * b.sk]) : 0.f;
        }
      __syncthreads();
      for (int kk = 0; kk < TK; ++kk)
        for (int i = 0; i < 4; ++i)
          for (int j = 0; j < 4; ++j) {
            acc[0][i][j] = fmaf(As[kk][ty * 4 + i], Bs[0][kk][tx + 16 * j], acc[0][i][j]);
            if (two) acc[1][i][j] = fmaf(As[kk][ty * 4 + i], Bs[1][kk][tx + 16 * j], acc[1][i][j]);
          }
      __syncthreads();
    }
  for (int i = 0; i < 4; ++i)
    for (int j = 0; j < 4; ++j) {
      const long long row = row0 + ty * 4 + i;
      const int col = col0 + tx + 16 * j;
      if (row >= p.M || col >= p.N) continue;
      const float v = acc[0][i][j] + (p.bias ? to_float<E>(p.bias[col]) : 0.f);
      if (p.mode == PLAIN) {
        p.C[row * p.ldc + col] = from_float<E>(v);
        continue;
      }
      const long long at = row * p.ldm + col;
      float a, s;
      if (p.mode == FORWARD) {
        act_and_slope(v, p.act, &a, &s);
        if (p.G) p.G[at] = v;
        if (p.gated) {
          if (p.U) p.U[at] = acc[1][i][j];
          a *= acc[1][i][j];
        }
        p.C[at] = from_float<E>(a);
      } else {
        act_and_slope(p.G[at], p.act, &a, &s);
        if (p.gated) {
          const float u = p.U[at];
          p.dG[at] = from_float<E>(v * u * s);
          p.dU[at] = from_float<E>(v * a);
          p.C[at] = from_float<E>(a * u);
        } else {
          p.dG[at] = from_float<E>(v * s);
          p.C[at] = from_float<E>(a);
        }
      }
    }
}

template <typename E>
__global__ void __launch_bounds__(256) column_sum_kernel(const E* in, long long rows, int cols, long long ld, E* out) {
  __shared__ float red[8][33];
  pdl_wait();
  const int c = blockIdx.x * 32 + (threadIdx.x & 31), w = threadIdx.x >> 5;
  float s = 0.f;
  if (c < cols) for (long long r = w; r < rows; r += 8) s += to_float<E>(in[r * ld + c]);
  red[w][threadIdx.x & 31] = s;
  __syncthreads();
  if (w == 0 && c < cols) {
    for (int i = 1; i < 8; ++i) s += red[i][threadIdx.x];
    out[c] = from_float<E>(s);
  }
}

}  // namespace train

namespace {

inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }

struct TrainLayout { size_t g, u, saved; size_t h, dg, du, end; };
TrainLayout train_layout(const ffsplit_shape& s, long long T) {
  TrainLayout L;
  const bool gated = s.act == FFSPLIT_SWIGLU;
  const size_t es = elem_size(s.dtype), n = static_cast<size_t>(T) * s.m;
  L.g = 0;
  L.u = up256(n * 4);
  L.saved = L.u + (gated ? up256(n * 4) : 0);
  L.h = 0;
  L.dg = up256(n * es);
  L.du = L.dg + up256(n * es);
  L.end = L.du + (gated ? up256(n * es) : 0);
  return L;
}

ffsplit_status check_train(ffsplit_ctx* ctx, const ffsplit_shape* shape, const ffsplit_weights* wt, const void* X, int64_t T) {
  ffsplit_status s = check_ctx(ctx, true);
  if (s != FFSPLIT_OK) return s;
  if ((s = check_shape(ctx, shape)) != FFSPLIT_OK) return s;
  if (T < 1 || T > 0x7fffff00ll) return fail(ctx, FFSPLIT_ERR_SHAPE, "T must be in [1, 2^31 - 256]");
  if (!wt || !wt->W1 || !wt->W2 || !X) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "NULL tensor");
  const bool gated = shape->act == FFSPLIT_SWIGLU;
  if (gated && (!wt->W1u || wt->b1)) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "SwiGLU needs W1u and no b1");
  if (!aligned16(wt->W1) || !aligned16(wt->W2) || !aligned16(X) || (gated && !aligned16(wt->W1u)) || !aligned16(wt->b1) ||
      !aligned16(wt->b2))
    return fail(ctx, FFSPLIT_ERR_ALIGN, "tensors must be 16-byte aligned");
  if (kCtrlBytes + train_layout(*shape, T).end > ctx->ws_bytes)
    return fail(ctx, FFSPLIT_ERR_BUFFER_TOO_SMALL, "workspace too small for this call (ffsplit_train_sizes)");
  return FFSPLIT_OK;
}

ffsplit_status check_saved(ffsplit_ctx* ctx, const ffsplit_shape& s, int64_t T, const void* saved, size_t bytes) {
  if (reinterpret_cast<uintptr_t>(saved) % 256 != 0) return fail(ctx, FFSPLIT_ERR_ALIGN, "saved must be 256-byte aligned");
  if (bytes < train_layout(s, T).saved) return fail(ctx, FFSPLIT_ERR_BUFFER_TOO_SMALL, "saved is too small (ffsplit_train_sizes)");
  return FFSPLIT_OK;
}

template <typename E>
ffsplit_status simple_launch(ffsplit_ctx* ctx, const train::SimpleArgs<E>& a, cudaStream_t st) {
  const cudaError_t e = launch_pdl(train::simple_kernel<E>, dim3((a.N + 63) / 64, static_cast<unsigned>((a.M + 63) / 64)), dim3(256), 0, st, a);
  ctx->launches++;
  return check_cuda(ctx, e, "train::simple_kernel launch");
}

template <typename E>
ffsplit_status run_train_forward(ffsplit_ctx* ctx, const ffsplit_shape& s, const ffsplit_weights& w, const void* X, long long T,
                                 char* saved, void* Y, cudaStream_t st) {
  const TrainLayout L = train_layout(s, T);
  const int d = s.d, m = s.m;
  E* H = reinterpret_cast<E*>(ctx->ws + kCtrlBytes + L.h);
  train::SimpleArgs<E> a;
  std::memset(&a, 0, sizeof(a));
  a.pairs = 1; a.mode = train::FORWARD; a.gated = s.act == FFSPLIT_SWIGLU; a.act = s.act;
  a.a[0] = {static_cast<const E*>(X), d, 1};
  a.b[0] = {static_cast<const E*>(w.W1), 1, m};
  a.b[1] = {static_cast<const E*>(w.W1u), 1, m};
  a.M = T; a.N = m; a.K = d; a.bias = static_cast<const E*>(w.b1);
  a.C = H; a.ldm = m;
  if (saved) { a.G = reinterpret_cast<float*>(saved + L.g); a.U = reinterpret_cast<float*>(saved + L.u); }
  ffsplit_status r = simple_launch(ctx, a, st);
  if (r != FFSPLIT_OK) return r;
  std::memset(&a, 0, sizeof(a));
  a.pairs = 1;
  a.a[0] = {H, m, 1};
  a.b[0] = {static_cast<const E*>(w.W2), 1, d};
  a.M = T; a.N = d; a.K = m; a.bias = static_cast<const E*>(w.b2);
  a.C = static_cast<E*>(Y); a.ldc = d;
  return simple_launch(ctx, a, st);
}

template <typename E>
ffsplit_status run_train_backward(ffsplit_ctx* ctx, const ffsplit_shape& s, const ffsplit_weights& w, const void* X, long long T,
                                  const char* saved, const void* dY, const ffsplit_train_grads& g, cudaStream_t st) {
  const TrainLayout L = train_layout(s, T);
  const int d = s.d, m = s.m;
  const bool gated = s.act == FFSPLIT_SWIGLU;
  char* base = ctx->ws + kCtrlBytes;
  E *H = reinterpret_cast<E*>(base + L.h), *dG = reinterpret_cast<E*>(base + L.dg), *dU = reinterpret_cast<E*>(base + L.du);
  const E *x = static_cast<const E*>(X), *dy = static_cast<const E*>(dY);
  train::SimpleArgs<E> a;
  ffsplit_status r = FFSPLIT_OK;
  if (g.dX || g.dW1 || g.dW1u || g.db1 || g.dW2) {
    std::memset(&a, 0, sizeof(a));
    a.pairs = 1; a.mode = train::BACKWARD; a.gated = gated; a.act = s.act;
    a.a[0] = {dy, d, 1};
    a.b[0] = {static_cast<const E*>(w.W2), d, 1};
    a.M = T; a.N = m; a.K = d;
    a.C = H; a.dG = dG; a.dU = dU; a.ldm = m;
    a.G = reinterpret_cast<float*>(const_cast<char*>(saved) + L.g);
    a.U = reinterpret_cast<float*>(const_cast<char*>(saved) + L.u);
    if ((r = simple_launch(ctx, a, st)) != FFSPLIT_OK) return r;
  }
  if (g.dX) {
    std::memset(&a, 0, sizeof(a));
    a.pairs = gated ? 2 : 1;
    a.a[0] = {dG, m, 1}; a.b[0] = {static_cast<const E*>(w.W1), m, 1};
    a.a[1] = {dU, m, 1}; a.b[1] = {static_cast<const E*>(w.W1u), m, 1};
    a.M = T; a.N = d; a.K = m; a.C = static_cast<E*>(g.dX); a.ldc = d;
    if ((r = simple_launch(ctx, a, st)) != FFSPLIT_OK) return r;
  }
  const E* left[3] = {x, x, H};
  const E* right[3] = {dG, dU, dy};
  void* out[3] = {g.dW1, g.dW1u, g.dW2};
  for (int i = 0; i < 3; ++i) {
    if (!out[i]) continue;
    const int M = i < 2 ? d : m, N = i < 2 ? m : d;
    std::memset(&a, 0, sizeof(a));
    a.pairs = 1;
    a.a[0] = {left[i], 1, M}; a.b[0] = {right[i], 1, N};
    a.M = M; a.N = N; a.K = T; a.C = static_cast<E*>(out[i]); a.ldc = N;
    if ((r = simple_launch(ctx, a, st)) != FFSPLIT_OK) return r;
  }
  const E* sums[2] = {dG, dy};
  void* bias[2] = {g.db1, g.db2};
  for (int i = 0; i < 2; ++i) {
    if (!bias[i]) continue;
    const int cols = i == 0 ? m : d;
    const cudaError_t e = launch_pdl(train::column_sum_kernel<E>, dim3((cols + 31) / 32), dim3(256), 0, st, sums[i], T, cols,
                                     static_cast<long long>(cols), static_cast<E*>(bias[i]));
    ctx->launches++;
    if (e != cudaSuccess) return check_cuda(ctx, e, "column_sum_kernel launch");
  }
  return FFSPLIT_OK;
}

}  // namespace
}  // namespace ffsp

extern "C" {

ffsplit_status ffsplit_train_sizes(const ffsplit_shape* shape, int64_t T, size_t* saved_bytes, size_t* workspace_bytes) {
  using namespace ffsp;
  const ffsplit_status s = check_shape(nullptr, shape);
  if (s != FFSPLIT_OK) return s;
  if (T < 1 || T > 0x7fffff00ll) return FFSPLIT_ERR_SHAPE;
  const TrainLayout L = train_layout(*shape, T);
  if (saved_bytes) *saved_bytes = L.saved;
  if (workspace_bytes) *workspace_bytes = kCtrlBytes + L.end;
  return FFSPLIT_OK;
}

ffsplit_status ffsplit_train_forward(ffsplit_ctx* ctx, const ffsplit_shape* shape, const ffsplit_weights* weights, const void* X,
                                     int64_t T, void* saved, size_t saved_bytes, void* Y, void* stream) {
  using namespace ffsp;
  ffsplit_status s = check_train(ctx, shape, weights, X, T);
  if (s != FFSPLIT_OK) return s;
  if (!Y) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "NULL tensor");
  if (!aligned16(Y)) return fail(ctx, FFSPLIT_ERR_ALIGN, "tensors must be 16-byte aligned");
  if (saved && (s = check_saved(ctx, *shape, T, saved, saved_bytes)) != FFSPLIT_OK) return s;
  ctx->score_prep.valid = false;   // the scoring buffers share the workspace
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  return shape->dtype == FFSPLIT_BF16
             ? run_train_forward<__nv_bfloat16>(ctx, *shape, *weights, X, T, static_cast<char*>(saved), Y, st)
             : run_train_forward<float>(ctx, *shape, *weights, X, T, static_cast<char*>(saved), Y, st);
}

ffsplit_status ffsplit_train_backward(ffsplit_ctx* ctx, const ffsplit_shape* shape, const ffsplit_weights* weights, const void* X,
                                      int64_t T, const void* saved, size_t saved_bytes, const void* dY,
                                      const ffsplit_train_grads* grads, void* stream) {
  using namespace ffsp;
  ffsplit_status s = check_train(ctx, shape, weights, X, T);
  if (s != FFSPLIT_OK) return s;
  if (!saved || !dY || !grads) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "NULL tensor");
  const bool gated = shape->act == FFSPLIT_SWIGLU;
  if (gated && grads->db1) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "SwiGLU has no b1");
  if (!gated && grads->dW1u) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "only SwiGLU has W1u");
  const void* out[6] = {grads->dX, grads->dW1, grads->dW1u, grads->db1, grads->dW2, grads->db2};
  bool any = false;
  for (const void* o : out) {
    any = any || o;
    if (!aligned16(o)) return fail(ctx, FFSPLIT_ERR_ALIGN, "tensors must be 16-byte aligned");
  }
  if (!any) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "no gradient asked for");
  if (!aligned16(dY)) return fail(ctx, FFSPLIT_ERR_ALIGN, "tensors must be 16-byte aligned");
  if ((s = check_saved(ctx, *shape, T, saved, saved_bytes)) != FFSPLIT_OK) return s;
  ctx->score_prep.valid = false;   // the scoring buffers share the workspace
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const char* sv = static_cast<const char*>(saved);
  return shape->dtype == FFSPLIT_BF16 ? run_train_backward<__nv_bfloat16>(ctx, *shape, *weights, X, T, sv, dY, *grads, st)
                                      : run_train_backward<float>(ctx, *shape, *weights, X, T, sv, dY, *grads, st);
}

}  // extern "C"
