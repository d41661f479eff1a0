// Training a feed-forward layer: forward and backward from the row-major weights.
//
//   gated:  G = X W1, U = X W1u, H = silu(G) U, Y = H W2 + b2
//           dH = dY W2^T, dU = dH silu(G), dG = dH U silu'(G), dX = dG W1^T + dU W1u^T,
//           dW1 = X^T dG, dW1u = X^T dU, dW2 = H^T dY, db2 = sum_t dY
//   GELU:   Z = X W1 + b1, H = act(Z), Y = H W2 + b2; dZ = (dY W2^T) act'(Z), the rest likewise, db1 = sum_t dZ
//
// The products run on the tensor cores from the tensors where they lie (train_gemm.cu): two launches forward, two
// backward (dH with the activation's derivative; then every gradient that was asked for, as one launch).
// fp32 layers are first split into bf16 planes here; bf16 layers whose m is no multiple of 8 get W1 (W1u) copied to
// rows of 16 bytes, which TMA asks for.
#include <cstring>

#include "epilogue.cuh"
#include "train_gemm.h"

namespace ffsp {
namespace train {

// fp32 -> three bf16 planes (F32), or a copy of a bf16 matrix to rows of 128 bytes.  Bound by memory: a thread takes eight
// columns at a time, 16 bytes of every output.  Rows of an odd bf16 matrix start on any two bytes: five aligned words hold
// the eight values, shifted by half a word in every other row.
template <bool F32>
__global__ void __launch_bounds__(PREP_THREADS) prepare_kernel(const __grid_constant__ PrepArgs a) {
  constexpr int UNROLL = PREP_UNROLL<F32>;
  if (!a.apart) pdl_wait();
  int j = 0;
  while (j + 1 < a.n && static_cast<int>(blockIdx.x) >= a.job[j + 1].block0) ++j;
  const PrepJob& job = a.job[j];
  const long long first = static_cast<long long>(blockIdx.x - job.block0) * (PREP_THREADS * UNROLL) + threadIdx.x;
  const long long all = job.rows * job.octets;
  uint32_t w[UNROLL][F32 ? 8 : 5];
  long long at[UNROLL];
  bool half[UNROLL];
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    const long long i = first + u * PREP_THREADS;
    at[u] = -1;
    if (i >= all) continue;
    // (32-bit division where it will do: the 64-bit one takes longer than the copy)
    const long long row = all <= 0xffffffffll ? static_cast<unsigned>(i) / static_cast<unsigned>(job.octets) : i / job.octets;
    const int c = static_cast<int>(i - row * job.octets) * 8;
    at[u] = row * job.ld + c;
    if constexpr (F32) {
      const float* in = static_cast<const float*>(job.in) + row * job.cols + c;
      if (c + 8 <= job.cols && (reinterpret_cast<uintptr_t>(in) & 15u) == 0) {
        const uint4 x = __ldg(reinterpret_cast<const uint4*>(in)), y = __ldg(reinterpret_cast<const uint4*>(in) + 1);
        w[u][0] = x.x; w[u][1] = x.y; w[u][2] = x.z; w[u][3] = x.w;
        w[u][4] = y.x; w[u][5] = y.y; w[u][6] = y.z; w[u][7] = y.w;
      } else {
#pragma unroll
        for (int k = 0; k < 8; ++k) w[u][k] = c + k < job.cols ? __float_as_uint(__ldg(in + k)) : 0u;
      }
    } else {
      const unsigned short* in = static_cast<const unsigned short*>(job.in) + row * job.cols + c;
      half[u] = (reinterpret_cast<uintptr_t>(in) & 2u) != 0;
      const uint32_t* word = reinterpret_cast<const uint32_t*>(in - (half[u] ? 1 : 0));
      // the eight values may run into the next row (pad columns, which nobody reads), but not past the matrix
      const char* end = static_cast<const char*>(job.in) + job.rows * job.cols * 2;
      if (reinterpret_cast<const char*>(word + 5) <= end) {
#pragma unroll
        for (int k = 0; k < 5; ++k) w[u][k] = __ldg(word + k);
      } else {
        half[u] = false;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint32_t lo = c + 2 * k < job.cols ? __ldg(in + 2 * k) : 0, hi = c + 2 * k + 1 < job.cols ? __ldg(in + 2 * k + 1) : 0;
          w[u][k] = lo | hi << 16;
        }
        w[u][4] = 0u;
      }
    }
  }
#pragma unroll
  for (int u = 0; u < UNROLL; ++u) {
    if (at[u] < 0) continue;
    uint4* out = reinterpret_cast<uint4*>(job.out + at[u]);
    if constexpr (F32) {
      uint32_t v[4][3];
#pragma unroll
      for (int k = 0; k < 4; ++k) tg::split3_pair(__uint_as_float(w[u][2 * k]), __uint_as_float(w[u][2 * k + 1]), v[k]);
#pragma unroll
      for (int k = 0; k < 3; ++k) *reinterpret_cast<uint4*>(job.out + k * job.plane_stride + at[u]) = make_uint4(v[0][k], v[1][k], v[2][k], v[3][k]);
    } else {
      const uint32_t* x = w[u];
      *out = half[u] ? make_uint4(__funnelshift_r(x[0], x[1], 16), __funnelshift_r(x[1], x[2], 16), __funnelshift_r(x[2], x[3], 16),
                                  __funnelshift_r(x[3], x[4], 16))
                     : make_uint4(x[0], x[1], x[2], x[3]);
    }
  }
  if (a.apart) pdl_wait();
}

// Bias gradients: out[c] = sum over rows of in[r, c], in fp32 and in a fixed order.  db2 sums the rows of dY; for db1 the
// launch of dH leaves sums of dZ over 32 rows (in fp32, before dZ is rounded: rounded terms that cancel left up to ten times
// the error) and this adds those.  Bound by reading its input once.  A block takes 32 columns (four threads to a row, 64 rows
// at a time, eight of those in flight).  Where there are few columns and many rows the rows are cut: each block leaves a
// partial, and the block that is the last of its columns to arrive (a ticket, zero again afterwards) adds them in order.
struct SumJob {
  const void* in;          // bf16, or fp32 with f32_in; [rows, cols], pitch ld
  void* out;               // bf16, or fp32 with f32_out
  float* partial;          // [splits][cols]
  long long rows, ld, rows_per;
  int cols, f32_in, f32_out, splits, col_blocks, block0;
};
struct SumArgs {
  SumJob job[2];
  int n;
  int* tickets;            // one to a block of columns of a job whose rows are cut, SUM_TICKETS to a job
};
constexpr int SUM_COLS = 32, SUM_TICKETS = 512;
// Eight columns c .. c + 7 of one row.
template <bool F32>
__device__ __forceinline__ void add8(const SumJob& j, long long row, int c, float* s) {
  if constexpr (F32) {
    const float* p = static_cast<const float*>(j.in) + row * j.ld + c;
    if (c + 8 <= j.cols && (reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float4 v = __ldg(reinterpret_cast<const float4*>(p) + i);
        s[4 * i] += v.x; s[4 * i + 1] += v.y; s[4 * i + 2] += v.z; s[4 * i + 3] += v.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) if (c + i < j.cols) s[i] += __ldg(p + i);
    }
  } else {      // (the pitch of a bf16 matrix is a multiple of 8)
    const uint4 q = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(j.in) + row * j.ld + c));
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[2 * i] += __uint_as_float(w[i] << 16);
      s[2 * i + 1] += __uint_as_float(w[i] & 0xffff0000u);
    }
  }
}
// Rows begin, begin + 64, ... of eight columns.
template <bool F32>
__device__ __forceinline__ void sum_rows(const SumJob& j, long long begin, long long end, int c, float* s) {
  long long r = begin;
  for (; r + 448 < end; r += 512) {
#pragma unroll
    for (int k = 0; k < 8; ++k) add8<F32>(j, r + 64 * k, c, s);
  }
#pragma unroll
  for (int k = 0; k < 7; ++k)
    if (r + 64 * k < end) add8<F32>(j, r + 64 * k, c, s);
}
__global__ void __launch_bounds__(256) column_sum_kernel(const __grid_constant__ SumArgs a) {
  __shared__ float red[8][SUM_COLS];
  __shared__ int last;
  pdl_wait();
  const int second = a.n > 1 && static_cast<int>(blockIdx.x) >= a.job[1].block0 ? 1 : 0;
  const SumJob& j = a.job[second];
  const int b = blockIdx.x - j.block0, split = b / j.col_blocks, c0 = (b - split * j.col_blocks) * SUM_COLS;
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, mine = c0 + (lane & 3) * 8;
  const long long begin = split * j.rows_per, end = begin + j.rows_per < j.rows ? begin + j.rows_per : j.rows;
  float s[8] = {};
  if (mine < j.cols) {
    const long long r = begin + (threadIdx.x >> 2);
    if (j.f32_in) sum_rows<true>(j, r, end, mine, s);
    else sum_rows<false>(j, r, end, mine, s);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    s[i] += __shfl_xor_sync(0xffffffffu, s[i], 4);
    s[i] += __shfl_xor_sync(0xffffffffu, s[i], 8);
    s[i] += __shfl_xor_sync(0xffffffffu, s[i], 16);
    if (lane < 4) red[w][lane * 8 + i] = s[i];
  }
  __syncthreads();
  const int c = threadIdx.x & (SUM_COLS - 1);
  float t = red[0][c];
  for (int k = 1; k < 8; ++k) t += red[k][c];
  if (j.splits > 1) {
    if (threadIdx.x < SUM_COLS && c0 + c < j.cols) j.partial[static_cast<long long>(split) * j.cols + c0 + c] = t;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
      int* ticket = a.tickets + second * SUM_TICKETS + c0 / SUM_COLS;
      last = atomicAdd(ticket, 1) == j.splits - 1 ? 1 : 0;
      if (last) *ticket = 0;
    }
    __syncthreads();
    if (!last) return;
    __threadfence();
    if (threadIdx.x < SUM_COLS && c0 + c < j.cols) {
      t = 0.f;
#pragma unroll 8
      for (int k = 0; k < j.splits; ++k) t += __ldcg(j.partial + static_cast<long long>(k) * j.cols + c0 + c);
    }
  }
  if (threadIdx.x >= SUM_COLS || c0 + c >= j.cols) return;
  if (j.f32_out) static_cast<float*>(j.out)[c0 + c] = t;
  else static_cast<__nv_bfloat16*>(j.out)[c0 + c] = __float2bfloat16_rn(t);
}

tg::Matrix operand(PrepArgs* prep, int* blocks, bool f32, const void* p, long long rows, int cols, long long ld, void* copy) {
  if (!f32 && cols % 8 == 0) return {p, rows, cols, cols, rows * cols, 1};
  PrepJob& j = prep->job[prep->n++];
  j.in = p;
  j.out = static_cast<__nv_bfloat16*>(copy);
  j.rows = rows; j.cols = cols; j.ld = ld; j.plane_stride = rows * ld;
  j.octets = (cols + 7) / 8;
  j.block0 = *blocks;
  const int per = PREP_THREADS * (f32 ? PREP_UNROLL<true> : PREP_UNROLL<false>);
  *blocks += static_cast<int>((rows * j.octets + per - 1) / per);
  return {j.out, rows, cols, ld, j.plane_stride, f32 ? 3 : 1};
}
ffsplit_status launch_prepare(ffsplit_ctx* ctx, const PrepArgs& prep, int blocks, bool f32, cudaStream_t st) {
  if (prep.n == 0) return FFSPLIT_OK;
  const cudaError_t e = f32 ? launch_pdl(prepare_kernel<true>, dim3(blocks), dim3(PREP_THREADS), 0, st, prep)
                            : launch_pdl(prepare_kernel<false>, dim3(blocks), dim3(PREP_THREADS), 0, st, prep);
  ctx->launches++;
  return check_cuda(ctx, e, "train::prepare_kernel launch");
}

}  // namespace train

namespace {

inline size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// Row ranges of a column sum: enough blocks for two on every SM, but no fewer than 512 rows in each.  (More than one only
// where there are fewer than SUM_BLOCKS blocks of columns, so a job needs no more tickets than that.)
constexpr int SUM_BLOCKS = 2 * 148;
static_assert(SUM_BLOCKS <= train::SUM_TICKETS && 2 * train::SUM_TICKETS <= kMaxTicketTiles, "tickets of the column sums");
int sum_splits(long long rows, int cols) {
  const long long col_blocks = (cols + train::SUM_COLS - 1) / train::SUM_COLS;
  long long n = (SUM_BLOCKS + col_blocks - 1) / col_blocks;
  if (n > (rows + 511) / 512) n = (rows + 511) / 512;
  return static_cast<int>(n < 1 ? 1 : n);
}

// Size of what the forward pass keeps, and offsets of the workspace's buffers.  The rows of both are padded to a multiple
// of 64 elements (ldm for m, ldd for d), so that every row starts on 128 bytes; the pads are neither written to by
// whole chunks that matter nor read (the tensor maps end at m and d).
struct TrainLayout {
  long long ldm, ldd;
  size_t savedH, saved;
  size_t H, dG, dU, W1, W1u, W2, X, dY, sums, groups, parts, parts_bytes, end;
};
TrainLayout train_layout(const ffsplit_shape& s, long long T) {
  TrainLayout L;
  const bool gated = s.act == FFSPLIT_SWIGLU, f32 = s.dtype == FFSPLIT_F32;
  L.ldm = round_up_ll(s.m, 64);
  L.ldd = round_up_ll(s.d, 64);
  const size_t hidden = static_cast<size_t>(T) * L.ldm;
  const size_t planes = f32 ? 3 : 1;
  // H is kept as well: writing it a second time costs the backward pass more than reading it (an SM writes 18 bytes a
  // nanosecond, and the epilogue of dH is bound by that)
  L.savedH = up256(tg::kept_bytes(T, L.ldm, gated, f32));
  L.saved = L.savedH + up256(hidden * 2 * planes);
  size_t off = 0;
  L.H = off;                                   // (a forward pass that keeps nothing)
  L.dG = off; off = up256(off + hidden * 2 * planes);
  L.dU = off; off = up256(off + (gated ? hidden * 2 * planes : 0));
  const bool copy_w1 = f32 || s.m % 8 != 0;
  const size_t w1 = copy_w1 ? static_cast<size_t>(s.d) * L.ldm * 2 * planes : 0;
  L.W1 = off;  off = up256(off + w1);
  L.W1u = off; off = up256(off + (gated ? w1 : 0));
  L.W2 = off;  off = up256(off + (f32 ? static_cast<size_t>(s.m) * L.ldd * 6 : 0));
  const size_t tokens = f32 ? static_cast<size_t>(T) * L.ldd * 6 : 0;
  L.X = off;  off = up256(off + tokens);
  L.dY = off; off = up256(off + tokens);
  L.sums = off; off = up256(off + 4 * (static_cast<size_t>(sum_splits(T, s.m)) * s.m + static_cast<size_t>(sum_splits(T, s.d)) * s.d));
  // partials of products that are cut along K: that pays where their outputs are small, and is bounded at 32 MB
  const size_t a = static_cast<size_t>(T) * (2 * L.ldm > L.ldd ? 2 * L.ldm : L.ldd), b = static_cast<size_t>(L.ldm) * L.ldd;
  const size_t want = 64 * (a > b ? a : b);
  L.parts_bytes = up256(want < (32u << 20) ? want : (32u << 20));
  L.parts = off; off += L.parts_bytes;
  // sums of dZ over groups of rows, or every row of it where that launch is joined: its partials, at least two times these
  // rows, are then no more than parts_bytes
  const size_t rows = static_cast<size_t>((T + tg::COL_SUM_ROWS - 1) / tg::COL_SUM_ROWS), whole = static_cast<size_t>(T) * L.ldm * 4;
  L.groups = off;
  if (!gated) off = up256(off + (whole <= L.parts_bytes / 2 ? whole : rows * L.ldm * 4));
  L.end = off;
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

// The operands of a pass: the caller's tensors, or their planes (or padded copies) in the workspace.
struct Pass {
  ffsplit_ctx* ctx;
  ffsplit_shape s;
  TrainLayout L;
  long long T;
  char* ws;
  cudaStream_t st;
  train::PrepArgs prep;
  int prep_blocks = 0;

  Pass(ffsplit_ctx* c, const ffsplit_shape& shape, long long tokens, cudaStream_t stream)
      : ctx(c), s(shape), L(train_layout(shape, tokens)), T(tokens), ws(c->ws + kCtrlBytes), st(stream) {
    std::memset(&prep, 0, sizeof(prep));
    ctx->score_prep.valid = false;   // the scoring buffers share the workspace
  }
  bool f32() const { return s.dtype == FFSPLIT_F32; }
  bool gated() const { return s.act == FFSPLIT_SWIGLU; }

  // A caller's tensor [rows, cols]: as it is, or as copied to `at` by the preparation launch.
  tg::Matrix tensor(const void* p, long long rows, int cols, long long ld, size_t at) {
    return train::operand(&prep, &prep_blocks, f32(), p, rows, cols, ld, ws + at);
  }
  tg::Matrix hidden(const void* at) const { return {at, T, s.m, L.ldm, T * L.ldm, f32() ? 3 : 1}; }
  tg::Hidden buffers(char* saved) const {
    tg::Hidden h;
    h.kept = saved;
    h.H = reinterpret_cast<__nv_bfloat16*>(saved ? saved + L.savedH : ws + L.H);
    h.dG = reinterpret_cast<__nv_bfloat16*>(ws + L.dG);
    h.dU = reinterpret_cast<__nv_bfloat16*>(ws + L.dU);
    h.ldm = L.ldm;
    h.plane_stride = T * L.ldm;
    h.col_sums = nullptr;
    return h;
  }
  ffsplit_status prepare() { return train::launch_prepare(ctx, prep, prep_blocks, f32(), st); }
};

tg::Product product(const tg::Matrix& a, int a_mn, const tg::Matrix& b, int b_mn, long long M, int N, long long K) {
  tg::Product g;
  std::memset(&g, 0, sizeof(g));
  g.a[0] = a; g.b[0] = b;
  g.pairs = 1;
  g.a_mn = a_mn; g.b_mn = b_mn;
  g.M = M; g.N = N; g.K = K;
  return g;
}

ffsplit_status run_train_forward(ffsplit_ctx* ctx, const ffsplit_shape& s, const ffsplit_weights& w, const void* X, long long T,
                                 char* saved, void* Y, cudaStream_t st) {
  Pass p(ctx, s, T, st);
  const int d = s.d, m = s.m;
  const tg::Matrix x = p.tensor(X, T, d, p.L.ldd, p.L.X), w1 = p.tensor(w.W1, d, m, p.L.ldm, p.L.W1),
                   w2 = p.tensor(w.W2, m, d, p.L.ldd, p.L.W2);
  tg::Product g = product(x, 0, w1, 1, T, m, d);
  if (p.gated()) g.b[1] = p.tensor(w.W1u, d, m, p.L.ldm, p.L.W1u);
  g.bias = w.b1;
  ffsplit_status r;
  if ((r = p.prepare()) != FFSPLIT_OK) return r;
  const tg::Hidden h = p.buffers(saved);
  if ((r = tg::launch(ctx, p.gated() ? tg::FORWARD_GATED : tg::FORWARD_ACT, s.act, p.f32(), &g, 1, h, p.ws + p.L.parts, p.L.parts_bytes, st)) != FFSPLIT_OK) return r;
  g = product(p.hidden(h.H), 0, w2, 1, T, d, m);
  g.C = Y; g.ldc = d; g.bias = w.b2;
  g.b_ready = 1;      // W2, or its planes: complete before the launch of the first product began to write
  return tg::launch(ctx, tg::PLAIN, s.act, p.f32(), &g, 1, h, p.ws + p.L.parts, p.L.parts_bytes, st);
}

ffsplit_status run_train_backward(ffsplit_ctx* ctx, const ffsplit_shape& s, const ffsplit_weights& w, const void* X, long long T,
                                  const char* saved, const void* dY, const ffsplit_train_grads& grads, cudaStream_t st) {
  Pass p(ctx, s, T, st);
  const int d = s.d, m = s.m;
  const bool inner = grads.dX || grads.dW1 || grads.dW1u || grads.db1 || grads.dW2;   // anything that needs dH or H
  tg::Hidden h = p.buffers(const_cast<char*>(saved));
  if (grads.db1) h.col_sums = reinterpret_cast<float*>(p.ws + p.L.groups);
  bool joined = false;
  const tg::Matrix H = p.hidden(h.H), dG = p.hidden(h.dG), dU = p.hidden(h.dU);
  tg::Product out[4];
  int n = 0;
  ffsplit_status r;
  if (inner) {
    const tg::Matrix dy = p.tensor(dY, T, d, p.L.ldd, p.L.dY), w2 = p.tensor(w.W2, m, d, p.L.ldd, p.L.W2);
    {
      tg::Product& g = out[n++] = product(dG, 0, grads.dX ? p.tensor(w.W1, d, m, p.L.ldm, p.L.W1) : tg::Matrix{}, 0, T, d, m);
      if (p.gated()) {
        g.pairs = 2;
        g.a[1] = dU;
        if (grads.dX) g.b[1] = p.tensor(w.W1u, d, m, p.L.ldm, p.L.W1u);
      }
      g.C = grads.dX; g.ldc = d;
    }
    const tg::Matrix x = grads.dW1 || grads.dW1u ? p.tensor(X, T, d, p.L.ldd, p.L.X) : tg::Matrix{};
    {
      tg::Product& g = out[n++] = product(x, 1, dG, 1, d, m, T);
      g.C = grads.dW1; g.ldc = m;
    }
    if (p.gated()) {
      tg::Product& g = out[n++] = product(x, 1, dU, 1, d, m, T);
      g.C = grads.dW1u; g.ldc = m;
    }
    {
      tg::Product& g = out[n++] = product(H, 1, dy, 1, m, d, T);
      g.C = grads.dW2; g.ldc = d;
    }
    if ((r = p.prepare()) != FFSPLIT_OK) return r;
    const tg::Product g = product(dy, 0, w2, 0, T, m, d);
    if ((r = tg::launch(ctx, p.gated() ? tg::BACKWARD_GATED : tg::BACKWARD_ACT, s.act, p.f32(), &g, 1, h, p.ws + p.L.parts, p.L.parts_bytes, st,
                        &joined)) != FFSPLIT_OK)
      return r;
    if ((grads.dX || grads.dW1 || grads.dW1u || grads.dW2) && (r = tg::launch(ctx, tg::PLAIN, s.act, p.f32(), out, n, h, p.ws + p.L.parts, p.L.parts_bytes, st)) != FFSPLIT_OK) return r;
  }
  if (grads.db1 || grads.db2) {
    train::SumArgs a;
    std::memset(&a, 0, sizeof(a));
    int blocks = 0;
    float* partial = reinterpret_cast<float*>(p.ws + p.L.sums);
    const auto add = [&](const void* in, bool f32_in, void* to, long long rows, long long ld, int n_cols) {
      train::SumJob& j = a.job[a.n++];
      j.in = in; j.out = to; j.partial = partial;
      j.rows = rows; j.ld = ld;
      j.cols = n_cols; j.f32_in = f32_in ? 1 : 0; j.f32_out = p.f32() ? 1 : 0;
      j.col_blocks = (n_cols + train::SUM_COLS - 1) / train::SUM_COLS;
      j.splits = sum_splits(rows, n_cols);
      j.rows_per = (rows + j.splits - 1) / j.splits;
      j.block0 = blocks;
      blocks += j.splits * j.col_blocks;
      partial += static_cast<size_t>(j.splits) * n_cols;
    };
    if (grads.db1) add(h.col_sums, true, grads.db1, joined ? T : (T + tg::COL_SUM_ROWS - 1) / tg::COL_SUM_ROWS, p.L.ldm, m);
    if (grads.db2) add(dY, p.f32(), grads.db2, T, d, d);
    a.tickets = ctx->tickets();
    const cudaError_t e = launch_pdl(train::column_sum_kernel, dim3(blocks), dim3(256), 0, st, a);
    ctx->launches++;
    return check_cuda(ctx, e, "column_sum_kernel launch");
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
  return run_train_forward(ctx, *shape, *weights, X, T, static_cast<char*>(saved), Y, static_cast<cudaStream_t>(stream));
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
  return run_train_backward(ctx, *shape, *weights, X, T, static_cast<const char*>(saved), dY, *grads, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
