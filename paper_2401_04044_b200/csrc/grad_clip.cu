// Global gradient norm over a list of tensors, and clipping to it.
//
//   norm = sqrt(sum over tensors, elements of g^2),   out = g * min(1, max_norm / (norm + 1e-6))
//
// Bound by memory: the norm reads every element once, the scaling reads and writes it once.  Two launches: the
// scaling needs the whole norm.  The list travels as a kernel argument (no copy to the device, nothing to keep
// alive after the call), cut into launches of at most 960 tensors.  Every tensor is cut into chunks of 16384
// elements (4096 where the list has no more than 2^20: one tensor of 100000 elements 7.2 -> 5.2 us, of a million 7.8 -> 6.0,
// but fifty of 50000 9.5 -> 12.1) from its first 16-byte boundary on; block b takes chunks b, b + grid, ...  The scaling walks them from
// the last to the first: what the norm read last is still in L2, and the norm reads everything but its last 80 MB (of
// each launch) so that it does not stay there (508 -> 498 us for twelve 4096 x 11008 bf16 gradients, 505 on other cards; three
// passes at the rate of a copy take 495 us.  Streaming stores, or streaming loads in the scaling, cost 10 to 20 us more).
//
// Sums: the squares of one 16-byte vector in fp32 (8 bf16 or 4 fp32 values), from there on in fp64.  Where the fp32
// sum leaves [2^-60, 2^120) the vector is summed in fp64 instead, so that neither large nor small gradients leave
// the range.  That holds for a vector of zeros too (a list of nothing else: 133 instead of 103 us in the norm of eight 4096 x
// 11008 bf16 tensors; looking at the values first costs every other list 0.6 to 2 %).
// Every block writes one partial, the scaling kernel's blocks each add all of them in the same order.
#include <cstring>

#include "epilogue.cuh"
#include "internal.h"

namespace ffsp {
namespace clip {

constexpr int THREADS = 256;
constexpr int CHUNK = 16384, SMALL_CHUNK = 4096;      // elements; the small one where the list has at most SMALL_LIST
constexpr long long SMALL_LIST = 1 << 20;
constexpr int MAX_TENSORS = 960;     // per launch: what 32 KB of arguments hold
constexpr long long KEEP_BYTES = 80ll << 20;
constexpr int MAX_BLOCKS = 148 * 8; // per launch: 8 to each of a B200's SMs (the norm's are all resident, of the scaling's 3 at a time)

template <int CAP>
struct Table {
  const void* in[CAP];
  void* out[CAP];
  long long n[CAP];
  int first[CAP + 1];     // first chunk of each tensor
  unsigned char f32[CAP];
  unsigned short owner[2 * CAP];    // tensor of each chunk, where there are no more chunks than this (many small tensors:
                                    // every step of a search is a load that waits for the one before)
  int count;
  int chunk;              // elements of a chunk
  int keep;               // the norm reads this many chunks, the last ones, so that they stay in L2
};

__device__ __forceinline__ double block_sum(double v, double* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_down_sync(0xffffffffu, v, o);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  double t = 0.0;
  for (int i = 0; i < THREADS / 32; ++i) t += red[i];
  return t;
}

struct Piece {      // the elements [head, body, tail) of one chunk: body starts on 16 bytes and is whole vectors
  long long begin, body, body_end, end;
};

// Tensor of chunk c (from the list, or by binary search over the first chunks) and the chunk's range.
template <int CAP>
__device__ __forceinline__ int find_tensor(const Table<CAP>& t, int c) {
  if (t.first[t.count] <= 2 * CAP) return t.owner[c];
  int lo = 0, hi = t.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (t.first[mid] <= c) lo = mid; else hi = mid - 1;
  }
  return lo;
}
__device__ __forceinline__ Piece piece_of(const void* in, long long n, int es, int k, int chunk) {
  const int mis = static_cast<int>(reinterpret_cast<uintptr_t>(in) & 15u);
  long long head = mis ? (16 - mis) / es : 0;
  if (head > n) head = n;
  Piece p;
  p.body = head + static_cast<long long>(k) * chunk;
  p.begin = k == 0 ? 0 : p.body;
  p.end = p.body + chunk < n ? p.body + chunk : n;
  const int per = 16 / es;
  p.body_end = p.end > p.body ? p.body + (p.end - p.body) / per * per : p.body;
  return p;
}

template <int N>
__device__ __forceinline__ void add_squares(double& acc, const float* v) {
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < N; ++i) s = fmaf(v[i], v[i], s);
  if (s >= 8.673617e-19f && s < 1.329228e36f) {
    acc += static_cast<double>(s);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) acc += static_cast<double>(v[i]) * static_cast<double>(v[i]);
  }
}
__device__ __forceinline__ void unpack8(const uint4& q, float* v) {
  const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack4(const uint4& q, float* v) {
  v[0] = __uint_as_float(q.x); v[1] = __uint_as_float(q.y); v[2] = __uint_as_float(q.z); v[3] = __uint_as_float(q.w);
}
template <bool F32>
__device__ __forceinline__ float load1(const void* p, long long i) {
  return F32 ? static_cast<const float*>(p)[i] : __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}
template <bool F32>
__device__ __forceinline__ void store1(void* p, long long i, float v) {
  if (F32) static_cast<float*>(p)[i] = v;
  else static_cast<__nv_bfloat16*>(p)[i] = __float2bfloat16_rn(v);
}

template <bool F32, bool KEEP>
__device__ __forceinline__ void norm_piece(double& acc, const void* in, const Piece& p) {
  constexpr int ES = F32 ? 4 : 2, PER = 16 / ES, UNROLL = 4;
  const uint4* v = reinterpret_cast<const uint4*>(static_cast<const char*>(in) + p.body * ES);
  const int nv = static_cast<int>((p.body_end - p.body) / PER);
  for (int i0 = threadIdx.x; i0 < nv; i0 += UNROLL * THREADS) {
    uint4 q[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) q[u] = i0 + u * THREADS < nv ? (KEEP ? __ldg(v + i0 + u * THREADS) : __ldcs(v + i0 + u * THREADS)) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      float x[PER];
      if (F32) unpack4(q[u], x); else unpack8(q[u], x);
      add_squares<PER>(acc, x);
    }
  }
  // the elements before the first 16-byte boundary and those behind the last whole vector: at most 7 each
  const long long e = p.begin + threadIdx.x;
  if (e < p.body && e < p.end) { const float x = load1<F32>(in, e); add_squares<1>(acc, &x); }
  const long long f = p.body_end + threadIdx.x;
  if (f < p.end) { const float x = load1<F32>(in, f); add_squares<1>(acc, &x); }
}

template <bool F32>
__device__ __forceinline__ void scale_piece(const void* in, void* out, const Piece& p, float factor) {
  constexpr int ES = F32 ? 4 : 2, PER = 16 / ES, UNROLL = 4;
  const uint4* v = reinterpret_cast<const uint4*>(static_cast<const char*>(in) + p.body * ES);
  char* o = static_cast<char*>(out) + p.body * ES;
  const bool wide = (reinterpret_cast<uintptr_t>(o) & 15u) == 0;
  const int nv = static_cast<int>((p.body_end - p.body) / PER);
  for (int i0 = threadIdx.x; i0 < nv; i0 += UNROLL * THREADS) {
    uint4 q[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) if (i0 + u * THREADS < nv) q[u] = v[i0 + u * THREADS];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      const int i = i0 + u * THREADS;
      if (i >= nv) break;
      float x[PER];
      if (F32) unpack4(q[u], x); else unpack8(q[u], x);
#pragma unroll
      for (int j = 0; j < PER; ++j) x[j] *= factor;
      if (wide) {
        uint4 r;
        if (F32) {
          r = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
        } else {
          r = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[PER > 4 ? 4 : 0], x[PER > 4 ? 5 : 0]),
                         pack_bf16x2(x[PER > 4 ? 6 : 0], x[PER > 4 ? 7 : 0]));
        }
        reinterpret_cast<uint4*>(o)[i] = r;
      } else {
#pragma unroll
        for (int j = 0; j < PER; ++j) store1<F32>(o, static_cast<long long>(i) * PER + j, x[j]);
      }
    }
  }
  const long long e = p.begin + threadIdx.x;
  if (e < p.body && e < p.end) store1<F32>(out, e, load1<F32>(in, e) * factor);
  const long long f = p.body_end + threadIdx.x;
  if (f < p.end) store1<F32>(out, f, load1<F32>(in, f) * factor);
}

template <int CAP>
__global__ void __launch_bounds__(THREADS) grad_norm_kernel(const __grid_constant__ Table<CAP> t, double* partial) {
  __shared__ double red[THREADS / 32];
  pdl_wait();
  double acc = 0.0;
  const int chunks = t.first[t.count];
  for (int c = blockIdx.x; c < chunks; c += gridDim.x) {
    const int i = find_tensor(t, c);
    const bool f32 = t.f32[i] != 0;
    const Piece p = piece_of(t.in[i], t.n[i], f32 ? 4 : 2, c - t.first[i], t.chunk);
    const void* in = t.in[i];
    if (c >= chunks - t.keep) {
      if (f32) norm_piece<true, true>(acc, in, p); else norm_piece<false, true>(acc, in, p);
    } else {
      if (f32) norm_piece<true, false>(acc, in, p); else norm_piece<false, false>(acc, in, p);
    }
  }
  const double s = block_sum(acc, red);
  if (threadIdx.x == 0) partial[blockIdx.x] = s;
}

// The norm from all partials, the same sum in every block.
__device__ __forceinline__ float total_norm(const double* partial, int n, double* red) {
  double acc = 0.0;
  for (int i = threadIdx.x; i < n; i += THREADS) acc += __ldcg(partial + i);
  return static_cast<float>(sqrt(block_sum(acc, red)));
}

__global__ void __launch_bounds__(THREADS) norm_finish_kernel(const double* partial, int n, float* norm, int* status) {
  __shared__ double red[THREADS / 32];
  pdl_wait();
  const float v = total_norm(partial, n, red);
  if (threadIdx.x == 0) {
    *norm = v;
    if (!isfinite(v)) record_status(status, FFSPLIT_ERR_NONFINITE, 0, KID_CLIP);
  }
}

template <int CAP>
__global__ void __launch_bounds__(THREADS) grad_scale_kernel(const __grid_constant__ Table<CAP> t, const double* partial, int n,
                                                             float max_norm, float* norm, int* status) {
  __shared__ double red[THREADS / 32];
  pdl_wait();
  const float v = total_norm(partial, n, red);
  const bool finite = isfinite(v);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) {
    *norm = v;
    if (!finite) record_status(status, FFSPLIT_ERR_NONFINITE, 0, KID_CLIP);
  }
  const float factor = finite ? fminf(1.0f, max_norm / (v + 1e-6f)) : 1.0f;
  const int chunks = t.first[t.count];
  for (int c = chunks - 1 - static_cast<int>(blockIdx.x); c >= 0; c -= gridDim.x) {
    const int i = find_tensor(t, c);
    if (factor == 1.0f && t.in[i] == t.out[i]) continue;
    const bool f32 = t.f32[i] != 0;
    const Piece p = piece_of(t.in[i], t.n[i], f32 ? 4 : 2, c - t.first[i], t.chunk);
    if (f32) scale_piece<true>(t.in[i], t.out[i], p, factor); else scale_piece<false>(t.in[i], t.out[i], p, factor);
  }
}

}  // namespace clip

namespace {

int clip_launches(int count) { return count > 0 ? (count + clip::MAX_TENSORS - 1) / clip::MAX_TENSORS : 0; }

ffsplit_status check_grads(ffsplit_ctx* ctx, const ffsplit_grad_tensor* t, int count, bool scale, const float* norm) {
  ffsplit_status s = check_ctx(ctx, true);
  if (s != FFSPLIT_OK) return s;
  if (count < 0 || (count > 0 && !t) || !norm) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "NULL list or norm, or a negative count");
  if ((reinterpret_cast<uintptr_t>(norm) & 3u) != 0) return fail(ctx, FFSPLIT_ERR_ALIGN, "norm must be 4-byte aligned");
  long long chunks = 0;
  for (int i = 0; i < count; ++i) {
    if (t[i].n < 0) return fail(ctx, FFSPLIT_ERR_SHAPE, "a tensor has a negative length");
    if (t[i].dtype != FFSPLIT_F32 && t[i].dtype != FFSPLIT_BF16) return fail(ctx, FFSPLIT_ERR_DTYPE, "unknown dtype in the list");
    if (t[i].n == 0) continue;
    if (!t[i].in || (scale && !t[i].out)) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "NULL tensor in the list");
    const uintptr_t mask = elem_size(t[i].dtype) - 1;
    if ((reinterpret_cast<uintptr_t>(t[i].in) & mask) || (scale && (reinterpret_cast<uintptr_t>(t[i].out) & mask)))
      return fail(ctx, FFSPLIT_ERR_ALIGN, "a tensor is not aligned to its element size");
    if (t[i].n > (1ll << 40)) return fail(ctx, FFSPLIT_ERR_SHAPE, "a tensor of more than 2^40 elements");
    chunks += t[i].n / clip::CHUNK + 1;
    if (chunks > 0x40000000ll) return fail(ctx, FFSPLIT_ERR_SHAPE, "more than 2^44 elements in all");
  }
  if (kCtrlBytes + static_cast<size_t>(clip_launches(count)) * clip::MAX_BLOCKS * 8 > ctx->ws_bytes)
    return fail(ctx, FFSPLIT_ERR_BUFFER_TOO_SMALL, "workspace too small for this list (ffsplit_grad_workspace_size)");
  return FFSPLIT_OK;
}

// One launch's tensors, the empty ones left out.  Returns the number of chunks.
template <int CAP>
int fill_table(clip::Table<CAP>* tab, const ffsplit_grad_tensor* t, int n, int chunk, bool scale) {
  int chunks = 0;
  long long bytes = 0;
  tab->count = 0;
  tab->chunk = chunk;
  for (int i = 0; i < n; ++i) {
    if (t[i].n == 0) continue;
    const int j = tab->count++;
    const int es = static_cast<int>(elem_size(t[i].dtype));
    const int mis = static_cast<int>(reinterpret_cast<uintptr_t>(t[i].in) & 15u);
    const long long body = t[i].n - (mis ? (16 - mis) / es : 0);
    tab->in[j] = t[i].in;
    tab->out[j] = scale ? t[i].out : nullptr;
    tab->n[j] = t[i].n;
    tab->f32[j] = t[i].dtype == FFSPLIT_F32 ? 1 : 0;
    tab->first[j] = chunks;
    bytes += t[i].n * es;
    const int mine = body > chunk ? static_cast<int>((body + chunk - 1) / chunk) : 1;
    for (int c = chunks; c < chunks + mine && c < 2 * CAP; ++c) tab->owner[c] = static_cast<unsigned short>(j);
    chunks += mine;
  }
  tab->first[tab->count] = chunks;
  tab->keep = chunks > 0 ? static_cast<int>(clip::KEEP_BYTES * chunks / (bytes > 0 ? bytes : 1) < chunks ? clip::KEEP_BYTES * chunks / bytes : chunks) : 0;
  return chunks;
}

// phase 0: partials of the norm (returns their number in *blocks); phase 1: scaling
template <int CAP>
ffsplit_status clip_launch(ffsplit_ctx* ctx, const ffsplit_grad_tensor* t, int n, int phase, double* partial, int* blocks, int total,
                           float max_norm, float* norm, cudaStream_t st) {
  clip::Table<CAP> tab;
  long long elements = 0;
  for (int i = 0; i < n; ++i) elements += t[i].n;
  const int chunks = fill_table(&tab, t, n, elements <= clip::SMALL_LIST ? clip::SMALL_CHUNK : clip::CHUNK, phase == 1);
  const int grid = chunks < clip::MAX_BLOCKS ? (chunks > 0 ? chunks : 1) : clip::MAX_BLOCKS;
  cudaError_t e;
  if (phase == 0) {
    *blocks = grid;
    e = launch_pdl(clip::grad_norm_kernel<CAP>, dim3(grid), dim3(clip::THREADS), 0, st, tab, partial);
  } else {
    e = launch_pdl(clip::grad_scale_kernel<CAP>, dim3(grid), dim3(clip::THREADS), 0, st, tab, static_cast<const double*>(partial), total, max_norm, norm,
                   ctx->status());
  }
  ctx->launches++;
  return check_cuda(ctx, e, phase == 0 ? "grad_norm_kernel launch" : "grad_scale_kernel launch");
}

ffsplit_status clip_dispatch(ffsplit_ctx* ctx, const ffsplit_grad_tensor* t, int n, int phase, double* partial, int* blocks, int total,
                             float max_norm, float* norm, cudaStream_t st) {
  // the argument block is copied with every launch: a short list gets a short one
  if (n <= 32) return clip_launch<32>(ctx, t, n, phase, partial, blocks, total, max_norm, norm, st);
  if (n <= 256) return clip_launch<256>(ctx, t, n, phase, partial, blocks, total, max_norm, norm, st);
  if (n <= 512) return clip_launch<512>(ctx, t, n, phase, partial, blocks, total, max_norm, norm, st);
  return clip_launch<clip::MAX_TENSORS>(ctx, t, n, phase, partial, blocks, total, max_norm, norm, st);
}

// The partials of the whole list; *total of them.
ffsplit_status run_norm(ffsplit_ctx* ctx, const ffsplit_grad_tensor* t, int count, double* partial, int* total, cudaStream_t st) {
  ctx->score_prep.valid = false;   // the scoring buffers share the workspace
  *total = 0;
  for (int at = 0; at < count; at += clip::MAX_TENSORS) {
    const int n = count - at < clip::MAX_TENSORS ? count - at : clip::MAX_TENSORS;
    int blocks = 0;
    const ffsplit_status s = clip_dispatch(ctx, t + at, n, 0, partial + *total, &blocks, 0, 0.f, nullptr, st);
    if (s != FFSPLIT_OK) return s;
    *total += blocks;
  }
  return FFSPLIT_OK;
}

ffsplit_status finish_norm(ffsplit_ctx* ctx, const double* partial, int total, float* norm, cudaStream_t st) {
  const cudaError_t e = launch_pdl(clip::norm_finish_kernel, dim3(1), dim3(clip::THREADS), 0, st, partial, total, norm, ctx->status());
  ctx->launches++;
  return check_cuda(ctx, e, "norm_finish_kernel launch");
}

}  // namespace
}  // namespace ffsp

extern "C" {

ffsplit_status ffsplit_grad_workspace_size(int32_t count, size_t* bytes) {
  using namespace ffsp;
  if (!bytes || count < 0) return FFSPLIT_ERR_INVALID_ARG;
  *bytes = kCtrlBytes + static_cast<size_t>(clip_launches(count)) * clip::MAX_BLOCKS * 8;
  return FFSPLIT_OK;
}

ffsplit_status ffsplit_grad_norm(ffsplit_ctx* ctx, const ffsplit_grad_tensor* tensors, int32_t count, float* norm, void* stream) {
  using namespace ffsp;
  ffsplit_status s = check_grads(ctx, tensors, count, false, norm);
  if (s != FFSPLIT_OK) return s;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  double* partial = reinterpret_cast<double*>(ctx->ws + kCtrlBytes);
  int total = 0;
  if ((s = run_norm(ctx, tensors, count, partial, &total, st)) != FFSPLIT_OK) return s;
  return finish_norm(ctx, partial, total, norm, st);
}

ffsplit_status ffsplit_grad_clip(ffsplit_ctx* ctx, const ffsplit_grad_tensor* tensors, int32_t count, float max_norm, float* norm,
                                 void* stream) {
  using namespace ffsp;
  ffsplit_status s = check_grads(ctx, tensors, count, true, norm);
  if (s != FFSPLIT_OK) return s;
  if (!(max_norm >= 0.f)) return fail(ctx, FFSPLIT_ERR_INVALID_ARG, "max_norm must be >= 0");
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  double* partial = reinterpret_cast<double*>(ctx->ws + kCtrlBytes);
  int total = 0;
  if ((s = run_norm(ctx, tensors, count, partial, &total, st)) != FFSPLIT_OK) return s;
  if (count == 0) return finish_norm(ctx, partial, 0, norm, st);
  // the last tensors first: they are what the norm read last
  const int launches = clip_launches(count);
  for (int l = launches - 1; l >= 0; --l) {
    const int at = l * clip::MAX_TENSORS, n = count - at < clip::MAX_TENSORS ? count - at : clip::MAX_TENSORS;
    if ((s = clip_dispatch(ctx, tensors + at, n, 1, partial, nullptr, total, max_norm, l == 0 ? norm : nullptr, st)) != FFSPLIT_OK) return s;
  }
  return FFSPLIT_OK;
}

}  // extern "C"
