// The products of a training pass, as train_gemm.cu runs them.  Not part of the public ABI.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>

#include "internal.h"

namespace ffsp {
namespace tg {

// One operand of a product: `planes` bf16 matrices [rows, cols] with pitch ld, plane_stride elements apart.  A bf16
// tensor is one plane; an fp32 tensor is three, whose sum it is to fp32 accuracy (split3() below).
struct Matrix {
  const void* p;
  long long rows, cols, ld, plane_stride;
  int planes;
};

enum Mode : int {
  PLAIN = 0,            // C = sum of the pairs' products (+ bias)
  FORWARD_GATED = 1,    // G = A0 B0, U = A0 B1: keeps G, U; H = silu(G) U
  FORWARD_ACT = 2,      // Z = A0 B0 + bias: keeps Z; H = act(Z)
  BACKWARD_GATED = 3,   // dH = A0 B0: dU = dH silu(G), dG = dH U silu'(G)
  BACKWARD_ACT = 4      // dH = A0 B0: dZ = dH act'(Z)
};

// C [M, N] = sum over pairs of A_i [M, K] B_i [K, N].  a_mn: A lies in memory as [K, M] rows (M runs along memory),
// else as [M, K]; b_mn: B as [K, N], else as [N, K].
struct Product {
  Matrix a[2], b[2];
  int pairs;
  int a_mn, b_mn;
  long long M, K;
  int N;
  void* C;               // PLAIN: bf16 or fp32 output; nullptr: not wanted.  Such a product is not run, but counts when
                         // the launch is planned: a gradient has the same bits whichever others are asked for
  long long ldc;
  const void* bias;      // [N], the layer's type, or nullptr
  int b_ready;           // the kernel before this launch in the stream does not write B
  int apart;             // ... writes nothing that this launch reads or writes, and reads nothing that it writes, and waited itself
                         // for those before it (one product): they run side by side, and whoever follows finds both done
};

// What the activation's epilogue reads and writes: what the forward pass keeps (see Kept in train_gemm.cu; nullptr:
// nothing) and the bf16 planes of H, dG (dZ) and dU, [T, ldm] each.
struct Hidden {
  void* kept;
  __nv_bfloat16 *H, *dG, *dU;
  long long ldm, plane_stride;
  float* col_sums;       // BACKWARD_ACT, or nullptr: sums of dZ before it is rounded, [row groups][ldm], for db1
};
constexpr int COL_SUM_ROWS = 32;   // rows of a group; one row where the launch was joined
// Bytes of what is kept of G and U, or of Z: 20 bits each, all 32 in fp32 layers; whole blocks of 32 rows.
inline size_t kept_bytes(long long T, long long ldm, bool gated, bool f32) {
  return static_cast<size_t>((T + 31) / 32 * 32) * ldm * (gated ? 2 : 1) * (f32 ? 8 : 5) / 2;
}

// More terms of a bf16 PLAIN product, of few k-blocks and different for each tile of 256 rows: C += Q_e F_i for what the tile's
// list names, i in the lower half of a word and e in the upper one.  Q_e of tile m is number m * most + e of [256, pitch] (pitch
// 64 or 128; columns from `rank` rounded up to 16 on are not read), rows that do not use it are zeros.  F lies along the axes of
// the product's own B.
struct Extension {
  const __nv_bfloat16* Q;
  long long entries;       // there is room for
  int pitch, most, rank;
  Matrix F;                // [planes][rows][cols], one plane to an i
  const int *count, *list; // [tiles], [tiles][most]
};

#ifdef __CUDACC__
// x = x0 + x1 + x2 with bf16 terms; non-finite values stay in x0 alone, and a finite x0 does not round to infinity.
__device__ __forceinline__ void split3(float x, float* o) {
  float a = __bfloat162float(__float2bfloat16_rn(x));
  if ((__float_as_uint(a) & 0x7f800000u) == 0x7f800000u) {
    const bool finite = (__float_as_uint(x) & 0x7f800000u) != 0x7f800000u;
    if (!finite) {
      o[0] = a; o[1] = 0.f; o[2] = 0.f;
      return;
    }
    a = __uint_as_float(__float_as_uint(x) & 0xffff0000u);
  }
  const float r = x - a, b = __bfloat162float(__float2bfloat16_rn(r));
  o[0] = a; o[1] = b; o[2] = r - b;
}
// Two values at once: w[k] holds the k-th term of both.
__device__ __forceinline__ uint32_t bf16_pair(float x, float y) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&t);
}
__device__ __forceinline__ void split3_pair(float x, float y, uint32_t* w) {
  if (fabsf(x) + fabsf(y) < 3.3e38f) {      // (false for NaN)
    w[0] = bf16_pair(x, y);
    const float rx = x - __uint_as_float(w[0] << 16), ry = y - __uint_as_float(w[0] & 0xffff0000u);
    w[1] = bf16_pair(rx, ry);
    w[2] = bf16_pair(rx - __uint_as_float(w[1] << 16), ry - __uint_as_float(w[1] & 0xffff0000u));
  } else {
    float p[3], q[3];
    split3(x, p);
    split3(y, q);
#pragma unroll
    for (int k = 0; k < 3; ++k) w[k] = bf16_pair(p[k], q[k]);
  }
}
#endif

// Up to four PLAIN products (or one of the other modes) as one launch, or as two where K is cut.  f32: three-plane
// operands and fp32 outputs.  partials: scratch for the fp32 partials of products that are cut along K.
// joined (may be nullptr): whether that was done.
ffsplit_status launch(ffsplit_ctx* ctx, Mode mode, int act, bool f32, const Product* products, int n, const Hidden& hidden, char* partials,
                      size_t partial_room, cudaStream_t st, bool* joined = nullptr, const Extension* extension = nullptr);

}  // namespace tg

// Operands that the tensor maps cannot take as they lie are copied first, one launch for all of a call (train.cu).
namespace train {

constexpr int MAX_JOBS = 5;
struct PrepJob {
  const void* in;          // [rows, cols], pitch cols
  __nv_bfloat16* out;      // pitch ld, a multiple of 64; fp32: three planes
  long long rows, ld, plane_stride;
  int cols, octets;        // octets of columns in a row
  int block0;              // first block
};
struct PrepArgs {
  PrepJob job[MAX_JOBS];
  int n;
  int apart;             // the launch before neither gives nor takes these tensors, and waited itself: waited for at the end
};
constexpr int PREP_THREADS = 256;
template <bool F32> constexpr int PREP_UNROLL = F32 ? 2 : 4;


// A caller's tensor [rows, cols] as an operand: where it lies, or as the preparation launch copies it to `copy` (pitch ld).
tg::Matrix operand(PrepArgs* prep, int* blocks, bool f32, const void* p, long long rows, int cols, long long ld, void* copy);
ffsplit_status launch_prepare(ffsplit_ctx* ctx, const PrepArgs& prep, int blocks, bool f32, cudaStream_t st);

}  // namespace train
}  // namespace ffsp
