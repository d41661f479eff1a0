// The matrix products of a training pass on the tensor cores, weights and activations where they lie.
//
//   C [M, N] = sum over pairs, k of A_i[m, k] B_i[k, n]
//
// A training pass multiplies the same row-major tensors along either of their axes (X W1, but X^T dG; H W2, but
// dY W2^T), and the weights change with every step, so nothing is transposed or packed beforehand: an operand whose
// contraction runs along memory goes to the tensor cores as a K-major tile, any other as an MN-major one.  Which of
// the two it is, is a bit of the instruction descriptor and the shape of the TMA box, both chosen at run time.
//
// One persistent pair of CTAs (two SMs, cta_group::2) per 256 x 256 tile: each CTA stages 128 rows of A and 128 rows
// of B per 64-deep k-block (32 KB) by TMA in a ring of six (more where there are fewer rows or columns), rank 0 issues the
// MMAs for both, and each CTA finishes the 128 accumulator rows in its own tensor memory.  Two accumulators of 256 columns: a tile's epilogue runs under the
// next tile's MMAs.  A gated tile is 256 x 128: rank 0 stages the 128 columns of W1, rank 1 those of W1u, so that
// every accumulator row holds G next to U and the product H leaves from the same registers.
//
// bf16 layers: sums are fp32; H, dG (dZ) and dU are rounded to bf16 between two products, because they are operands of the
// next one and the tensor cores take both operands in one type (a second plane would double that product).  G, U and Z are
// kept in 20 bits, see Kept.  Outputs are 2.3e-3 off 64 bits that way; the rounding of the output alone is 1.7e-3.
//
// fp32 layers: every fp32 matrix is split into three bf16 planes (x0 = bf16(x), x1 = bf16(x - x0), ...: 24 significant
// bits), and the six products of planes (i, j), i + j <= 2, are accumulated as six runs over K, the smallest first.
// What is dropped is below 2^-24 of a term.  The tensor cores cut their running sums to 24 bits instead of rounding them
// (measured: a bias of about 3e-8 of the sum per MMA, 8e-6 in all at K = 2752), so the sum is taken out of tensor memory
// every PROMOTE k-blocks of the largest product and added up in registers; the five small products before it (2^-8 of
// the sum and less) need no such care.
//
// Few tiles, long sums (few tokens, small layers): a tile's K range is cut into `split` units that leave fp32 partials, and
// a second launch (join_kernel) adds them in order and does what the epilogue would have done; or the tile is halved to
// 256 x 128.  plan() weighs both.
//
// Warp roles: 0 TMA producer (both CTAs), 1 MMA issuer (rank 0), from 2 on (fp32 layers: from 4 on) epilogue, four lane
// quarters x two or four groups of columns.
// Every wait is bounded; on expiry the CTA records FFSPLIT_ERR_TIMEOUT, lets its copies and MMAs land and returns.
#include <cstring>

#include "epilogue.cuh"
#include "ptx.cuh"
#include "train_gemm.h"

namespace ffsp {
namespace tg {

constexpr int CTA_M = 128, TILE_M = 256, TILE_N = 256, BLOCK_K = 64;
constexpr int MAX_STAGES = 10;
constexpr int BLOCK64_BYTES = 64 * BLOCK_K * 2;      // 64 x 64 elements: MN-major tiles are staged in two of these
constexpr int TMEM_COLS = 512;
constexpr int BAR_BYTES = 256;
constexpr int MAX_SMEM = 232448;
// Epilogue warps and the output staging of each.  The activations' epilogues need many warps to hide their latencies (dH of
// a 4096 x 11008 gated layer, 2048 tokens: 154 us with 8, 135 us with 16); plain outputs do not, and leave the tensor cores
// more of the power and of the issue slots with 8 (the gradients of a 5120 x 20480 layer: 1.68 ms, 1.80 ms with 16).
// fp32 sums take 128 registers of a thread; fp32 activations write straight to memory.
template <int MODE, bool F32> constexpr int EPI_WARPS = F32 || MODE == PLAIN ? 8 : 16;
template <int MODE, bool F32> constexpr int OUT_BYTES = MODE == PLAIN ? 4096 : F32 ? 0 : MODE == BACKWARD_GATED ? 4096 : 2048;
// The first epilogue warp.  fp32 kernels keep it on a warpgroup's boundary, so that registers can move from the group of the
// producer and the MMA issuer to the epilogue's two: with 168 for every thread the sums were spilled, and with the ring
// taking nearly all of the SM's memory a spill goes to L2 (380 -> 342 us for a 1024 x 2752 gated layer, 1024 tokens; of dH's
// epilogues 116 bytes a thread still spill where the layer is gated, 16 in GELU layers).  384 threads start with 168 registers
// each (64512); 128 of them go down to 56 and 256 up to 224: 7168 + 57344 = 64512.
template <bool F32> constexpr int FIRST_EPI = F32 ? 4 : 2;
constexpr int START_REGS = 168, ROLE_REGS = 56, EPI_REGS = 224;
static_assert(ROLE_REGS * 128 + EPI_REGS * 256 <= START_REGS * 384, "a split above what the block starts with waits forever");
template <int MODE, bool F32> constexpr int THREADS = 32 * (EPI_WARPS<MODE, F32> + FIRST_EPI<F32>);
// What is left for the ring of stages.  A stage holds a_rows rows of A and half a tile's columns of B, 128 bytes each.
template <int MODE, bool F32>
constexpr int RING_BYTES = (MAX_SMEM - 1024 - BAR_BYTES - EPI_WARPS<MODE, F32> * OUT_BYTES<MODE, F32>) / 1024 * 1024;
constexpr int MAX_PRODUCTS = 4;
// k-blocks: 8 MMAs, 2.4e-7 at most.  (Of a 1024 x 2752 gated layer on 1024 tokens 4.0e-7 is left and a pass takes 364 us; 4
// k-blocks: 7.4e-7 and 333 us.  A 256 x 1024 layer on 128 tokens: 2.9e-7 and 87 us against 5.3e-7 and 81; plain fp32 sums 4.2e-7.)
constexpr int PROMOTE = 2;

struct Unit {
  int prod, m_blk, n_blk;
  int split, k0, k1;     // k-blocks [k0, k1), counted over all runs
};

struct DevProduct {
  CUtensorMap a[2], b[2], c;
  long long M;
  int N, kb;             // k-blocks per run
  int runs, pairs;       // runs over K: pairs x (1, or the 6 products of planes)
  int a_mn, b_mn;
  int a_rows;            // rows of A that a CTA's box holds: 128, or (K-major, one tile) what M needs
  int tiles_m, tiles_n, panel_m;
  int unit0;             // first unit of this product
  int splits, per;       // ranges of K, and k-blocks in each (the last one may be shorter)
  float* partial;        // splits > 1: [splits][M][ldp] fp32; the gated forward pass keeps U at column ldp / 2
  long long ldp;
  void* C;
  long long ldc;
  const void* bias;
  int ragged;            // rows of C do not all start on 16 bytes
};

template <int CAP>
struct Params {
  DevProduct prod[CAP];
  int n_prod;
  int tile_n;            // accumulator columns of a tile, 256 or 128
  int stages, a_bytes, stage_bytes;   // the ring
  int units;             // work units of all products, the products with the longer runs first
  // Units are dealt to the clusters in turn.  The first `heavy` ones (the product with the longest tiles) may leave the
  // clusters from `short_from` on one tile short: `extra` of the following units go to those clusters first.
  int heavy, short_from, extra;
  int early;             // B of the first stages is loaded before the wait for the kernel before
  int apart;             // that wait is at the end
  int act;
  Hidden hid;
  CUtensorMap hid_map[2];  // bf16 layers: H, or dG (dZ) and dU, as outputs
  int box_cols;            // columns of an output box
  int* status;
};

// The same with an extension (PLAIN, bf16, one product).
struct ExtendedParams : Params<1> {
  CUtensorMap q, f;
  const int *count, *list;
  int most, blocks, steps; // k-blocks of an entry, and MMAs of 16
};
template <int CAP, bool EXTENDED> struct KernelParams { typedef Params<CAP> type; };
template <> struct KernelParams<1, true> { typedef ExtendedParams type; };
// How many entries follow the last k-block of a unit.
__device__ __forceinline__ int entries_of(const ExtendedParams& p, const Unit& t) {
  return t.k1 == p.prod[0].runs * p.prod[0].kb ? __ldcg(p.count + t.m_blk) : 0;
}

// Units of one cluster in order.
struct Walk {
  int c, C, next, phase, given;
  __device__ __forceinline__ Walk() : c(blockIdx.x >> 1), C(gridDim.x >> 1), next(blockIdx.x >> 1), phase(0), given(0) {}
  // next unit, or -1
  template <int CAP>
  __device__ __forceinline__ int take(const Params<CAP>& p) {
    if (phase == 0) {
      if (next < p.heavy) {
        const int u = next;
        next += C;
        return u;
      }
      phase = 1;
    }
    const int narrow = C - p.short_from;       // clusters that are one heavy tile short
    if (phase == 1) {
      if (c >= p.short_from && given < p.extra) {
        const int u = p.heavy + (c - p.short_from) + given * narrow;
        ++given;
        return u;                              // extra * narrow <= units - heavy, by construction
      }
      phase = 2;
      int turn = c - p.short_from;             // the short clusters first again
      if (turn < 0) turn += C;
      next = p.heavy + p.extra * narrow + turn;
    }
    if (next >= p.units) return -1;
    const int u = next;
    next += C;
    return u;
  }
};

template <int CAP>
__device__ __forceinline__ Unit find_unit(const Params<CAP>& p, int u) {
  Unit r;
  r.prod = 0;
  while (CAP > 1 && r.prod + 1 < p.n_prod && u >= p.prod[r.prod + 1].unit0) ++r.prod;
  const DevProduct& d = p.prod[r.prod];
  const int tiles = d.tiles_m * d.tiles_n;
  r.split = (u - d.unit0) / tiles;
  r.k0 = r.split * d.per;
  r.k1 = r.k0 + d.per < d.runs * d.kb ? r.k0 + d.per : d.runs * d.kb;
  const int tile = u - d.unit0 - r.split * tiles;
  const int per_panel = d.panel_m * d.tiles_n;
  const int panel = tile / per_panel, in_panel = tile - panel * per_panel, m0 = panel * d.panel_m;
  const int h = d.tiles_m - m0 < d.panel_m ? d.tiles_m - m0 : d.panel_m;
  r.n_blk = in_panel / h;
  r.m_blk = m0 + (in_panel - r.n_blk * h);
  return r;
}

// Planes of run r: the pairs of one product of planes one after the other, small products first.
template <bool F32>
__device__ __forceinline__ void run_planes(const DevProduct& d, int run, int* pair, int* pa, int* pb) {
  if (!F32) {
    *pair = run; *pa = 0; *pb = 0;
    return;
  }
  const int combo = run / d.pairs;
  *pair = run - combo * d.pairs;
  // (0,2) (1,1) (2,0) (0,1) (1,0) (0,0)
  *pa = (0x012010 >> (4 * (5 - combo))) & 0xF;
  *pb = (0x001012 >> (4 * combo)) & 0xF;
}

// fp32 layers: end of the part of a unit's sum that begins at k-block `begin`.
__device__ __forceinline__ int part_end(const DevProduct& d, const Unit& t, int begin) {
  const int large = (d.runs - d.pairs) * d.kb;       // the last `pairs` runs are the largest product
  const int end = (begin > large ? begin : large) + PROMOTE;
  return end < t.k1 ? end : t.k1;
}

// ---------------------------------------------------------------------------------------------- activations
// Values go through in pairs (the packed fp32 instructions of sm_100): the epilogue of a 256 x 256 tile has 32768 values
// per SM, and at one instruction issued per clock and scheduler every instruction per value costs 0.14 us.  bf16 layers
// use the hardware's exponential and reciprocal (a few 2^-22 of the value) and for the tail of Phi a polynomial whose error
// is absolute (1.5e-7: below bf16's 2^-9 of Phi down to z = -5).  fp32 layers use the library functions, whose errors are
// relative on both sides: with the polynomial GELU(z) was 5e-5 off at z = -3 and 5e-4 at z = -4, and neurons that are mostly
// negative had their whole share of dW1, db1 and dW2 off by that (GELU layers of 256 x 1024, 128 tokens: 84 us a pass with
// the polynomial, 87 us; 1007 x 6196, 786 tokens: 545 and 560 us; gated layers the same).
__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }
__device__ __forceinline__ float2 ex2(float2 x) {
  float2 r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(x.x));
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(x.y));
  return r;
}
__device__ __forceinline__ float2 rcp(float2 x) {
  float2 r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.x) : "f"(x.x));
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r.y) : "f"(x.y));
  return r;
}
// 1 / (1 + exp(-z))
template <bool F32>
__device__ __forceinline__ float2 sigmoid2(float2 z) {
  if constexpr (F32) return make_float2(__fdividef(1.0f, 1.0f + expf(-z.x)), __fdividef(1.0f, 1.0f + expf(-z.y)));     // 2 ulp
  return rcp(__fadd2_rn(ex2(__fmul2_rn(z, both(-1.4426950408889634f))), both(1.0f)));
}
// GELU and, where asked for, its slope.
template <bool F32, bool SLOPE>
__device__ __forceinline__ void gelu2(float2 z, int act, float2* value, float2* slope) {
  if (act == FFSPLIT_GELU_ERF) {
    // z Phi(z), Phi + z phi
    float2 below, density;
    if constexpr (F32) {
      below = make_float2(0.5f * erfcf(-0.70710678118654752f * z.x), 0.5f * erfcf(-0.70710678118654752f * z.y));
      if (SLOPE) density = make_float2(expf(-0.5f * z.x * z.x), expf(-0.5f * z.y * z.y));
    } else {
      // Abramowitz and Stegun 7.1.26 for the tail of Phi, on the exponential that phi needs anyway
      density = ex2(__fmul2_rn(__fmul2_rn(z, z), both(-0.72134752044448170f)));       // exp(-z^2 / 2)
      const float2 t = rcp(__ffma2_rn(make_float2(fabsf(z.x), fabsf(z.y)), both(0.3275911f * 0.70710678118654752f), both(1.0f)));
      float2 q = __ffma2_rn(t, both(0.5f * 1.061405429f), both(0.5f * -1.453152027f));
      q = __ffma2_rn(q, t, both(0.5f * 1.421413741f));
      q = __ffma2_rn(q, t, both(0.5f * -0.284496736f));
      q = __ffma2_rn(q, t, both(0.5f * 0.254829592f));
      q = __fmul2_rn(q, __fmul2_rn(t, density));
      const float2 over = __ffma2_rn(q, both(-1.0f), both(1.0f));
      below = make_float2(z.x >= 0.f ? over.x : q.x, z.y >= 0.f ? over.y : q.y);
    }
    *value = __fmul2_rn(z, below);
    if (SLOPE) *slope = __ffma2_rn(z, __fmul2_rn(density, both(0.3989422804014327f)), below);
  } else {
    // tanh form: (1 + tanh u) / 2 = sigmoid(2 u), u = c (z + a z^3)
    const float c = 0.79788456080286536f, a = 0.044715f;
    const float2 z2 = __fmul2_rn(z, z);
    const float2 s = sigmoid2<F32>(__fmul2_rn(z, __ffma2_rn(z2, both(2.0f * c * a), both(2.0f * c))));
    const float2 v = __fmul2_rn(z, s);
    *value = v;
    if (SLOPE) {
      const float2 rest = __ffma2_rn(s, both(-1.0f), both(1.0f));
      *slope = __ffma2_rn(__fmul2_rn(v, rest), __ffma2_rn(z2, both(6.0f * c * a), both(2.0f * c)), s);
    }
  }
}

// ---------------------------------------------------------------------------------------------- epilogue pieces
__device__ __forceinline__ void store32_bytes(void* base, const uint32_t* w) {   // 32-byte aligned
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(base), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]),
               "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}
__device__ __forceinline__ void pack16(const float* v, uint32_t* w) {
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
}
// 16 values into the library's own buffers (pitch a multiple of 64 elements): one bf16 plane, or three.
template <bool F32>
__device__ __forceinline__ void store16_planes(__nv_bfloat16* base, long long plane_stride, const float2* v) {
  uint32_t w[F32 ? 3 : 1][8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (!F32) {
      w[0][i] = pack_bf16x2(v[i].x, v[i].y);
    } else {
      uint32_t o[3];
      split3_pair(v[i].x, v[i].y, o);
#pragma unroll
      for (int k = 0; k < 3; ++k) w[k][i] = o[k];
    }
  }
#pragma unroll
  for (int k = 0; k < (F32 ? 3 : 1); ++k) store32_bytes(base + k * plane_stride, w[k]);
}
__device__ __forceinline__ void store16_f32(float* base, const float* v) {   // 16-byte aligned
#pragma unroll
  for (int i = 0; i < 4; ++i) reinterpret_cast<float4*>(base)[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
}
template <bool F32>
__device__ __forceinline__ void add_bias(const void* bias, int n0, int N, float* v) {
  if (F32) {
    const float* b = static_cast<const float*>(bias) + n0;
#pragma unroll
    for (int i = 0; i < 16; ++i) if (n0 + i < N) v[i] += __ldg(b + i);
  } else {
    const __nv_bfloat16* b = static_cast<const __nv_bfloat16*>(bias) + n0;
    if (n0 + 16 <= N) {
      const uint4 q[2] = {__ldg(reinterpret_cast<const uint4*>(b)), __ldg(reinterpret_cast<const uint4*>(b) + 1)};
      const uint32_t* w = reinterpret_cast<const uint32_t*>(q);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[2 * i] += __uint_as_float(w[i] << 16);
        v[2 * i + 1] += __uint_as_float(w[i] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) if (n0 + i < N) v[i] += __bfloat162float(b[i]);
    }
  }
}

// What is kept of G (Z) and U between forward and backward.  Their own rounding to bf16 would be a third one on the way
// to dX and dW1 besides those of dG and of the result; with four more bits it is not seen: 16 + 4 bits each, two values'
// low nibbles in one byte (G's and U's, or those of the two halves of the 16 values of Z).
// It lies in blocks of 32 rows x 16 columns, which is what a warp of either pass handles at once (a lane to a row): pieces
// of 16 bytes a lane (the last 8, for Z), each contiguous over the warp.  (Row by row, every lane's piece was a line of
// its own.)
template <bool F32, bool GATED>
struct Kept {
  static constexpr int Q = F32 ? 4 : 2;                                    // pieces of 16 values of one of G, U, Z
  static constexpr int LOW = F32 ? 0 : GATED ? 16 : 8;                     // bytes of low nibbles
  static constexpr int BLOCK = 32 * ((GATED ? 2 : 1) * Q * 16 + LOW);
  uint4 a[Q], b[GATED ? Q : 1];
  __align__(16) uint32_t lo[4];
  __device__ __forceinline__ static char* block(const Hidden& h, long long row, int n0) {
    return static_cast<char*>(h.kept) + ((row >> 5) * (h.ldm >> 4) + (n0 >> 4)) * BLOCK;
  }
  __device__ __forceinline__ void load(const Hidden& h, long long row, int n0) {
    const char* at = block(h, row, n0);
    const int lane = static_cast<int>(row & 31);
    const uint4* p = reinterpret_cast<const uint4*>(at) + lane;
#pragma unroll
    for (int i = 0; i < Q; ++i) {
      a[i] = __ldcs(p + i * 32);
      if (GATED) b[i] = __ldcs(p + (Q + i) * 32);
    }
    if constexpr (LOW == 16) *reinterpret_cast<uint4*>(lo) = __ldcs(p + 2 * Q * 32);
    if constexpr (LOW == 8) *reinterpret_cast<uint2*>(lo) = __ldcs(reinterpret_cast<const uint2*>(at + Q * 512) + lane);
  }
  __device__ __forceinline__ void store(const Hidden& h, long long row, int n0) const {
    char* at = block(h, row, n0);
    const int lane = static_cast<int>(row & 31);
    uint4* p = reinterpret_cast<uint4*>(at) + lane;
#pragma unroll
    for (int i = 0; i < Q; ++i) {
      p[i * 32] = a[i];
      if (GATED) p[(Q + i) * 32] = b[i];
    }
    if constexpr (LOW == 16) p[2 * Q * 32] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    if constexpr (LOW == 8) reinterpret_cast<uint2*>(at + Q * 512)[lane] = make_uint2(lo[0], lo[1]);
  }
  // Values i and i + 1 (i even) of the first or the second of what is kept.  One byte permutation builds a value; the low
  // byte, which is not kept, repeats the one above it.
  __device__ __forceinline__ static float2 pair(const uint4* q, int i, uint32_t low_bytes) {
    const uint32_t* words = reinterpret_cast<const uint32_t*>(q);
    if constexpr (F32) {
      return make_float2(__uint_as_float(words[i]), __uint_as_float(words[i + 1]));
    } else {
      const uint32_t w = words[i >> 1], j = 4 + (i & 3), k = j + 1;
      return make_float2(__uint_as_float(__byte_perm(w, low_bytes, 0x1000 | j << 4 | j)),
                         __uint_as_float(__byte_perm(w, low_bytes, 0x3200 | k << 4 | k)));
    }
  }
  __device__ __forceinline__ float2 first(int i) const {
    if constexpr (F32) return pair(a, i, 0u);
    if constexpr (GATED) return pair(a, i, lo[i >> 2] & 0xf0f0f0f0u);
    return pair(a, i, i < 8 ? lo[i >> 2] & 0xf0f0f0f0u : lo[(i >> 2) & 1] << 4 & 0xf0f0f0f0u);
  }
  __device__ __forceinline__ float2 second(int i) const { return pair(b, i, F32 ? 0u : lo[i >> 2] << 4 & 0xf0f0f0f0u); }

  // byte 1 of four words
  __device__ __forceinline__ static uint32_t second_bytes(const uint32_t* x) {
    return __byte_perm(__byte_perm(x[0], x[1], 0x0051), __byte_perm(x[2], x[3], 0x0051), 0x5410);
  }
  // Four values: their upper halves to `top`, returns their second bytes.  20 bits are cut, not rounded; the factor
  // 1 + 0.7 2^-12 moves the middle of what is cut off to zero.
  __device__ __forceinline__ static uint32_t cut4(const float2* v, uint32_t* top) {
    uint32_t x[4];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float2 s = __fmul2_rn(v[k], both(1.00017f));
      x[2 * k] = __float_as_uint(s.x);
      x[2 * k + 1] = __float_as_uint(s.y);
      top[k] = __byte_perm(x[2 * k], x[2 * k + 1], 0x7632);
    }
    return second_bytes(x);
  }
  __device__ __forceinline__ void set(const float2* g, const float2* u) {
    uint32_t *wa = reinterpret_cast<uint32_t*>(a), *wb = reinterpret_cast<uint32_t*>(b);
    if constexpr (F32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        wa[2 * i] = __float_as_uint(g[i].x);
        wa[2 * i + 1] = __float_as_uint(g[i].y);
        if (GATED) { wb[2 * i] = __float_as_uint(u[i].x); wb[2 * i + 1] = __float_as_uint(u[i].y); }
      }
    } else if constexpr (GATED) {
#pragma unroll
      for (int i = 0; i < 4; ++i) lo[i] = (cut4(g + 2 * i, wa + 2 * i) & 0xf0f0f0f0u) | (cut4(u + 2 * i, wb + 2 * i) >> 4 & 0x0f0f0f0fu);
    } else {
#pragma unroll
      for (int i = 0; i < 2; ++i) lo[i] = (cut4(g + 2 * i, wa + 2 * i) & 0xf0f0f0f0u) | (cut4(g + 4 + 2 * i, wa + 4 + 2 * i) >> 4 & 0x0f0f0f0fu);
    }
  }
};

// The activation's part of a pass for 16 columns of one row.  x holds the accumulators (FORWARD_GATED: G, with U in y) and
// becomes H or dG (dZ), y becomes dU.
template <int MODE, bool F32>
__device__ __forceinline__ void activate16(const Hidden& h, int act, long long row, int n0, float2* x, float2* y,
                                           const Kept<F32, MODE == FORWARD_GATED || MODE == BACKWARD_GATED>& loaded, bool in) {
  constexpr bool GATED = MODE == FORWARD_GATED || MODE == BACKWARD_GATED;
  if (MODE == FORWARD_GATED || MODE == FORWARD_ACT) {
    if (h.kept) {
      Kept<F32, GATED> k;
      k.set(x, y);
      if (in) k.store(h, row, n0);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (GATED) x[i] = __fmul2_rn(__fmul2_rn(x[i], sigmoid2<F32>(x[i])), y[i]);
      else gelu2<F32, false>(x[i], act, &x[i], nullptr);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float2 g = loaded.first(2 * i);
      if (GATED) {
        const float2 up = loaded.second(2 * i), s = sigmoid2<F32>(g);
        const float2 rest = __ffma2_rn(s, both(-1.0f), both(1.0f));
        y[i] = __fmul2_rn(x[i], __fmul2_rn(g, s));
        x[i] = __fmul2_rn(__fmul2_rn(x[i], up), __fmul2_rn(s, __ffma2_rn(g, rest, both(1.0f))));
      } else {
        float2 value, slope;
        gelu2<F32, true>(g, act, &value, &slope);
        x[i] = __fmul2_rn(x[i], slope);
      }
    }
  }
}
// What activate16() leaves, straight to memory.
template <int MODE, bool F32>
__device__ __forceinline__ void store_hidden16(const Hidden& h, long long row, int n0, const float2* x, const float2* y) {
  const long long at = row * h.ldm + n0;
  if (MODE == FORWARD_GATED || MODE == FORWARD_ACT) {
    store16_planes<F32>(h.H + at, h.plane_stride, x);
  } else {
    store16_planes<F32>(h.dG + at, h.plane_stride, x);
    if (MODE == BACKWARD_GATED) store16_planes<F32>(h.dU + at, h.plane_stride, y);
  }
}
__device__ __forceinline__ void pairs_back16(const float2* x, float* v) {
#pragma unroll
  for (int i = 0; i < 8; ++i) { v[2 * i] = x[i].x; v[2 * i + 1] = x[i].y; }
}
// Column sums over the warp's 32 rows (a lane to a row) of 16 columns, in a fixed order: lane l has that of column l / 2.
__device__ __forceinline__ float column_sums16(const float2* x, int lane) {
  float v[16];
  pairs_back16(x, v);
#pragma unroll
  for (int half = 8, bit = 16; half >= 1; half >>= 1, bit >>= 1) {
    const bool upper = (lane & bit) != 0;
#pragma unroll
    for (int i = 0; i < half; ++i) {
      const float send = upper ? v[i] : v[i + half], keep = upper ? v[i + half] : v[i];
      v[i] = keep + __shfl_xor_sync(0xffffffffu, send, bit);
    }
  }
  return v[0] + __shfl_xor_sync(0xffffffffu, v[0], 1);
}
__device__ __forceinline__ void pairs16(const float* v, float2* x) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = make_float2(v[2 * i], v[2 * i + 1]);
}

// Rows that do not start on 16 bytes (m odd, or fp32 widths that are no multiple of 4) leave through shared memory, so
// that a warp writes along one row at a time: SPAN columns of 32 rows, one word a lane and row.  (One lane to a row wrote
// two bytes into each of 32 lines per instruction: 88 us for the gradients of a 1000 x 2731 gated layer.)
template <bool F32> constexpr int SPAN_COLS = F32 ? 32 : 64;
template <bool F32>
__device__ __forceinline__ void stage16(uint32_t* buf, int lane, int col, const float* v) {   // word w of row r at w ^ r
  uint32_t* row = buf + lane * 32;
  if constexpr (F32) {
#pragma unroll
    for (int i = 0; i < 16; ++i) row[(col + i) ^ lane] = __float_as_uint(v[i]);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) row[((col >> 1) + i) ^ lane] = pack_bf16x2(v[2 * i], v[2 * i + 1]);
  }
}
// The same for a TMA store of rows of 1 << row_shift bytes (32, 64 or 128) with the swizzle of that width: 16-byte piece
// j of row r at j ^ (r % 8), j ^ (r / 2 % 4) or j ^ (r / 4 % 2).
template <bool F32>
__device__ __forceinline__ void stage16_swizzled(uint32_t* buf, int lane, int col, int row_shift, const uint32_t* w) {
  char* row = reinterpret_cast<char*>(buf) + (lane << row_shift);
  const int turn = (lane >> (7 - row_shift)) & ((1 << (row_shift - 4)) - 1);
  constexpr int PIECES = F32 ? 4 : 2;
#pragma unroll
  for (int i = 0; i < PIECES; ++i) {
    const int j = (F32 ? col >> 2 : col >> 3) + i;
    *reinterpret_cast<uint4*>(row + ((j ^ turn) << 4)) = make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
  }
}
// The staged columns n .. n + valid - 1 of rows row0 .. of C.
template <bool F32>
__device__ __forceinline__ void write_staged(const uint32_t* buf, int lane, void* C, long long ldc, long long row0, int rows, int n, int valid) {
  for (int r = 0; r < rows; ++r) {
    const uint32_t mine = buf[r * 32 + (lane ^ r)], next = buf[r * 32 + (((lane + 1) & 31) ^ r)];
    const long long at = (row0 + r) * ldc + n;
    if constexpr (F32) {
      if (lane < valid) static_cast<uint32_t*>(C)[at + lane] = mine;
    } else {
      unsigned short* out = static_cast<unsigned short*>(C) + at;
      if ((reinterpret_cast<uintptr_t>(out) & 3u) == 0) {
        if (2 * lane + 1 < valid) *reinterpret_cast<uint32_t*>(out + 2 * lane) = mine;
        else if (2 * lane < valid) out[2 * lane] = static_cast<unsigned short>(mine);
      } else {
        // words start at the odd columns; column 0 is left over, and the last one where valid is even
        const uint32_t word = mine >> 16 | next << 16;
        if (lane < 31 && 2 * lane + 2 < valid) *reinterpret_cast<uint32_t*>(out + 2 * lane + 1) = word;
        else if (2 * lane + 1 < valid) out[2 * lane + 1] = static_cast<unsigned short>(word);
        if (lane == 0) out[0] = static_cast<unsigned short>(mine);
      }
    }
  }
}

// ---------------------------------------------------------------------------------------------- the kernel
template <int MODE, bool F32, int CAP, bool EXTENDED = false>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(THREADS<MODE, F32>, 1)
    train_gemm_kernel(const __grid_constant__ typename KernelParams<CAP, EXTENDED>::type p) {
  constexpr bool GATED = MODE == FORWARD_GATED || MODE == BACKWARD_GATED;
  const int out_n = MODE == FORWARD_GATED ? p.tile_n / 2 : p.tile_n;     // output columns of a tile
  const int half_n = p.tile_n / 2;                                       // rows of B that one CTA stages
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* out_stage = smem + RING_BYTES<MODE, F32>;
  uint64_t* bars = reinterpret_cast<uint64_t*>(out_stage + EPI_WARPS<MODE, F32> * OUT_BYTES<MODE, F32>);
  uint64_t* full = bars;                  // [stages] TMA of both CTAs -> MMA (rank 0's are used)
  uint64_t* empty = full + MAX_STAGES;    // [stages] MMA -> TMA, one set in each CTA
  uint64_t* tfull = empty + MAX_STAGES;       // [2] MMA -> epilogue, one set in each CTA
  uint64_t* tempty = tfull + 2;           // [2] epilogue warps of both CTAs -> MMA (rank 0's are used)
  uint64_t* drain = tempty + 2;           // used only when giving up
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int stages = p.stages, stage_bytes = p.stage_bytes, a_bytes = p.a_bytes;
  const uint32_t rank = ptx::cluster_rank();

  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(&tfull[a], 1);
      ptx::mbar_init(&tempty[a], 2 * EPI_WARPS<MODE, F32>);
    }
    ptx::mbar_init(drain, 1);
    *abort_flag = 0;
    ptx::mbar_fence_init();
  }
  if (warp == FIRST_EPI<F32> && lane < 2) {
    ptx::prefetch_tmap(&p.prod[0].a[0]);
    ptx::prefetch_tmap(&p.prod[0].b[MODE == FORWARD_GATED ? lane : 0]);
  }
  if (warp == 1) {
    ptx::tmem_alloc_pair(tmem_holder, TMEM_COLS);
    ptx::tmem_relinquish_pair();
  }
  ptx::tc_fence_before();
  ptx::cluster_sync_all();     // also: the other CTA's barriers are set up
  ptx::tc_fence_after();
  const uint32_t tmem_base = *tmem_holder;
  const uint32_t smem0 = ptx::smem_u32(smem), full0 = ptx::map_to_cta(ptx::smem_u32(full), 0);
  // This CTA's half of B of one k-block, into stage s.
  const auto load_b = [&](const CUtensorMap* map, bool mn, int n0, int kb, int plane, int s) {
    const uint32_t to = smem0 + s * stage_bytes + a_bytes, bar = full0 + s * 8;
    if (mn) {
      ptx::tma_load_3d_pair(map, to, bar, n0, kb * BLOCK_K, plane);
      if (half_n > 64) ptx::tma_load_3d_pair(map, to + BLOCK64_BYTES, bar, n0 + 64, kb * BLOCK_K, plane);
    } else {
      ptx::tma_load_3d_pair(map, to, bar, kb * BLOCK_K, n0, plane);
    }
  };
  const auto first_column = [&](const Unit& t) { return t.n_blk * out_n + (MODE == FORWARD_GATED ? 0 : static_cast<int>(rank) * half_n); };
  const auto stage_tx = [&](const DevProduct& d) {
    return static_cast<uint32_t>((d.M > CTA_M ? 2 : 1) * d.a_rows * BLOCK_K * 2 + 2 * half_n * BLOCK_K * 2);
  };

  // Launched with programmatic stream serialisation: all of the above ran under the tail of the kernel before; so do the
  // loads of weights that it does not write.  The kernel after this one may be set up only now that this CTA holds its
  // tensor memory (see gemm_tc.cu).
  int ahead = 0;     // stages of the first unit whose B is on its way
  if (warp == 0 && p.early) {
    Walk walk;
    const int u = walk.take(p);
    if (u >= 0) {
      const Unit t = find_unit(p, u);
      const DevProduct& d = p.prod[t.prod];
      ahead = t.k1 - t.k0 < stages ? t.k1 - t.k0 : stages;
      if (ptx::elect_one()) {
        for (int i = 0; i < ahead; ++i) {
          if (rank == 0) ptx::mbar_expect_tx(&full[i], stage_tx(d));
          int pair, pa, pb;
          const int run = (t.k0 + i) / d.kb;
          run_planes<F32>(d, run, &pair, &pa, &pb);
          load_b(&d.b[MODE == FORWARD_GATED ? static_cast<int>(rank) : pair], d.b_mn, first_column(t), t.k0 + i - run * d.kb, pb, i);
        }
      }
      __syncwarp();
    }
  }
  if (!p.apart) pdl_wait();

  if (warp < FIRST_EPI<F32>) {
    if constexpr (F32) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(ROLE_REGS));
    if (warp == 0) {
      if (ptx::elect_one()) {
        // ------------------------------------------------------------ TMA producer
        Walk walk;
        uint32_t ph = 0;
        int s = 0;
        bool ok = true;
        for (int u = walk.take(p); u >= 0 && ok; u = walk.take(p)) {
          const Unit t = find_unit(p, u);
          const DevProduct& d = p.prod[t.prod];
          const uint32_t tx = stage_tx(d);
          int entries = 0;
          if constexpr (EXTENDED) entries = entries_of(p, t);
          const int m0 = t.m_blk * TILE_M + static_cast<int>(rank) * CTA_M, n0 = first_column(t);
          // Few rows: what A's box leaves out, and all of rank 1's half where M <= 128, is not staged at all.  Whatever lies
          // in shared memory there only reaches accumulator rows behind M.  (One token: the empty rows cost as much of the
          // copy engine as real ones, and the weights wait behind them.)
          const bool has_a = rank == 0 || d.M > CTA_M;
          int run = t.k0 / d.kb, kb = t.k0 - run * d.kb;
          for (; run < d.runs && run * d.kb < t.k1 && ok; ++run, kb = 0) {
            int pair, pa, pb;
            run_planes<F32>(d, run, &pair, &pa, &pb);
            const CUtensorMap* ta = &d.a[pair];
            const CUtensorMap* tb = &d.b[MODE == FORWARD_GATED ? static_cast<int>(rank) : pair];
            const int kb_end = t.k1 - run * d.kb < d.kb ? t.k1 - run * d.kb : d.kb;
            for (; kb < kb_end; ++kb) {
              if (ahead > 0) {
                --ahead;       // (an empty ring: nothing to wait for)
              } else {
                if (!ptx::mbar_wait(&empty[s], ph ^ 1, abort_flag)) { ok = false; break; }
                if (rank == 0) ptx::mbar_expect_tx(&full[s], tx);
                load_b(tb, d.b_mn, n0, kb, pb, s);
              }
              if (has_a) {
                const uint32_t to = smem0 + s * stage_bytes, bar = full0 + s * 8;
                if (d.a_mn) {
                  ptx::tma_load_3d_pair(ta, to, bar, m0, kb * BLOCK_K, pa);
                  if (d.a_rows > 64) ptx::tma_load_3d_pair(ta, to + BLOCK64_BYTES, bar, m0 + 64, kb * BLOCK_K, pa);
                } else {
                  ptx::tma_load_3d_pair(ta, to, bar, kb * BLOCK_K, m0, pa);
                }
              }
              if (++s == stages) { s = 0; ph ^= 1u; }
            }
          }
          if constexpr (EXTENDED) {
            // the entries of this tile, behind the last k-block of its sum; the next one's word is loaded ahead
            const int* list = p.list + t.m_blk * p.most;
            int word = entries > 0 ? __ldcg(list) : 0;
            for (int e = 0; e < entries && ok; ++e) {
              const int now = word;
              if (e + 1 < entries) word = __ldcg(list + e + 1);
              for (int b = 0; b < p.blocks; ++b) {
                if (!ptx::mbar_wait(&empty[s], ph ^ 1, abort_flag)) { ok = false; break; }
                if (rank == 0) ptx::mbar_expect_tx(&full[s], tx);
                load_b(&p.f, d.b_mn, n0, b, now & 0xffff, s);
                if (has_a)
                  ptx::tma_load_3d_pair(&p.q, smem0 + s * stage_bytes, full0 + s * 8, b * BLOCK_K,
                                        (t.m_blk * p.most + (now >> 16)) * TILE_M + static_cast<int>(rank) * CTA_M, 0);
                if (++s == stages) { s = 0; ph ^= 1u; }
              }
            }
          }
        }
        // The last stages: their release arrives here from rank 0, and must find this CTA's barriers still in place.
        for (int i = 0; i < stages && ok; ++i) {
          ok = ptx::mbar_wait(&empty[s], ph ^ 1, abort_flag);
          if (++s == stages) { s = 0; ph ^= 1u; }
        }
        if (!ok) {
          // Copies into this CTA's shared memory are counted on rank 0's barriers: give what is in flight a bounded time
          // to land before the CTA exits.
          const long long t0 = clock64();
          while (clock64() - t0 < ptx::kWaitLimitCycles / 64) {}
        }
      }
      __syncwarp();
    } else if (warp == 1) {
      if (rank == 0) {
        // ------------------------------------------------------------ MMA issuer (the whole warp walks, one lane issues)
        const uint32_t idesc0 = ptx::umma_idesc_bf16(TILE_M, p.tile_n);
        Walk walk;
        uint32_t tl = 0, ph = 0;
        int s = 0;
        bool ok = true;
        const auto steps_left = [&](int block) {
          if constexpr (EXTENDED) return p.steps - (block % p.blocks) * (BLOCK_K / 16);
          else return BLOCK_K / 16;
        };
        for (int u = walk.take(p); u >= 0 && ok; u = walk.take(p)) {
          const Unit t = find_unit(p, u);
          const DevProduct& d = p.prod[t.prod];
          int more = 0;      // k-blocks of entries (the load is over long before it is needed)
          if constexpr (EXTENDED) more = entries_of(p, t) * p.blocks;
          // bits 15, 16: the operand's rows run along memory
          const uint32_t idesc = idesc0 | (d.a_mn ? 1u << 15 : 0u) | (d.b_mn ? 1u << 16 : 0u);
          const uint64_t a_desc0 = d.a_mn ? ptx::umma_desc_mn128(smem0, BLOCK64_BYTES) : ptx::umma_desc_k128(smem0);
          const uint64_t b_desc0 = d.b_mn ? ptx::umma_desc_mn128(smem0 + a_bytes, BLOCK64_BYTES) : ptx::umma_desc_k128(smem0 + a_bytes);
          // 16 further along K: 32 bytes inside the swizzled row, or 16 rows of 128 bytes (addresses count 16 bytes)
          const uint32_t a_step = d.a_mn ? 2048 >> 4 : 32 >> 4, b_step = d.b_mn ? 2048 >> 4 : 32 >> 4;
          // fp32: the unit is summed in parts, each through an accumulator of its own
          for (int begin = t.k0; begin < t.k1 && ok; ++tl) {
            const int end = F32 ? part_end(d, t, begin) : t.k1;
            const uint32_t acc = tl & 1, aph = (tl >> 1) & 1;
            ok = __shfl_sync(0xffffffffu, ptx::mbar_wait_cluster(&tempty[acc], aph ^ 1, abort_flag) ? 1 : 0, 0) != 0;
            if (!ok) break;
            ptx::tc_fence_after();
            const uint32_t d_tmem = tmem_base + acc * TILE_N;
            for (int kb = begin; kb < end || (EXTENDED && kb < end + more); ++kb) {
              ok = ptx::mbar_wait_warp(&full[s], ph, abort_flag);
              if (!ok) break;
              ptx::tc_fence_after();
              const uint64_t a_desc = a_desc0 + static_cast<uint32_t>(s) * (stage_bytes >> 4);
              const uint64_t b_desc = b_desc0 + static_cast<uint32_t>(s) * (stage_bytes >> 4);
              if (ptx::elect_one()) {
  #pragma unroll
                for (int k = 0; k < BLOCK_K / 16; ++k) {
                  // (of an entry's last block what its rank needs)
                  if (EXTENDED && kb >= end && k >= steps_left(kb - end)) break;
                  ptx::umma_bf16_pair(d_tmem, a_desc + k * a_step, b_desc + k * b_step, idesc, (kb > begin || k > 0) ? 1u : 0u);
                }
                ptx::umma_commit_pair(&empty[s]);
              }
              __syncwarp();
              if (++s == stages) { s = 0; ph ^= 1u; }
            }
            if (ok) {
              if (ptx::elect_one()) ptx::umma_commit_pair(&tfull[acc]);
              __syncwarp();
            }
            begin = end;
          }
        }
        if (!ok) {
          // wait (bounded) until the MMAs issued so far have retired before tensor memory is freed
          if (ptx::elect_one()) {
            ptx::umma_commit_pair(drain);
            const long long t0 = clock64();
            while (!ptx::mbar_try_wait(drain, 0) && clock64() - t0 < ptx::kWaitLimitCycles / 8) {}
          }
          __syncwarp();
        }
      }
    }
  } else {
    if constexpr (F32) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(EPI_REGS));
    // -------------------------------------------------------------- epilogue warps
    constexpr bool LOADS = MODE == BACKWARD_GATED || MODE == BACKWARD_ACT;
    const int q = warp & 3;                             // tensor-memory lane quarter
    constexpr int GROUPS = EPI_WARPS<MODE, F32> / 4;
    const int cols = out_n / GROUPS;                    // output columns of this warp's part of the tile
    const int col0 = ((warp - FIRST_EPI<F32>) >> 2) * cols;
    const uint32_t t_quarter = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + col0;
    uint32_t* buf = reinterpret_cast<uint32_t*>(out_stage + (warp - FIRST_EPI<F32>) * OUT_BYTES<MODE, F32>);
    Walk walk;
    uint32_t tl = 0;
    bool live = true;
    for (int u = walk.take(p); u >= 0 && live; u = walk.take(p), ++tl) {
      const Unit t = find_unit(p, u);
      const DevProduct& d = p.prod[t.prod];
      const bool parts = d.splits > 1;                  // this unit leaves a partial
      const long long row = static_cast<long long>(t.m_blk) * TILE_M + rank * CTA_M + q * 32 + lane;
      const bool in = row < d.M;
      const int c0 = t.n_blk * out_n + col0;
      Kept<F32, GATED> kept;
      if (LOADS && !F32 && !parts && in && c0 < d.N) kept.load(p.hid, row, c0);
      if ((MODE == PLAIN || MODE == FORWARD_ACT) && d.bias && lane * 32 < cols && c0 + lane * 32 < d.N)
        asm volatile("prefetch.global.L1 [%0];" ::"l"(static_cast<const char*>(d.bias) + (c0 + lane * 32) * (F32 ? 4 : 2)));
      if constexpr (F32) {
        // All parts of the sum but the last are added up in registers (a gated tile's two halves lie 128 columns
        // apart); then it goes back to where the last part lies, and on as for bf16.
        constexpr int BLOCKS = TILE_N / GROUPS / 32, SKIP = MODE == FORWARD_GATED ? TILE_N / 2 - BLOCKS * 16 : 0;     // (fp32 tiles are 256 wide)
        float sum[BLOCKS][32];
        bool first = true;
        for (int begin = t.k0;; ++tl) {
          const int end = part_end(d, t, begin);
          const bool last = end == t.k1;
          if (first && last) break;      // one part: nothing to add
          if (!ptx::mbar_wait(&tfull[tl & 1], (tl >> 1) & 1, abort_flag)) { live = false; break; }
          ptx::tc_fence_after();
          const uint32_t t_part = t_quarter + (tl & 1) * TILE_N;
#pragma unroll
          for (int b = 0; b < BLOCKS; ++b) {
            const uint32_t at = t_part + b * 32 + (b >= BLOCKS / 2 ? SKIP : 0);
            float v[32];
            ptx::tmem_ld32(at, v);
            ptx::tmem_ld_wait();
            if (first) {
#pragma unroll
              for (int i = 0; i < 32; ++i) sum[b][i] = v[i];
            } else {
#pragma unroll
              for (int i = 0; i < 32; ++i) sum[b][i] += v[i];
            }
            if (last) {
              ptx::tmem_st16(at, sum[b]);
              ptx::tmem_st16(at + 16, sum[b] + 16);
            }
          }
          first = false;
          if (last) {
            ptx::tmem_st_wait();
            break;
          }
          ptx::tc_fence_before();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive_cluster(ptx::map_to_cta(ptx::smem_u32(&tempty[tl & 1]), 0));
          begin = end;
        }
        if (!live) break;
        if (LOADS && !parts && in && c0 < d.N) kept.load(p.hid, row, c0);
      }
      const uint32_t acc = tl & 1, aph = (tl >> 1) & 1;
      if (!ptx::mbar_wait(&tfull[acc], aph, abort_flag)) break;
      ptx::tc_fence_after();
      const uint32_t t_row = t_quarter + acc * TILE_N;
      const int width = d.N - c0 < cols ? d.N - c0 : cols;       // (may be negative)
      if (parts) {
        float* base = d.partial + (t.split * d.M + row) * d.ldp + c0;
#pragma unroll 1
        for (int c = 0; c < width; c += 16) {
          float v[16];
          ptx::tmem_ld16(t_row + c, v);
          ptx::tmem_ld_wait();
          if (in) store16_f32(base + c, v);
          if (MODE == FORWARD_GATED) {
            ptx::tmem_ld16(t_row + half_n + c, v);
            ptx::tmem_ld_wait();
            if (in) store16_f32(base + d.ldp / 2 + c, v);
          }
        }
      } else {
        const long long row0 = row - lane;
        const int rows = d.M - row0 >= 32 ? 32 : static_cast<int>(d.M - row0);      // (may be negative)
        constexpr int SPAN = SPAN_COLS<F32>;
        const int box = p.box_cols, row_shift = F32 ? 7 : box == 64 ? 7 : box == 32 ? 6 : 5;
        uint32_t* buf2 = buf + 512;      // BACKWARD_GATED: dU, in the second half
#pragma unroll 1
        for (int c = 0; c < width; c += 16) {
          const int n0 = c0 + c;
          float v[16];
          float2 x[8], y[8];
          ptx::tmem_ld16(t_row + c, v);
          if (MODE == FORWARD_GATED) {
            float w[16];
            ptx::tmem_ld16(t_row + half_n + c, w);
            ptx::tmem_ld_wait();
            pairs16(w, y);
          } else {
            ptx::tmem_ld_wait();
          }
          if ((MODE == PLAIN || MODE == FORWARD_ACT) && d.bias) add_bias<F32>(d.bias, n0, d.N, v);
          if (MODE != PLAIN) {
            pairs16(v, x);
            activate16<MODE, F32>(p.hid, p.act, row, n0, x, y, kept, in);
            // what was kept of the next columns is on its way while these leave
            if (LOADS && in && c + 16 < width) kept.load(p.hid, row, n0 + 16);
            if (MODE == BACKWARD_ACT && p.hid.col_sums) {
              if (!in) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = make_float2(0.f, 0.f);
              }
              const float sum = column_sums16(x, lane);
              if (rows > 0 && (lane & 1) == 0) p.hid.col_sums[(row0 / COL_SUM_ROWS) * p.hid.ldm + n0 + (lane >> 1)] = sum;
            }
          }
          if (MODE != PLAIN && F32) {
            if (in) store_hidden16<MODE, F32>(p.hid, row, n0, x, y);
          } else if (MODE == PLAIN && d.ragged) {
            const int col = c % SPAN;
            if (c == 0) {
              // the unit before may have been another product's, whose TMA stores still read the buffer
              if (lane == 0) ptx::tma_store_wait_read();
              __syncwarp();
            }
            stage16<F32>(buf, lane, col, v);
            if (col + 16 == SPAN || c + 16 >= width) {
              __syncwarp();
              const int n = n0 - col, valid = d.N - n < col + 16 ? d.N - n : col + 16;
              write_staged<F32>(buf, lane, d.C, d.ldc, row0, rows, n, valid);
              __syncwarp();
            }
          } else {
            const int col = c & (box - 1);
            if (col == 0) {
              // the stores before must have read the buffer
              if (lane == 0) ptx::tma_store_wait_read();
              __syncwarp();
            }
            uint32_t words[16];
            if (MODE == PLAIN) {
              if (F32) {
#pragma unroll
                for (int i = 0; i < 16; ++i) words[i] = __float_as_uint(v[i]);
              } else {
                pack16(v, words);
              }
            } else {
#pragma unroll
              for (int i = 0; i < 8; ++i) words[i] = pack_bf16x2(x[i].x, x[i].y);
            }
            stage16_swizzled<F32>(buf, lane, col, row_shift, words);
            if (MODE == BACKWARD_GATED) {
#pragma unroll
              for (int i = 0; i < 8; ++i) words[i] = pack_bf16x2(y[i].x, y[i].y);
              stage16_swizzled<F32>(buf2, lane, col, row_shift, words);
            }
            if (col + 16 == box || c + 16 >= width) {
              ptx::fence_proxy_async();
              __syncwarp();
              if (lane == 0 && rows > 0) {
                ptx::tma_store_2d(MODE == PLAIN ? &d.c : &p.hid_map[0], ptx::smem_u32(buf), n0 - col, static_cast<int>(row0));
                if (MODE == BACKWARD_GATED) ptx::tma_store_2d(&p.hid_map[1], ptx::smem_u32(buf2), n0 - col, static_cast<int>(row0));
              }
            }
          }
        }
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive_cluster(ptx::map_to_cta(ptx::smem_u32(&tempty[acc]), 0));
    }
    if (lane == 0) ptx::tma_store_wait();
  }

  if (p.apart) pdl_wait();     // (so that this kernel's end is the end of the one before, too)
  ptx::tc_fence_before();
  ptx::cluster_sync_all();     // neither CTA leaves while the other may still signal it or read its shared memory
  if (threadIdx.x == 0 && *abort_flag) record_status(p.status, FFSPLIT_ERR_TIMEOUT, blockIdx.x, KID_TRAIN);
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc_pair(tmem_base, TMEM_COLS);
  }
}

// Adds the partials of every product that was cut along K, in order, and finishes it.
struct JoinProduct {
  const float* partial;
  long long M, ldp, ldc;
  int N, chunks, splits;
  void* C;
  const void* bias;
  long long chunk0;      // first chunk of 16 columns of one row
};
struct JoinParams {
  JoinProduct prod[MAX_PRODUCTS];
  int n;
  long long chunks;
  int act;
  Hidden hid;
};
constexpr int JOIN_THREADS = 128, JOIN_CHUNKS = JOIN_THREADS / 4;
// The sum of four values over n partials, in order.  Eight loads are issued before the first is used (left to itself the
// compiler waited for every load in turn), and a warp reads 512 contiguous bytes (with 16 columns to a thread its requests
// fell into 16 lines each: 6 us for 9 partials of 40 rows).
__device__ __forceinline__ float4 add_partials(const float* p, long long stride, int n) {
  constexpr int FLIGHT = 8;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int k0 = 0; k0 < n; k0 += FLIGHT) {
    float4 x[FLIGHT];
#pragma unroll
    for (int k = 0; k < FLIGHT; ++k)
      x[k] = k0 + k < n ? __ldg(reinterpret_cast<const float4*>(p + (k0 + k) * stride)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int k = 0; k < FLIGHT; ++k) {
      s.x += x[k].x; s.y += x[k].y; s.z += x[k].z; s.w += x[k].w;
    }
  }
  return s;
}
// Four threads sum 16 columns of one row; where an activation follows, the block's first warp takes it from there with one
// thread to 16 columns, as in the products' epilogue.
template <int MODE, bool F32>
__global__ void __launch_bounds__(JOIN_THREADS) join_kernel(const __grid_constant__ JoinParams p) {
  constexpr bool GATED = MODE == FORWARD_GATED || MODE == BACKWARD_GATED;
  __shared__ float4 sums[MODE == PLAIN ? 1 : MODE == FORWARD_GATED ? 2 : 1][MODE == PLAIN ? 1 : JOIN_THREADS + JOIN_CHUNKS];
  pdl_wait();
  const long long chunk0 = static_cast<long long>(blockIdx.x) * JOIN_CHUNKS;
  const auto place = [&](long long chunk, int* i, long long* row, int* n0) {
    *i = 0;
    while (*i + 1 < p.n && chunk >= p.prod[*i + 1].chunk0) ++*i;
    const JoinProduct& d = p.prod[*i];
    *row = (chunk - d.chunk0) / d.chunks;
    *n0 = static_cast<int>(chunk - d.chunk0 - *row * d.chunks) * 16;
  };
  int i, n0;
  long long row;
  const long long mine = chunk0 + threadIdx.x / 4;
  if (mine < p.chunks) {
    place(mine, &i, &row, &n0);
    const JoinProduct& d = p.prod[i];
    const int col = n0 + (threadIdx.x & 3) * 4;
    const float* at = d.partial + row * d.ldp + col;      // (the partials' pitch is a multiple of 64: no chunk is short there)
    float4 v = add_partials(at, d.M * d.ldp, d.splits);
    if (MODE != PLAIN) {
      sums[0][threadIdx.x + threadIdx.x / 4] = v;
      if (MODE == FORWARD_GATED) sums[MODE == FORWARD_GATED ? 1 : 0][threadIdx.x + threadIdx.x / 4] = add_partials(at + d.ldp / 2, d.M * d.ldp, d.splits);
    } else {
      const int valid = d.N - col;
      float o[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (d.bias && k < valid)
          o[k] += F32 ? static_cast<const float*>(d.bias)[col + k] : __bfloat162float(static_cast<const __nv_bfloat16*>(d.bias)[col + k]);
      if constexpr (F32) {
        float* out = static_cast<float*>(d.C) + row * d.ldc + col;
        if (valid >= 4 && (reinterpret_cast<uintptr_t>(out) & 15u) == 0) {
          *reinterpret_cast<float4*>(out) = make_float4(o[0], o[1], o[2], o[3]);
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) if (k < valid) out[k] = o[k];
        }
      } else {
        __nv_bfloat16* out = static_cast<__nv_bfloat16*>(d.C) + row * d.ldc + col;
        if (valid >= 4 && (reinterpret_cast<uintptr_t>(out) & 7u) == 0) {
          *reinterpret_cast<uint2*>(out) = make_uint2(pack_bf16x2(o[0], o[1]), pack_bf16x2(o[2], o[3]));
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k) if (k < valid) out[k] = __float2bfloat16_rn(o[k]);
        }
      }
    }
  }
  if constexpr (MODE != PLAIN) {
    __syncthreads();
    const long long chunk = chunk0 + threadIdx.x;
    if (threadIdx.x >= JOIN_CHUNKS || chunk >= p.chunks) return;
    place(chunk, &i, &row, &n0);
    const JoinProduct& d = p.prod[i];
    Kept<F32, GATED> kept;
    if (MODE == BACKWARD_GATED || MODE == BACKWARD_ACT) kept.load(p.hid, row, n0);
    float v[16], w[16];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4 x = sums[0][threadIdx.x * 5 + k], y = sums[MODE == FORWARD_GATED ? 1 : 0][threadIdx.x * 5 + k];
      v[4 * k] = x.x; v[4 * k + 1] = x.y; v[4 * k + 2] = x.z; v[4 * k + 3] = x.w;
      w[4 * k] = y.x; w[4 * k + 1] = y.y; w[4 * k + 2] = y.z; w[4 * k + 3] = y.w;
    }
    if (MODE == FORWARD_ACT && d.bias) add_bias<F32>(d.bias, n0, d.N, v);
    float2 x[8], y[8];
    pairs16(v, x);
    pairs16(w, y);
    activate16<MODE, F32>(p.hid, p.act, row, n0, x, y, kept, true);
    store_hidden16<MODE, F32>(p.hid, row, n0, x, y);
    if (MODE == BACKWARD_ACT && p.hid.col_sums) {
      pairs_back16(x, v);
      store16_f32(p.hid.col_sums + row * p.hid.ldm + n0, v);
    }
  }
}

// ---------------------------------------------------------------------------------------------- host side
namespace {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Tensor map over [planes][rows][cols]; box of 64 columns by box_rows rows, 128-byte swizzle, zeros outside.  Made anew
// for every launch: it costs the host well under a microsecond.
ffsplit_status encode(ffsplit_ctx* ctx, const Matrix& m, int box_rows, CUtensorMap* out) {
  if (!ctx->encode_fn) {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult qres;
    const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres);
    if (e != cudaSuccess || qres != cudaDriverEntryPointSuccess || !fn)
      return fail(ctx, FFSPLIT_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
    ctx->encode_fn = fn;
  }
  cuuint64_t dims[3] = {static_cast<cuuint64_t>(m.cols), static_cast<cuuint64_t>(m.rows), static_cast<cuuint64_t>(m.planes)};
  cuuint64_t strides[2] = {static_cast<cuuint64_t>(m.ld) * 2, static_cast<cuuint64_t>(m.plane_stride) * 2};
  cuuint32_t box[3] = {BLOCK_K, static_cast<cuuint32_t>(box_rows), 1}, estr[3] = {1, 1, 1};
  const CUresult r = reinterpret_cast<EncodeTiledFn>(ctx->encode_fn)(
      out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(m.p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
      CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return fail(ctx, FFSPLIT_ERR_CUDA, "cuTensorMapEncodeTiled failed (" + std::to_string((int)r) + ")");
  return FFSPLIT_OK;
}

// Row-major output [rows, cols]: boxes of 32 rows x box_cols columns (32, 64 or 128 bytes), swizzled over that width.
ffsplit_status encode_out(ffsplit_ctx* ctx, bool f32, void* p, long long rows, int cols, long long ld, int box_cols, CUtensorMap* out) {
  const int es = f32 ? 4 : 2, bytes = box_cols * es;
  cuuint64_t dims[2] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows)}, strides[1] = {static_cast<cuuint64_t>(ld) * es};
  cuuint32_t box[2] = {static_cast<cuuint32_t>(box_cols), 32}, estr[2] = {1, 1};
  const CUresult r = reinterpret_cast<EncodeTiledFn>(ctx->encode_fn)(
      out, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p, dims, strides, box, estr,
      CU_TENSOR_MAP_INTERLEAVE_NONE,
      bytes == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_32B,
      CU_TENSOR_MAP_L2_PROMOTION_NONE, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return fail(ctx, FFSPLIT_ERR_CUDA, "cuTensorMapEncodeTiled failed (" + std::to_string((int)r) + ")");
  return FFSPLIT_OK;
}

long long ceil_div(long long a, long long b) { return (a + b - 1) / b; }

// How a launch is cut: the width of its tiles, and the ranges of K of each product.
struct Plan {
  int tile_n;
  int splits[MAX_PRODUCTS], per[MAX_PRODUCTS];
  size_t partial_bytes[MAX_PRODUCTS];
  double cost;
};

// Estimated time of a plan in microseconds, from these measurements:
//  - from launch to the first operands in shared memory 2.8 us;
//  - a k-block 0.27 us in a 256-wide tile (the tensor cores' rate), 0.2 us in a 128-wide one (shared memory's;
//    0.33 us among the gradients, both of whose operands are MN-major); where
//    every weight is read once (one row of tiles) the clusters at work share 6.2 TB/s;
//  - an epilogue is bound by what an SM can write, 18 bytes a nanosecond: the rows that exist times the bytes a column
//    leaves (kept, H; dG, dU; the output; or fp32 partials).  It runs under the next unit's sum;
//  - a join 5 us, launch included, 0.2 us for each partial and its traffic (partials, what an epilogue reads and leaves).
void estimate(Plan* plan, Mode mode, bool f32, const Product* products, int n, int clusters) {
  const int out_n = mode == FORWARD_GATED ? plan->tile_n / 2 : plan->tile_n;
  double work = 0.0, longest = 0.0, join = 0.0, tail = 0.0;
  for (int i = 0; i < n; ++i) {
    const Product& g = products[i];
    const long long u = ceil_div(g.M, TILE_M) * ceil_div(g.N, out_n) * plan->splits[i];
    const bool cut = plan->splits[i] > 1;
    const double rows = g.M < CTA_M ? static_cast<double>(g.M) : CTA_M;
    double column = f32 ? 4.0 : 2.0;                     // bytes written per row and column
    if (mode == FORWARD_GATED) column = cut ? 8.0 : f32 ? 14.0 : 7.0;
    else if (cut) column = 4.0;
    else if (mode == FORWARD_ACT) column = f32 ? 10.0 : 4.5;
    else if (mode == BACKWARD_GATED) column = f32 ? 12.0 : 4.0;
    else if (mode == BACKWARD_ACT) column = f32 ? 6.0 : 2.0;
    // (rows off 16 bytes leave word by word)
    if (mode == PLAIN && !cut && g.ldc * (f32 ? 4 : 2) % 16 != 0) column *= 2.0;
    const double epilogue = 0.7 + rows * out_n * column / 18e3;
    const double block = plan->tile_n == 256 ? 0.27 : n == 1 ? 0.2 : 0.33, len = plan->per[i] * block;
    const double hbm = g.M <= TILE_M ? plan->per[i] * plan->tile_n * 128.0 / 6.2e6 : 0.0;    // times the clusters at work
    const auto round = [&](long long busy) {
      const double t = len > hbm * busy ? len : hbm * busy;
      return t > epilogue ? t : epilogue;
    };
    const long long rounds = u / clusters, left = u % clusters;
    if (n == 1) work += rounds * round(clusters) + (left ? round(left) : 0.0);
    else work += u * round(clusters) / clusters;
    if (len + epilogue > longest) longest = len + epilogue;
    const double last = len < epilogue ? len : epilogue;
    if (last > tail) tail = last;
    if (cut) {
      const double leaves = mode == PLAIN ? 2.0 : mode == FORWARD_GATED ? 7.0 : mode == FORWARD_ACT ? 4.5 : mode == BACKWARD_GATED ? 9.0 : 4.5;
      join += 0.2 * plan->splits[i] + (plan->partial_bytes[i] + static_cast<double>(g.M) * g.N * leaves * (f32 ? 2.2 : 1.0)) / 4e6;
    }
  }
  double t = work + tail;
  if (t < longest) t = longest;
  plan->cost = 2.8 + t + (join > 0.0 ? 5.0 + join : 0.0);
}

Plan make_plan(Mode mode, bool f32, const Product* products, int n, int clusters, size_t room) {
  Plan best;
  best.cost = 1e300;
  long long total[MAX_PRODUCTS];
  for (int i = 0; i < n; ++i) total[i] = static_cast<long long>(products[i].pairs) * (f32 ? 6 : 1) * ceil_div(products[i].K, BLOCK_K);
  for (int tile_n = 256; tile_n >= (f32 ? 256 : 128); tile_n /= 2) {      // (the fp32 epilogue is written for full tiles)
    // candidates: units of at most `len` k-blocks
    long long last_len = -1;
    for (int cut = 1; cut <= 16; ++cut) {
      long long longest = 0;
      for (int i = 0; i < n; ++i) longest = total[i] > longest ? total[i] : longest;
      const long long len = ceil_div(longest, cut);
      if (len == last_len || (cut > 1 && len < 4)) break;
      last_len = len;
      Plan p;
      p.tile_n = tile_n;
      size_t bytes = 0;
      for (int i = 0; i < n; ++i) {
        const Product& g = products[i];
        const int s = static_cast<int>(ceil_div(total[i], len));
        p.per[i] = static_cast<int>(ceil_div(total[i], s));
        p.splits[i] = static_cast<int>(ceil_div(total[i], p.per[i]));
        const long long ldp = (mode == FORWARD_GATED ? 2 : 1) * round_up_ll(g.N, 64);
        p.partial_bytes[i] = p.splits[i] > 1 ? static_cast<size_t>(p.splits[i]) * g.M * ldp * 4 : 0;
        bytes += p.partial_bytes[i];
      }
      if (cut > 1 && bytes > room) break;
      estimate(&p, mode, f32, products, n, clusters);
      if (p.cost < best.cost) best = p;
    }
  }
  return best;
}

template <int MODE, bool F32, int CAP, bool EXTENDED = false>
ffsplit_status launch_mode(ffsplit_ctx* ctx, typename KernelParams<CAP, EXTENDED>::type& p, const JoinParams& join, int clusters, cudaStream_t st) {
  const unsigned bit = EXTENDED ? 1u << 31 : 1u << (MODE * 2 + (F32 ? 1 : 0) + (CAP > 1 ? 10 : 0));
  if (!(ctx->attr_train_set & bit)) {
    const cudaError_t e = cudaFuncSetAttribute(train_gemm_kernel<MODE, F32, CAP, EXTENDED>, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_SMEM);
    if (e != cudaSuccess) return check_cuda(ctx, e, "cudaFuncSetAttribute(train_gemm_kernel)");
    if (F32) {
      // the split of registers in the kernel counts on what the block starts with
      cudaFuncAttributes attr;
      const cudaError_t a = cudaFuncGetAttributes(&attr, train_gemm_kernel<MODE, F32, CAP, EXTENDED>);
      if (a != cudaSuccess) return check_cuda(ctx, a, "cudaFuncGetAttributes(train_gemm_kernel)");
      if (attr.numRegs < START_REGS) return fail(ctx, FFSPLIT_ERR_CUDA, "train_gemm_kernel was built with fewer registers than it divides");
    }
    ctx->attr_train_set |= bit;
  }
  p.stages = RING_BYTES<MODE, F32> / p.stage_bytes < MAX_STAGES ? RING_BYTES<MODE, F32> / p.stage_bytes : MAX_STAGES;
  cudaError_t e = launch_pdl(train_gemm_kernel<MODE, F32, CAP, EXTENDED>, dim3(2 * clusters), dim3(THREADS<MODE, F32>), MAX_SMEM, st, p);
  ctx->launches++;
  if (e != cudaSuccess || join.n == 0) return check_cuda(ctx, e, "train_gemm_kernel launch");
  e = launch_pdl(join_kernel<MODE, F32>, dim3(static_cast<unsigned>(ceil_div(join.chunks, JOIN_CHUNKS))), dim3(JOIN_THREADS), 0, st, join);
  ctx->launches++;
  return check_cuda(ctx, e, "join_kernel launch");
}

// CAP: products that the argument block has room for (it is copied with every launch).
template <int CAP>
ffsplit_status launch_products(ffsplit_ctx* ctx, Mode mode, int act, bool f32, const Product* products, int n, const Hidden& hidden,
                               char* partials, size_t partial_room, cudaStream_t st, bool* joined, const Extension* extension) {
  // The tensor maps are made by a driver call, which needs a current context; a thread that has only asked the runtime for
  // its device (autograd's backward threads) has none yet.
  const cudaError_t bound = cudaSetDevice(ctx->device);
  if (bound != cudaSuccess) return check_cuda(ctx, bound, "cudaSetDevice");
  Params<CAP> p;
  JoinParams join;
  std::memset(&p, 0, sizeof(p));
  std::memset(&join, 0, sizeof(join));
  const int clusters_max = ctx->num_sms / 2;
  const Plan plan = make_plan(mode, f32, products, n, clusters_max, partial_room);
  // longest units first
  int order[MAX_PRODUCTS], wanted = 0;
  for (int i = 0; i < n; ++i) {
    if (mode == PLAIN && !products[i].C) continue;
    int at = wanted++;
    for (; at > 0 && plan.per[order[at - 1]] < plan.per[i]; --at) order[at] = order[at - 1];
    order[at] = i;
  }
  n = wanted;
  const int out_n = mode == FORWARD_GATED ? plan.tile_n / 2 : plan.tile_n;
  const int planes6 = f32 ? 6 : 1;
  // an output box is as wide as a warp's part of the tile, but no wider than 128 bytes (64 where
  // there are 16 warps)
  const int part = out_n / (f32 || mode == PLAIN ? 2 : 4), widest = f32 || mode != PLAIN ? 32 : 64;
  p.box_cols = part < widest ? part : widest;
  long long units = 0;
  for (int i = 0; i < n; ++i) {
    const Product& g = products[order[i]];
    DevProduct& d = p.prod[i];
    const int maps_b = mode == FORWARD_GATED ? 2 : g.pairs;
    d.a_rows = g.M >= CTA_M ? CTA_M : g.a_mn ? (g.M > 64 ? 128 : 64) : static_cast<int>(round_up_ll(g.M, 8));
    ffsplit_status s;
    for (int j = 0; j < g.pairs; ++j)
      if ((s = encode(ctx, g.a[j], g.a_mn ? BLOCK_K : d.a_rows, &d.a[j])) != FFSPLIT_OK) return s;
    for (int j = 0; j < maps_b; ++j)
      if ((s = encode(ctx, g.b[j], g.b_mn ? BLOCK_K : plan.tile_n / 2, &d.b[j])) != FFSPLIT_OK) return s;
    d.M = g.M; d.N = g.N;
    d.kb = static_cast<int>(ceil_div(g.K, BLOCK_K));
    d.pairs = g.pairs; d.runs = g.pairs * planes6;
    d.a_mn = g.a_mn; d.b_mn = g.b_mn;
    d.tiles_m = static_cast<int>(ceil_div(g.M, TILE_M));
    d.tiles_n = static_cast<int>(ceil_div(g.N, out_n));
    d.unit0 = static_cast<int>(units);
    d.splits = plan.splits[order[i]];
    d.per = plan.per[order[i]];
    d.C = g.C; d.ldc = g.ldc; d.bias = g.bias;
    d.ragged = (g.ldc * (f32 ? 4 : 2)) % 16 != 0 ? 1 : 0;     // (the tensors themselves start on 16 bytes)
    if (mode == PLAIN && d.splits == 1 && !d.ragged && (s = encode_out(ctx, f32, g.C, g.M, g.N, g.ldc, p.box_cols, &d.c)) != FFSPLIT_OK) return s;
    if (d.splits > 1) {
      d.partial = reinterpret_cast<float*>(partials);
      d.ldp = (mode == FORWARD_GATED ? 2 : 1) * round_up_ll(g.N, 64);
      partials += plan.partial_bytes[order[i]];
      JoinProduct& j = join.prod[join.n++];
      j.partial = d.partial;
      j.M = g.M; j.ldp = d.ldp; j.ldc = g.ldc; j.N = g.N; j.splits = d.splits;
      j.chunks = (g.N + 15) / 16;
      j.C = g.C; j.bias = g.bias;
      j.chunk0 = join.chunks;
      join.chunks += g.M * j.chunks;
    }
    // panel height: the tiles in flight form a block whose two sides carry about the same operand bytes
    int best = 1;
    double best_cost = 1e300;
    for (int h = 1; h <= d.tiles_m && h <= clusters_max; ++h) {
      const double w = static_cast<double>(clusters_max) / h;
      const double cost = h * 256.0 + (w < d.tiles_n ? w : d.tiles_n) * plan.tile_n;
      if (cost < best_cost - 1e-9) { best_cost = cost; best = h; }
    }
    d.panel_m = best;
    units += static_cast<long long>(d.tiles_m) * d.tiles_n * d.splits;
    if (units > 0x3fffffffll) return fail(ctx, FFSPLIT_ERR_SHAPE, "more than 2^30 tiles in one product");
  }
  p.n_prod = n;
  p.tile_n = plan.tile_n;
  int a_rows = 8;
  for (int i = 0; i < n; ++i) a_rows = p.prod[i].a_rows > a_rows ? p.prod[i].a_rows : a_rows;
  p.a_bytes = a_rows * 128;
  p.stage_bytes = p.a_bytes + plan.tile_n / 2 * 128;
  p.units = static_cast<int>(units);
  const int clusters = units < clusters_max ? static_cast<int>(units) : clusters_max;
  // The product with the longest units is dealt first; where its last round does not reach every cluster and shorter
  // units follow, the clusters left out get as many of those as fit into the length of one long unit.
  if (CAP > 1 && n > 1 && p.prod[0].per > p.prod[CAP > 1 ? 1 : 0].per) {
    p.heavy = p.prod[CAP > 1 ? 1 : 0].unit0;
    const int left = p.heavy % clusters;
    if (left) {
      constexpr int EPILOGUE_BLOCKS = 4;    // a unit's set-up and tail, in k-blocks
      p.short_from = left;
      const long long extra = (p.prod[0].per + EPILOGUE_BLOCKS) / (p.prod[CAP > 1 ? 1 : 0].per + EPILOGUE_BLOCKS);
      const long long most = (units - p.heavy) / (clusters - left);
      p.extra = static_cast<int>(extra < most ? extra : most);
    }
  }
  p.apart = n == 1 && products[0].apart ? 1 : 0;
  p.early = n == 1 && products[0].b_ready && !p.apart ? 1 : 0;
  p.act = act;
  p.hid = hidden;
  if (mode != PLAIN && !f32) {
    const bool forward = mode == FORWARD_GATED || mode == FORWARD_ACT;
    void* outs[2] = {forward ? hidden.H : hidden.dG, mode == BACKWARD_GATED ? hidden.dU : nullptr};
    for (int i = 0; i < 2; ++i) {
      ffsplit_status s;
      if (outs[i] && (s = encode_out(ctx, false, outs[i], products[0].M, products[0].N, hidden.ldm, p.box_cols, &p.hid_map[i])) != FFSPLIT_OK) return s;
    }
  }
  p.status = ctx->status();
  join.act = act;
  join.hid = hidden;
  if (joined) *joined = join.n > 0;
  if constexpr (CAP == 1) {
    if (extension) {
      ExtendedParams x;
      std::memset(&x, 0, sizeof(x));
      static_cast<Params<1>&>(x) = p;
      const Extension& e = *extension;
      const Matrix q = {e.Q, e.entries * TILE_M, e.pitch, e.pitch, e.entries * TILE_M * e.pitch, 1};
      ffsplit_status s;
      if ((s = encode(ctx, q, p.prod[0].a_rows, &x.q)) != FFSPLIT_OK) return s;
      if ((s = encode(ctx, e.F, products[0].b_mn ? BLOCK_K : p.tile_n / 2, &x.f)) != FFSPLIT_OK) return s;
      x.count = e.count; x.list = e.list;
      x.most = e.most;
      x.blocks = e.pitch / BLOCK_K;
      x.steps = (e.rank + 15) / 16;
      return launch_mode<PLAIN, false, 1, true>(ctx, x, join, clusters, st);
    }
  }
  if constexpr (CAP > 1) {
    return f32 ? launch_mode<PLAIN, true, CAP>(ctx, p, join, clusters, st) : launch_mode<PLAIN, false, CAP>(ctx, p, join, clusters, st);
  } else {
    switch (mode) {
      case PLAIN: return f32 ? launch_mode<PLAIN, true, CAP>(ctx, p, join, clusters, st) : launch_mode<PLAIN, false, CAP>(ctx, p, join, clusters, st);
      case FORWARD_GATED:
        return f32 ? launch_mode<FORWARD_GATED, true, CAP>(ctx, p, join, clusters, st) : launch_mode<FORWARD_GATED, false, CAP>(ctx, p, join, clusters, st);
      case FORWARD_ACT:
        return f32 ? launch_mode<FORWARD_ACT, true, CAP>(ctx, p, join, clusters, st) : launch_mode<FORWARD_ACT, false, CAP>(ctx, p, join, clusters, st);
      case BACKWARD_GATED:
        return f32 ? launch_mode<BACKWARD_GATED, true, CAP>(ctx, p, join, clusters, st) : launch_mode<BACKWARD_GATED, false, CAP>(ctx, p, join, clusters, st);
      default:
        return f32 ? launch_mode<BACKWARD_ACT, true, CAP>(ctx, p, join, clusters, st) : launch_mode<BACKWARD_ACT, false, CAP>(ctx, p, join, clusters, st);
    }
  }
}

}  // namespace

ffsplit_status launch(ffsplit_ctx* ctx, Mode mode, int act, bool f32, const Product* products, int n, const Hidden& hidden, char* partials,
                      size_t partial_room, cudaStream_t st, bool* joined, const Extension* extension) {
  return n == 1 ? launch_products<1>(ctx, mode, act, f32, products, n, hidden, partials, partial_room, st, joined, extension)
                : launch_products<MAX_PRODUCTS>(ctx, mode, act, f32, products, n, hidden, partials, partial_room, st, joined, nullptr);
}

}  // namespace tg
}  // namespace ffsp
