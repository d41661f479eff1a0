// The three products of a Newton-Schulz iteration on the tensor cores:
//
//   S = X X^T,   P = a I + b S + c S S,   X <- P X          (rows > cols: S = X^T X, X <- X P)
//
// for a group of matrices of one shape, up to four groups to a launch.  A persistent pair of CTAs (cta_group::2) takes
// 256 x 256 (or 256 x 128) tiles: TMA into a ring of stages, one thread issues the MMAs of both CTAs, two accumulators, the
// epilogue of a tile under the MMAs of the next.  X lies as it came: whichever of its axes a product sums over, the operand
// is staged K-major or MN-major (a bit of the instruction descriptor and the shape of the TMA box).
//
// S and S S are symmetric: only tiles on and above the diagonal are computed, the others are written by their mirror images
// (of 4 p^2 q + 2 p^3 operations per iteration, p <= q, p^2 q + p^3 go).
//
// Operands are fp16 (11 bits; bf16 has 8 at the same rate).  Rounding S or P multiplies X by a matrix close to the identity,
// which the iteration corrects or carries along as it is.  Rounding X would add noise in every direction, and directions
// with small singular values would drown in what is rounded off the large ones (a momentum with a few strong directions: 1e-2
// of the result, with bf16 8e-2).  So X has a second plane for the next 11 bits.  a is added to the diagonal of P, so that the
// tensor cores form a X + P X from the first plane, and the epilogue adds a times the second: 5e-4 to 4e-3, for 2 bytes read and
// written per element.  precise: the tensor cores take the second planes of all operands (three products of planes, the small
// ones first), and sums leave them every few k-blocks, because their running sums are cut, not rounded (see train_gemm.cu).
//
// Every wait is bounded; on expiry the CTA records FFSPLIT_ERR_TIMEOUT, lets its copies and MMAs land and returns.
#include <cstring>

#include "epilogue.cuh"
#include "muon.h"
#include "ptx.cuh"

namespace ffsp {
namespace muon {

constexpr int CTA_M = 128, TILE_M = 256, TILE_N = 256, BLOCK_K = 64;
constexpr int MAX_STAGES = 8;
constexpr int BLOCK64_BYTES = 64 * BLOCK_K * 2;
constexpr int TMEM_COLS = 512;
constexpr int BAR_BYTES = 256;
constexpr int MAX_SMEM = 232448;
// Outputs leave through shared memory: 32 x 32 values of a warp at a time, one TMA store to a plane, and another to the mirror
// image.  (A row to a lane, as the sums lie in tensor memory, every store falls into 32 lines: 126 us for the third product of
// twelve 1024 x 4096 matrices, now 98.)  What is left holds the ring.
constexpr int BOX = 32, BOX_BYTES = BOX * BOX * 2;
// An epilogue reads 2 bytes of every value and writes 4 while the tensor cores take 17 us over a tile (K = 4096): with 8 warps,
// each waiting for its next 16 columns, it took 35 us.  precise: 8, for the sake of their registers.
template <bool PRECISE> constexpr int EPI_WARPS = PRECISE ? 8 : 16;
template <bool PRECISE> constexpr int GROUPS = EPI_WARPS<PRECISE> / 4;
// precise: the epilogue's sums take 128 registers a thread; it starts on a warpgroup's boundary so that registers can move
// to it (384 threads start with 168 each; 128 of them go down to 56 and 256 up to 224: 64512 in all).
template <bool PRECISE> constexpr int FIRST_EPI = PRECISE ? 4 : 2;
constexpr int START_REGS = 168, ROLE_REGS = 56, EPI_REGS = 224;
static_assert(ROLE_REGS * 128 + EPI_REGS * 256 <= START_REGS * 384, "a split above what the block starts with waits forever");
template <bool PRECISE> constexpr int GEMM_THREADS = 32 * (EPI_WARPS<PRECISE> + FIRST_EPI<PRECISE>);
// Every PROMOTE k-blocks, and every one of P = a I + b S + c S S: S S is what a whole P is off by, three times what the other sums'
// loss comes to (of S itself most is lost again between b S and 2 c S S).  512 x 4096 fp32: 5.4e-6, with four k-blocks there too
// 1.1e-5; three 1024 x 2752: 725 us, 677.  All sums after one k-block: 4.7e-6 and 855 us.
constexpr int PROMOTE = 4, PROMOTE_POLYNOMIAL = 1;

struct DevProduct {
  CUtensorMap a, b, c;
  int M, N, kb, count;
  int promote;                // precise: k-blocks of a part
  int a_mn, b_mn, symmetric;
  int tiles_m, tiles_n, tiles, panel_m;
  int unit0;
  float alpha, beta, beta_low, diagonal;
  const __half *D, *D_low;    // either may be missing
  long long d_each, d_low_each;
  int ldd;
  __half* C_low;              // in blocks, or nullptr
  long long c_low_each;
  int ldc;
  const Target* target;
};
struct Params {
  DevProduct prod[MAX_GROUPS];
  int n, units, tile_n, stages, stage_bytes;
  int ring_bytes, out_bytes;  // out_bytes: of one epilogue warp
  int* status;
};
struct Unit {
  int prod, batch, m_blk, n_blk;
};
__device__ __forceinline__ Unit find_unit(const Params& p, int u) {
  Unit r;
  r.prod = 0;
  while (r.prod + 1 < p.n && u >= p.prod[r.prod + 1].unit0) ++r.prod;
  const DevProduct& d = p.prod[r.prod];
  const int in = u - d.unit0;
  r.batch = in / d.tiles;
  int tile = in - r.batch * d.tiles;
  if (d.symmetric) {
    // row block m starts at the column block that holds its diagonal
    const int step = TILE_M / p.tile_n;
    int m = 0, width = d.tiles_n;
    while (tile >= width) { tile -= width; ++m; width -= step; }
    r.m_blk = m;
    r.n_blk = m * step + tile;
  } else {
    const int per_panel = d.panel_m * d.tiles_n;
    const int panel = tile / per_panel, in_panel = tile - panel * per_panel, m0 = panel * d.panel_m;
    const int h = d.tiles_m - m0 < d.panel_m ? d.tiles_m - m0 : d.panel_m;
    r.n_blk = in_panel / h;
    r.m_blk = m0 + (in_panel - r.n_blk * h);
  }
  return r;
}
// precise: k-blocks of a unit are counted over three runs, (low, high), (high, low), (high, high).  End of the part of the
// sum that begins at `begin`: both small runs are one part.
__device__ __forceinline__ int part_end(const DevProduct& d, int begin) {
  const int small = 2 * d.kb;
  if (begin < small) return small;
  return begin + d.promote < 3 * d.kb ? begin + d.promote : 3 * d.kb;
}

__device__ __forceinline__ float2 half_pair(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }
// 16 columns of one row in a second plane of blocks.
__device__ __forceinline__ void store_block(__half* at, const uint32_t* w) {
  reinterpret_cast<uint4*>(at)[0] = make_uint4(w[0], w[1], w[2], w[3]);
  reinterpret_cast<uint4*>(at)[32] = make_uint4(w[4], w[5], w[6], w[7]);
}
__device__ __forceinline__ void load_block(const __half* at, uint32_t* w) {
  const uint4 x = __ldcg(reinterpret_cast<const uint4*>(at)), y = __ldcg(reinterpret_cast<const uint4*>(at) + 32);
  w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w; w[4] = y.x; w[5] = y.y; w[6] = y.z; w[7] = y.w;
}
// 16 columns of a lane's row into a box of 32 x 32 with the 64-byte swizzle: 16-byte piece j of row r at j ^ (r / 2 % 4).
__device__ __forceinline__ void stage16(uint8_t* buf, int lane, int col, const uint32_t* w) {
  uint8_t* row = buf + lane * (BOX * 2);
  const int turn = (lane >> 1) & 3, j = col >> 3;
  *reinterpret_cast<uint4*>(row + ((j ^ turn) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
  *reinterpret_cast<uint4*>(row + (((j + 1) ^ turn) << 4)) = make_uint4(w[4], w[5], w[6], w[7]);
}
// The same, rows and columns exchanged.  (Four addresses, the rest are immediate offsets: sixteen of them in registers spilled.)
__device__ __forceinline__ void stage16_turned(uint8_t* buf, int lane, int col, const uint32_t* w) {
  const uint32_t base = ptx::smem_u32(buf) + (lane & 7) * 2;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const uint32_t at = base + (((lane >> 3) ^ q) << 4);
#pragma unroll
    for (int i = 2 * q; i < 16; i += 8) {       // rows i and i + 1
      const uint32_t to = at + (col + i) * (BOX * 2);
      asm volatile("st.shared.u16 [%0], %1;" ::"r"(to), "h"(static_cast<unsigned short>(w[i >> 1])) : "memory");
      asm volatile("st.shared.u16 [%0 + 64], %1;" ::"r"(to), "h"(static_cast<unsigned short>(w[i >> 1] >> 16)) : "memory");
    }
  }
}
static_assert(BOX * 2 == 64, "the offset of the next row");
__device__ __forceinline__ void load32_bytes(const void* base, uint32_t* w) {
  asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
               : "l"(base));
}
// v += beta times 16 halves
__device__ __forceinline__ void add16(float* v, float beta, const uint32_t* w) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float2 x = half_pair(w[i]);
    v[2 * i] = fmaf(beta, x.x, v[2 * i]);
    v[2 * i + 1] = fmaf(beta, x.y, v[2 * i + 1]);
  }
}
__device__ __forceinline__ uint32_t pair_half(float x, float y) {
  const __half2 h = __floats2half2_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// The last product: 32 x 32 values of a warp (X times HELD), turned to rows in shared memory, update a matrix.  A warp goes along
// its rows, two columns to a lane and two rows at a time where the matrix allows words of two (`even`), else a row at a time;
// the weights of 16 rows are on their way at once.  (A row to a lane: 190 us for twelve 1024 x 4096 matrices where the same product
// without an update takes 126, and 150 instead of 50 for 1000 x 2731, whose rows start anywhere.)
constexpr int TURN_PITCH = 33, TURN_BYTES = BOX * TURN_PITCH * 4;
template <bool F32>
__device__ __forceinline__ void update_rows(const Target& t, const float* turn, int lane, long long row0, int rows, int n0, int N) {
  const float step = t.step * (1.f / HELD), keep = t.keep;
  const int col = n0 + lane;
  if (col >= N) return;
#pragma unroll
  for (int r0 = 0; r0 < BOX; r0 += 16) {
    float w[16];
    const long long at = (row0 + r0) * N + col;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      w[i] = 0.f;
      if (t.W && r0 + i < rows)
        w[i] = F32 ? static_cast<const float*>(t.W)[at + static_cast<long long>(i) * N] : __bfloat162float(static_cast<const __nv_bfloat16*>(t.W)[at + static_cast<long long>(i) * N]);
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      if (r0 + i >= rows) break;
      const float x = turn[(r0 + i) * TURN_PITCH + lane], o = t.W ? fmaf(keep, w[i], -step * x) : -step * x;
      if (F32) static_cast<float*>(t.out)[at + static_cast<long long>(i) * N] = o;
      else static_cast<__nv_bfloat16*>(t.out)[at + static_cast<long long>(i) * N] = __float2bfloat16_rn(o);
    }
  }
}
__device__ __forceinline__ void update_rows_even(const Target& t, const float* turn, int lane, long long row0, int rows, int n0, int N) {
  const float step = t.step * (1.f / HELD), keep = t.keep;
  const int c = (lane & 15) * 2, up = lane >> 4;
  if (n0 + c >= N) return;      // (N is even)
  const long long at = (row0 + up) * N + n0 + c;
  uint32_t w[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    w[i] = 0u;
    if (t.W && 2 * i + up < rows) w[i] = *reinterpret_cast<const uint32_t*>(static_cast<const __nv_bfloat16*>(t.W) + at + 2ll * i * N);
  }
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    if (2 * i + up >= rows) break;
    const float* x = turn + (2 * i + up) * TURN_PITCH + c;
    float lo = -step * x[0], hi = -step * x[1];
    if (t.W) {
      lo = fmaf(keep, __uint_as_float(w[i] << 16), lo);
      hi = fmaf(keep, __uint_as_float(w[i] & 0xffff0000u), hi);
    }
    *reinterpret_cast<uint32_t*>(static_cast<__nv_bfloat16*>(t.out) + at + 2ll * i * N) = pack_bf16x2(lo, hi);
  }
}

// LAST: the matrices are updated with the product.
template <bool PRECISE, bool LAST>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(GEMM_THREADS<PRECISE>, 1) muon_gemm_kernel(const __grid_constant__ Params p) {
  constexpr int FIRST = FIRST_EPI<PRECISE>;
  const int half_n = p.tile_n / 2;          // rows of B that one CTA stages
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* out_stage = smem + p.ring_bytes;
  uint64_t* bars = reinterpret_cast<uint64_t*>(out_stage + EPI_WARPS<PRECISE> * p.out_bytes);
  uint64_t* full = bars;                    // [stages] TMA of both CTAs -> MMA (rank 0's are used)
  uint64_t* empty = full + MAX_STAGES;      // [stages] MMA -> TMA, one set in each CTA
  uint64_t* tfull = empty + MAX_STAGES;     // [2] MMA -> epilogue, one set in each CTA
  uint64_t* tempty = tfull + 2;             // [2] epilogue warps of both CTAs -> MMA (rank 0's are used)
  uint64_t* drain = tempty + 2;             // used only when giving up
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int stages = p.stages, stage_bytes = p.stage_bytes;
  constexpr int a_bytes = CTA_M * BLOCK_K * 2;
  const uint32_t rank = ptx::cluster_rank();

  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) {
      ptx::mbar_init(&tfull[a], 1);
      ptx::mbar_init(&tempty[a], 2 * EPI_WARPS<PRECISE>);
    }
    ptx::mbar_init(drain, 1);
    *abort_flag = 0;
    ptx::mbar_fence_init();
  }
  if (warp == FIRST && lane == 0) {
    ptx::prefetch_tmap(&p.prod[0].a);
    ptx::prefetch_tmap(&p.prod[0].b);
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
  pdl_wait();

  const int first_unit = blockIdx.x >> 1, unit_step = gridDim.x >> 1;
  if (warp < FIRST) {
    if constexpr (PRECISE) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(ROLE_REGS));
    if (warp == 0) {
      if (ptx::elect_one()) {
        // ------------------------------------------------------------ TMA producer
        uint32_t ph = 0;
        int s = 0;
        bool ok = true;
        const uint32_t tx = 2u * stage_bytes;
        for (int u = first_unit; u < p.units && ok; u += unit_step) {
          const Unit t = find_unit(p, u);
          const DevProduct& d = p.prod[t.prod];
          const int m0 = t.m_blk * TILE_M + static_cast<int>(rank) * CTA_M, n0 = t.n_blk * p.tile_n + static_cast<int>(rank) * half_n;
          for (int run = 0; run < (PRECISE ? 3 : 1) && ok; ++run) {
            const int za = (PRECISE && run == 0 ? d.count : 0) + t.batch, zb = (PRECISE && run == 1 ? d.count : 0) + t.batch;
            for (int kb = 0; kb < d.kb; ++kb) {
              if (!ptx::mbar_wait(&empty[s], ph ^ 1, abort_flag)) { ok = false; break; }
              if (rank == 0) ptx::mbar_expect_tx(&full[s], tx);
              const uint32_t to = smem0 + s * stage_bytes, bar = full0 + s * 8;
              if (d.a_mn) {
                ptx::tma_load_3d_pair(&d.a, to, bar, m0, kb * BLOCK_K, za);
                ptx::tma_load_3d_pair(&d.a, to + BLOCK64_BYTES, bar, m0 + 64, kb * BLOCK_K, za);
              } else {
                ptx::tma_load_3d_pair(&d.a, to, bar, kb * BLOCK_K, m0, za);
              }
              if (d.b_mn) {
                ptx::tma_load_3d_pair(&d.b, to + a_bytes, bar, n0, kb * BLOCK_K, zb);
                if (half_n > 64) ptx::tma_load_3d_pair(&d.b, to + a_bytes + BLOCK64_BYTES, bar, n0 + 64, kb * BLOCK_K, zb);
              } else {
                ptx::tma_load_3d_pair(&d.b, to + a_bytes, bar, kb * BLOCK_K, n0, zb);
              }
              if (++s == stages) { s = 0; ph ^= 1u; }
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
    } else if (warp == 1 && rank == 0) {
      // -------------------------------------------------------------- MMA issuer (the whole warp walks, one lane issues)
      const uint32_t idesc0 = ptx::umma_idesc_f16(TILE_M, p.tile_n);
      uint32_t tl = 0, ph = 0;
      int s = 0;
      bool ok = true;
      for (int u = first_unit; u < p.units && ok; u += unit_step) {
        const Unit t = find_unit(p, u);
        const DevProduct& d = p.prod[t.prod];
        // bits 15, 16: the operand's rows run along memory
        const uint32_t idesc = idesc0 | (d.a_mn ? 1u << 15 : 0u) | (d.b_mn ? 1u << 16 : 0u);
        const uint64_t a_desc0 = d.a_mn ? ptx::umma_desc_mn128(smem0, BLOCK64_BYTES) : ptx::umma_desc_k128(smem0);
        const uint64_t b_desc0 = d.b_mn ? ptx::umma_desc_mn128(smem0 + a_bytes, BLOCK64_BYTES) : ptx::umma_desc_k128(smem0 + a_bytes);
        const uint32_t a_step = d.a_mn ? 2048 >> 4 : 32 >> 4, b_step = d.b_mn ? 2048 >> 4 : 32 >> 4;
        const int all = (PRECISE ? 3 : 1) * d.kb;
        for (int begin = 0; begin < all && ok; ++tl) {
          const int end = PRECISE ? part_end(d, begin) : all;
          const uint32_t acc = tl & 1, aph = (tl >> 1) & 1;
          ok = __shfl_sync(0xffffffffu, ptx::mbar_wait_cluster(&tempty[acc], aph ^ 1, abort_flag) ? 1 : 0, 0) != 0;
          if (!ok) break;
          ptx::tc_fence_after();
          const uint32_t d_tmem = tmem_base + acc * TILE_N;
          for (int kb = begin; kb < end; ++kb) {
            ok = ptx::mbar_wait_warp(&full[s], ph, abort_flag);
            if (!ok) break;
            ptx::tc_fence_after();
            const uint64_t a_desc = a_desc0 + static_cast<uint32_t>(s) * (stage_bytes >> 4);
            const uint64_t b_desc = b_desc0 + static_cast<uint32_t>(s) * (stage_bytes >> 4);
            if (ptx::elect_one()) {
#pragma unroll
              for (int k = 0; k < BLOCK_K / 16; ++k)
                ptx::umma_bf16_pair(d_tmem, a_desc + k * a_step, b_desc + k * b_step, idesc, (kb > begin || k > 0) ? 1u : 0u);
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
  } else {
    if constexpr (PRECISE) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(EPI_REGS));
    // -------------------------------------------------------------- epilogue warps
    const int q = warp & 3;                                // tensor-memory lane quarter
    const int cols = p.tile_n / GROUPS<PRECISE>;                    // columns of this warp's part of the tile
    const int col0 = ((warp - FIRST) >> 2) * cols;
    const uint32_t t_quarter = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + col0;
    uint8_t* buf = out_stage + (warp - FIRST) * p.out_bytes;
    uint32_t tl = 0;
    bool live = true;
    for (int u = first_unit; u < p.units && live; u += unit_step, ++tl) {
      const Unit t = find_unit(p, u);
      const DevProduct& d = p.prod[t.prod];
      const int row0 = t.m_blk * TILE_M + static_cast<int>(rank) * CTA_M + q * 32, row = row0 + lane;
      const bool in = row < d.M;
      const int c0 = t.n_blk * p.tile_n + col0;
      const int width = d.N - c0 < cols ? d.N - c0 : cols;       // (may be negative)
      const bool leaves = row0 < d.M;                            // (a warp without rows stores nothing)
      const bool mirror = d.symmetric && t.n_blk * p.tile_n >= (t.m_blk + 1) * TILE_M;
      // What is added is on its way two pieces of 16 columns ahead: the first plane of S, or the second of X.
      const bool blocks = !PRECISE && !d.D;                      // (how that lies)
      const __half* add = nullptr;
      if (in && d.D) add = d.D + t.batch * d.d_each + static_cast<long long>(row) * d.ldd + c0;
      else if (in && blocks && d.D_low) add = d.D_low + t.batch * d.d_low_each + block_at(row, c0 >> 3, d.ldd);
      const float beta = blocks ? d.beta_low : d.beta;
      uint32_t next[2][8];
      const auto load_ahead = [&](int c, uint32_t* w) {
        if (blocks) load_block(add + c * 32, w);
        else load32_bytes(add + c, w);
      };
      if (add) {
#pragma unroll
        for (int k = 0; k < 2; ++k) if (16 * k < width) load_ahead(16 * k, next[k]);
      }
      if constexpr (PRECISE) {
        // All parts of the sum but the last are added up in registers; then it goes back to where the last part lies.
        constexpr int BLOCKS = TILE_N / GROUPS<PRECISE> / 32;             // (the first half of them in narrow tiles)
        float sum[BLOCKS][32];
        for (int begin = 0;; ++tl) {
          const int end = part_end(d, begin);
          const bool last = end == 3 * d.kb;
          if (!ptx::mbar_wait(&tfull[tl & 1], (tl >> 1) & 1, abort_flag)) { live = false; break; }
          ptx::tc_fence_after();
          const uint32_t t_part = t_quarter + (tl & 1) * TILE_N;
#pragma unroll
          for (int b = 0; b < BLOCKS; ++b) {
            if (b * 32 >= cols) break;
            const uint32_t at = t_part + b * 32;
            float v[32];
            ptx::tmem_ld32(at, v);
            ptx::tmem_ld_wait();
            if (begin == 0) {
#pragma unroll
              for (int i = 0; i < 32; ++i) sum[b][i] = v[i] * (1.f / LOW);
            } else {
#pragma unroll
              for (int i = 0; i < 32; ++i) sum[b][i] += v[i];
            }
            if (last) {
              ptx::tmem_st16(at, sum[b]);
              ptx::tmem_st16(at + 16, sum[b] + 16);
            }
          }
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
      } else {
        if (!ptx::mbar_wait(&tfull[tl & 1], (tl >> 1) & 1, abort_flag)) break;
        ptx::tc_fence_after();
      }
      const uint32_t acc = tl & 1, t_row = t_quarter + acc * TILE_N;
#pragma unroll 1
      for (int c0b = 0; c0b < width; c0b += BOX) {
        if constexpr (!LAST) {
          // the stores before must have read the buffers
          if (lane == 0) ptx::tma_store_wait_read();
          __syncwarp();
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int c = c0b + 16 * k;
          if (c >= width) break;
          float v[16];
          ptx::tmem_ld16(t_row + c, v);
          ptx::tmem_ld_wait();
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] *= d.alpha;
          if (add) {
            add16(v, beta, next[k]);
            if (c + 32 < width) load_ahead(c + 32, next[k]);
            if (PRECISE && !LAST && d.D_low) {
              uint32_t low[8];
              load32_bytes(d.D_low + (add - d.D) + c, low);
              add16(v, d.beta_low, low);
            }
          }
          if (!LAST && d.diagonal != 0.f && row >= c0 + c && row < c0 + c + 16) {
#pragma unroll
            for (int i = 0; i < 16; ++i) if (row == c0 + c + i) v[i] += d.diagonal;
          }
          if constexpr (LAST) {
            float* to = reinterpret_cast<float*>(buf) + lane * TURN_PITCH + 16 * k;
#pragma unroll
            for (int i = 0; i < 16; ++i) to[i] = v[i];
            continue;
          }
          uint32_t w[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            w[i] = pair_half(v[2 * i], v[2 * i + 1]);
            const float2 x = half_pair(w[i]);
            v[2 * i] = (v[2 * i] - x.x) * LOW;
            v[2 * i + 1] = (v[2 * i + 1] - x.y) * LOW;
          }
          stage16(buf, lane, 16 * k, w);
          if (mirror) stage16_turned(buf + (PRECISE ? 2 : 1) * BOX_BYTES, lane, 16 * k, w);
          if (PRECISE || d.C_low) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = pair_half(v[2 * i], v[2 * i + 1]);
            if (!PRECISE) {
              if (in) store_block(d.C_low + t.batch * d.c_low_each + block_at(row, (c0 + c) >> 3, d.ldc), w);
            } else {
              stage16(buf + BOX_BYTES, lane, 16 * k, w);
              if (mirror) stage16_turned(buf + 3 * BOX_BYTES, lane, 16 * k, w);
            }
          }
        }
        if constexpr (LAST) {
          __syncwarp();
          const Target& to = d.target[t.batch];
          const float* turn = reinterpret_cast<const float*>(buf);
          const int rows = d.M - row0;
          if (to.f32) update_rows<true>(to, turn, lane, row0, rows, c0 + c0b, d.N);
          else if (to.even) update_rows_even(to, turn, lane, row0, rows, c0 + c0b, d.N);
          else update_rows<false>(to, turn, lane, row0, rows, c0 + c0b, d.N);
          __syncwarp();
        } else {
          ptx::fence_proxy_async();
          __syncwarp();
          if (lane == 0 && leaves) {
            const int n0 = c0 + c0b;
            const uint32_t from = ptx::smem_u32(buf);
            ptx::tma_store_3d(&d.c, from, n0, row0, t.batch);
            if (PRECISE) ptx::tma_store_3d(&d.c, from + BOX_BYTES, n0, row0, d.count + t.batch);
            if (mirror) {
              ptx::tma_store_3d(&d.c, from + (PRECISE ? 2 : 1) * BOX_BYTES, row0, n0, t.batch);
              if (PRECISE) ptx::tma_store_3d(&d.c, from + 3 * BOX_BYTES, row0, n0, d.count + t.batch);
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

  ptx::tc_fence_before();
  ptx::cluster_sync_all();     // neither CTA leaves while the other may still signal it or read its shared memory
  if (threadIdx.x == 0 && *abort_flag) record_status(p.status, FFSPLIT_ERR_TIMEOUT, blockIdx.x, KID_MUON);
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc_pair(tmem_base, TMEM_COLS);
  }
}

// ---------------------------------------------------------------------------------------------- small squares
// p <= 256: S is one tile, so the pair of CTAs that has summed it can go on to P.  Each CTA rounds its 128 rows of S into shared
// memory, where they are at once its rows of A and its half of the rows of B of the product S S; the sum of S itself has such
// operands too, so X is staged once.  One launch instead of two: 17.1 us an
// iteration on a 256 x 1024 matrix instead of 19.7, 41 instead of 49 on 74 of them; most of what is left is latency.
constexpr int SQUARE_STAGES = 8, SQUARE_STAGE_BYTES = CTA_M * BLOCK_K * 2, SQUARE_S_BYTES = CTA_M * SQUARE_MOST * 2;
constexpr int SQUARE_WARPS = 16, SQUARE_FIRST = 2, SQUARE_THREADS = 32 * (SQUARE_WARPS + SQUARE_FIRST);
constexpr int SQUARE_SMEM = 1024 + SQUARE_STAGES * SQUARE_STAGE_BYTES + SQUARE_S_BYTES + SQUARE_WARPS * BOX_BYTES + BAR_BYTES;
static_assert(SQUARE_STAGES <= MAX_STAGES && SQUARE_SMEM <= MAX_SMEM && SQUARE_MOST == TILE_M, "one tile");
struct DevSquare {
  CUtensorMap x, p;
  int rows, kb, mn, unit0;
  float a, b, c;
};
struct SquareParams {
  DevSquare square[MAX_GROUPS];
  int n;
  int* status;
};

__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(SQUARE_THREADS, 1) muon_square_kernel(const __grid_constant__ SquareParams p) {
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* S = smem + SQUARE_STAGES * SQUARE_STAGE_BYTES;         // [4 blocks of 64 columns][128 rows], 128-byte swizzle
  uint8_t* out_stage = S + SQUARE_S_BYTES;
  uint64_t* bars = reinterpret_cast<uint64_t*>(out_stage + SQUARE_WARPS * BOX_BYTES);
  uint64_t* full = bars;                    // [stages] TMA of both CTAs -> MMA (rank 0's are used)
  uint64_t* empty = full + MAX_STAGES;      // [stages] MMA -> TMA, one set in each CTA
  uint64_t* sums = empty + MAX_STAGES;      // [2] MMA -> epilogue: S, S S, one set in each CTA
  uint64_t* rounded = sums + 2;             // epilogue warps of both CTAs -> MMA (rank 0's is used)
  uint64_t* drain = rounded + 1;            // used only when giving up
  uint32_t* tmem_holder = reinterpret_cast<uint32_t*>(drain + 1);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_holder + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t rank = ptx::cluster_rank();
  const int unit = blockIdx.x >> 1;
  int which = 0;
  while (which + 1 < p.n && unit >= p.square[which + 1].unit0) ++which;
  const DevSquare& d = p.square[which];
  const int batch = unit - d.unit0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < SQUARE_STAGES; ++s) {
      ptx::mbar_init(&full[s], 1);
      ptx::mbar_init(&empty[s], 1);
    }
    for (int a = 0; a < 2; ++a) ptx::mbar_init(&sums[a], 1);
    ptx::mbar_init(rounded, 2 * SQUARE_WARPS);
    ptx::mbar_init(drain, 1);
    *abort_flag = 0;
    ptx::mbar_fence_init();
  }
  if (warp == SQUARE_FIRST && lane == 0) {
    ptx::prefetch_tmap(&d.x);
    ptx::prefetch_tmap(&d.p);
  }
  if (warp == 1) {
    ptx::tmem_alloc_pair(tmem_holder, TMEM_COLS);
    ptx::tmem_relinquish_pair();
  }
  ptx::tc_fence_before();
  ptx::cluster_sync_all();     // also: the other CTA's barriers are set up
  ptx::tc_fence_after();
  const uint32_t tmem_base = *tmem_holder;
  const uint32_t smem0 = ptx::smem_u32(smem), S0 = ptx::smem_u32(S), full0 = ptx::map_to_cta(ptx::smem_u32(full), 0);
  pdl_wait();

  if (warp == 0) {
    if (ptx::elect_one()) {
      // -------------------------------------------------------------- TMA producer
      bool ok = true;
      const int m0 = static_cast<int>(rank) * CTA_M;
      for (int kb = 0; kb < d.kb; ++kb) {
        const int s = kb % SQUARE_STAGES;
        if (!ptx::mbar_wait(&empty[s], ((kb / SQUARE_STAGES) & 1) ^ 1, abort_flag)) { ok = false; break; }
        if (rank == 0) ptx::mbar_expect_tx(&full[s], 2 * SQUARE_STAGE_BYTES);
        const uint32_t to = smem0 + s * SQUARE_STAGE_BYTES, bar = full0 + s * 8;
        if (d.mn) {
          ptx::tma_load_3d_pair(&d.x, to, bar, m0, kb * BLOCK_K, batch);
          ptx::tma_load_3d_pair(&d.x, to + BLOCK64_BYTES, bar, m0 + 64, kb * BLOCK_K, batch);
        } else {
          ptx::tma_load_3d_pair(&d.x, to, bar, kb * BLOCK_K, m0, batch);
        }
      }
      // The last stages: their release arrives here from rank 0, and must find this CTA's barriers still in place.
      for (int i = 0; i < SQUARE_STAGES && i < d.kb && ok; ++i) {
        const int kb = d.kb - 1 - i;
        ok = ptx::mbar_wait(&empty[kb % SQUARE_STAGES], (kb / SQUARE_STAGES) & 1, abort_flag);
      }
      if (!ok) {
        // give the copies in flight a bounded time to land before the CTA exits
        const long long t0 = clock64();
        while (clock64() - t0 < ptx::kWaitLimitCycles / 64) {}
      }
    }
    __syncwarp();
  } else if (warp == 1) {
    if (rank == 0) {
      // -------------------------------------------------------------- MMA issuer (the whole warp walks, one lane issues)
      const uint32_t idesc = ptx::umma_idesc_f16(TILE_M, SQUARE_MOST);
      const uint32_t idesc_x = idesc | (d.mn ? 3u << 15 : 0u);
      const uint64_t desc0 = d.mn ? ptx::umma_desc_mn128(smem0, BLOCK64_BYTES) : ptx::umma_desc_k128(smem0);
      const uint32_t step = d.mn ? 2048 >> 4 : 32 >> 4;
      bool ok = true;
      for (int kb = 0; kb < d.kb; ++kb) {
        const int s = kb % SQUARE_STAGES;
        ok = ptx::mbar_wait_warp(&full[s], (kb / SQUARE_STAGES) & 1, abort_flag);
        if (!ok) break;
        ptx::tc_fence_after();
        const uint64_t x = desc0 + static_cast<uint32_t>(s) * (SQUARE_STAGE_BYTES >> 4);
        if (ptx::elect_one()) {
#pragma unroll
          for (int k = 0; k < BLOCK_K / 16; ++k) ptx::umma_bf16_pair(tmem_base, x + k * step, x + k * step, idesc_x, (kb > 0 || k > 0) ? 1u : 0u);
          ptx::umma_commit_pair(&empty[s]);
        }
        __syncwarp();
      }
      if (ok) {
        if (ptx::elect_one()) ptx::umma_commit_pair(&sums[0]);
        __syncwarp();
        ok = __shfl_sync(0xffffffffu, ptx::mbar_wait_cluster(rounded, 0, abort_flag) ? 1 : 0, 0) != 0;
      }
      if (ok) {
        ptx::tc_fence_after();
        const int blocks = (d.rows + BLOCK_K - 1) / BLOCK_K;
        if (ptx::elect_one()) {
          for (int b = 0; b < blocks; ++b) {
            const uint64_t x = ptx::umma_desc_k128(S0 + b * SQUARE_STAGE_BYTES);
#pragma unroll
            for (int k = 0; k < BLOCK_K / 16; ++k)
              ptx::umma_bf16_pair(tmem_base + TILE_N, x + k * (32 >> 4), x + k * (32 >> 4), idesc, (b > 0 || k > 0) ? 1u : 0u);
          }
          ptx::umma_commit_pair(&sums[1]);
        }
        __syncwarp();
      } else {
        // wait (bounded) until the MMAs issued so far have retired before tensor memory is freed
        if (ptx::elect_one()) {
          ptx::umma_commit_pair(drain);
          const long long t0 = clock64();
          while (!ptx::mbar_try_wait(drain, 0) && clock64() - t0 < ptx::kWaitLimitCycles / 8) {}
        }
        __syncwarp();
      }
    }
  } else {
    // ---------------------------------------------------------------- epilogue warps: 32 rows x one block of 64 columns
    const int q = warp & 3, block = (warp - SQUARE_FIRST) >> 2;
    const int local = q * 32 + lane, row0 = static_cast<int>(rank) * CTA_M + q * 32, row = row0 + lane;
    const uint32_t t_row = tmem_base + (static_cast<uint32_t>(q * 32) << 16) + block * 64;
    uint8_t* s_row = S + block * SQUARE_STAGE_BYTES + local * 128;
    uint8_t* buf = out_stage + (warp - SQUARE_FIRST) * BOX_BYTES;
    if (ptx::mbar_wait(&sums[0], 0, abort_flag)) {
      ptx::tc_fence_after();
#pragma unroll 1
      for (int c = 0; c < 64; c += 16) {
        float v[16];
        ptx::tmem_ld16(t_row + c, v);
        ptx::tmem_ld_wait();
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = pair_half(v[2 * i] * (1.f / HELD), v[2 * i + 1] * (1.f / HELD));
        const int j = c >> 3;
        *reinterpret_cast<uint4*>(s_row + ((j ^ (local & 7)) << 4)) = make_uint4(w[0], w[1], w[2], w[3]);
        *reinterpret_cast<uint4*>(s_row + (((j + 1) ^ (local & 7)) << 4)) = make_uint4(w[4], w[5], w[6], w[7]);
      }
      ptx::fence_proxy_async();
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive_cluster(ptx::map_to_cta(ptx::smem_u32(rounded), 0));
    }
    __syncwarp();
    if (ptx::mbar_wait(&sums[1], 0, abort_flag)) {
      ptx::tc_fence_after();
#pragma unroll 1
      for (int c0 = 0; c0 < 64; c0 += BOX) {
        if (lane == 0) ptx::tma_store_wait_read();
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const int c = c0 + 16 * k, j = c >> 3;
          float v[16];
          ptx::tmem_ld16(t_row + TILE_N + c, v);
          ptx::tmem_ld_wait();
          const uint4 x = *reinterpret_cast<const uint4*>(s_row + ((j ^ (local & 7)) << 4)), y = *reinterpret_cast<const uint4*>(s_row + (((j + 1) ^ (local & 7)) << 4));
          uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
          for (int i = 0; i < 16; ++i) v[i] *= d.c;
          add16(v, d.b, w);
#pragma unroll
          for (int i = 0; i < 16; ++i) if (row == block * 64 + c + i) v[i] += d.a;
#pragma unroll
          for (int i = 0; i < 8; ++i) w[i] = pair_half(v[2 * i], v[2 * i + 1]);
          stage16(buf, lane, 16 * k, w);
        }
        ptx::fence_proxy_async();
        __syncwarp();
        if (lane == 0 && row0 < d.rows && block * 64 + c0 < d.rows) ptx::tma_store_3d(&d.p, ptx::smem_u32(buf), block * 64 + c0, row0, batch);
      }
    }
    if (lane == 0) ptx::tma_store_wait();
    __syncwarp();
  }

  ptx::tc_fence_before();
  ptx::cluster_sync_all();     // neither CTA leaves while the other may still signal it or read its shared memory
  if (threadIdx.x == 0 && *abort_flag) record_status(p.status, FFSPLIT_ERR_TIMEOUT, blockIdx.x, KID_MUON);
  if (warp == 1) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc_pair(tmem_base, TMEM_COLS);
  }
}

// ---------------------------------------------------------------------------------------------- host side
namespace {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// Tensor map over [planes x count][rows][cols]; box of 64 (32) columns by box_rows rows, 128-byte (64-byte) swizzle, zeros
// outside.
ffsplit_status encode(ffsplit_ctx* ctx, const Matrices& m, int box_cols, int box_rows, int planes, CUtensorMap* out) {
  if (!ctx->encode_fn) {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult qres;
    const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres);
    if (e != cudaSuccess || qres != cudaDriverEntryPointSuccess || !fn)
      return fail(ctx, FFSPLIT_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
    ctx->encode_fn = fn;
  }
  // (the second plane follows the first without a gap, so both are one run of matrices)
  cuuint64_t dims[3] = {static_cast<cuuint64_t>(m.cols), static_cast<cuuint64_t>(m.rows), static_cast<cuuint64_t>(m.count) * planes};
  cuuint64_t strides[2] = {static_cast<cuuint64_t>(m.ld) * 2, static_cast<cuuint64_t>(m.each) * 2};
  cuuint32_t box[3] = {static_cast<cuuint32_t>(box_cols), static_cast<cuuint32_t>(box_rows), 1}, estr[3] = {1, 1, 1};
  const CUresult r = reinterpret_cast<EncodeTiledFn>(ctx->encode_fn)(
      out, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, m.p, dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
      box_cols == BOX ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return fail(ctx, FFSPLIT_ERR_CUDA, "cuTensorMapEncodeTiled failed (" + std::to_string((int)r) + ")");
  return FFSPLIT_OK;
}

int tiles_of(const Product& g, int tile_n) {
  const int tm = (g.M + TILE_M - 1) / TILE_M, tn = (g.N + tile_n - 1) / tile_n, step = TILE_M / tile_n;
  if (!g.symmetric) return tm * tn;
  int tiles = 0;
  for (int m = 0; m < tm; ++m) tiles += tn - m * step;
  return tiles;
}

}  // namespace

ffsplit_status launch_products(ffsplit_ctx* ctx, bool precise, const Product* products, int n, cudaStream_t st) {
  // The tensor maps are made by a driver call, which needs a current context (see train_gemm.cu).
  const cudaError_t bound = cudaSetDevice(ctx->device);
  if (bound != cudaSuccess) return check_cuda(ctx, bound, "cudaSetDevice");
  const bool last = products[0].target != nullptr;      // (all of a launch, or none)
  const unsigned bit = 1u << ((precise ? 2 : 0) + (last ? 1 : 0));
  const auto kernel = precise ? (last ? muon_gemm_kernel<true, true> : muon_gemm_kernel<true, false>)
                              : (last ? muon_gemm_kernel<false, true> : muon_gemm_kernel<false, false>);
  if (!(ctx->attr_muon_set & bit)) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, MAX_SMEM);
    if (e != cudaSuccess) return check_cuda(ctx, e, "cudaFuncSetAttribute(muon_gemm_kernel)");
    if (precise) {
      cudaFuncAttributes attr;
      const cudaError_t a = cudaFuncGetAttributes(&attr, kernel);
      if (a != cudaSuccess) return check_cuda(ctx, a, "cudaFuncGetAttributes(muon_gemm_kernel)");
      if (attr.numRegs < START_REGS) return fail(ctx, FFSPLIT_ERR_CUDA, "muon_gemm_kernel was built with fewer registers than it divides");
    }
    ctx->attr_muon_set |= bit;
  }
  Params p;
  std::memset(&p, 0, sizeof(p));
  const int clusters_max = ctx->num_sms / 2;
  // longest sums first
  int order[MAX_GROUPS];
  for (int i = 0; i < n; ++i) {
    int at = i;
    for (; at > 0 && products[order[at - 1]].K < products[i].K; --at) order[at] = order[at - 1];
    order[at] = i;
  }
  // 256 x 128 tiles where the wide ones leave pairs of SMs idle: a k-block takes 0.27 us in a wide tile (the tensor cores'
  // rate) and 0.2 us in a narrow one (shared memory's)
  p.tile_n = TILE_N;
  {
    long long wide = 0, narrow = 0;
    for (int i = 0; i < n; ++i) {
      wide += static_cast<long long>(tiles_of(products[i], 256)) * products[i].c.count;
      narrow += static_cast<long long>(tiles_of(products[i], 128)) * products[i].c.count;
    }
    if (((narrow + clusters_max - 1) / clusters_max) * 0.2 < ((wide + clusters_max - 1) / clusters_max) * 0.27) p.tile_n = 128;
  }
  p.stage_bytes = (CTA_M + p.tile_n / 2) * BLOCK_K * 2;
  bool mirrored = false;
  for (int i = 0; i < n; ++i) mirrored = mirrored || products[i].symmetric;
  p.out_bytes = last ? round_up(TURN_BYTES, 128) : (precise ? 2 : 1) * (mirrored ? 2 : 1) * BOX_BYTES;
  const int room = MAX_SMEM - 1024 - BAR_BYTES - (precise ? EPI_WARPS<true> : EPI_WARPS<false>) * p.out_bytes;
  p.stages = room / p.stage_bytes < MAX_STAGES ? room / p.stage_bytes : MAX_STAGES;
  p.ring_bytes = p.stages * p.stage_bytes;
  long long units = 0;
  for (int i = 0; i < n; ++i) {
    const Product& g = products[order[i]];
    DevProduct& d = p.prod[i];
    ffsplit_status s;
    const int planes = precise ? 2 : 1;
    if ((s = encode(ctx, g.a, BLOCK_K, g.a_mn ? BLOCK_K : CTA_M, planes, &d.a)) != FFSPLIT_OK) return s;
    if ((s = encode(ctx, g.b, BLOCK_K, g.b_mn ? BLOCK_K : p.tile_n / 2, planes, &d.b)) != FFSPLIT_OK) return s;
    if (!g.target && (s = encode(ctx, g.c, BOX, BOX, planes, &d.c)) != FFSPLIT_OK) return s;
    d.M = g.M; d.N = g.N; d.count = g.c.count;
    d.kb = (g.K + BLOCK_K - 1) / BLOCK_K;
    d.promote = g.a.p == g.b.p && g.d ? PROMOTE_POLYNOMIAL : PROMOTE;
    d.a_mn = g.a_mn; d.b_mn = g.b_mn; d.symmetric = g.symmetric;
    d.tiles_m = (g.M + TILE_M - 1) / TILE_M;
    d.tiles_n = (g.N + p.tile_n - 1) / p.tile_n;
    d.tiles = tiles_of(g, p.tile_n);
    d.unit0 = static_cast<int>(units);
    d.alpha = g.alpha; d.beta = g.beta;
    if (g.d) {
      d.D = g.d_high ? g.d->p : nullptr;
      d.D_low = g.d_low ? g.d->low : nullptr;
      d.d_each = g.d->each; d.d_low_each = g.d->low_each; d.ldd = g.d->ld;
    }
    d.beta_low = g.beta * (1.f / LOW);
    d.diagonal = g.diagonal * HELD;
    d.C_low = g.c_low && !precise ? g.c.low : nullptr;
    d.c_low_each = g.c.low_each; d.ldc = g.c.ld;
    d.target = g.target;
    // panel height: the tiles in flight form a block whose two sides carry about the same operand bytes
    d.panel_m = 1;
    double best = 1e300;
    for (int h = 1; h <= d.tiles_m && h <= clusters_max; ++h) {
      const double w = static_cast<double>(clusters_max) / h;
      const double cost = h * 256.0 + (w < d.tiles_n ? w : d.tiles_n) * p.tile_n;
      if (cost < best - 1e-9) { best = cost; d.panel_m = h; }
    }
    units += static_cast<long long>(d.tiles) * d.count;
    if (units > 0x3fffffffll) return fail(ctx, FFSPLIT_ERR_SHAPE, "more than 2^30 tiles in one product");
  }
  p.n = n;
  p.units = static_cast<int>(units);
  p.status = ctx->status();
  const int clusters = units < clusters_max ? static_cast<int>(units) : clusters_max;
  const cudaError_t e = launch_pdl(kernel, dim3(2 * clusters), dim3(precise ? GEMM_THREADS<true> : GEMM_THREADS<false>), MAX_SMEM, st, p);
  ctx->launches++;
  return check_cuda(ctx, e, "muon_gemm_kernel launch");
}

ffsplit_status launch_squares(ffsplit_ctx* ctx, const Gram* squares, int n, cudaStream_t st) {
  const cudaError_t bound = cudaSetDevice(ctx->device);      // (see launch_products())
  if (bound != cudaSuccess) return check_cuda(ctx, bound, "cudaSetDevice");
  if (!(ctx->attr_muon_set & 16u)) {
    const cudaError_t e = cudaFuncSetAttribute(muon_square_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SQUARE_SMEM);
    if (e != cudaSuccess) return check_cuda(ctx, e, "cudaFuncSetAttribute(muon_square_kernel)");
    ctx->attr_muon_set |= 16u;
  }
  SquareParams p;
  std::memset(&p, 0, sizeof(p));
  int units = 0;
  for (int i = 0; i < n; ++i) {
    const Gram& g = squares[i];
    DevSquare& d = p.square[i];
    ffsplit_status s;
    if ((s = encode(ctx, g.X, BLOCK_K, g.mn ? BLOCK_K : CTA_M, 1, &d.x)) != FFSPLIT_OK) return s;
    if ((s = encode(ctx, g.P, BOX, BOX, 1, &d.p)) != FFSPLIT_OK) return s;
    d.rows = g.P.rows;
    d.kb = (g.K + BLOCK_K - 1) / BLOCK_K;
    d.mn = g.mn;
    d.a = g.a * HELD; d.b = g.b; d.c = g.c / HELD;
    d.unit0 = units;
    units += g.P.count;
  }
  p.n = n;
  p.status = ctx->status();
  const cudaError_t e = launch_pdl(muon_square_kernel, dim3(2 * units), dim3(SQUARE_THREADS), SQUARE_SMEM, st, p);
  ctx->launches++;
  return check_cuda(ctx, e, "muon_square_kernel launch");
}

}  // namespace muon
}  // namespace ffsp
