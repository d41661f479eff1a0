// Low-rank adapters on the tensor cores, for batches of more than a few tokens (bf16).
//
// The tokens are sorted by adapter first (a list of indices; nothing moves), so that every tile of 128 rows belongs to one
// adapter.  (One product over tiles as they come, with the rows of other adapters set to zero, would be simpler; but zero
// times an infinity or NaN is NaN, and a broken adapter or token would reach the other requests of its tile.)  Rows are
// gathered by TMA, four to an instruction; rows behind a tile's last token are not loaded, or zeros.
//
//   shrink    P = scale_i V F_i       tiles x ranges of K; the ranges of a tile are a cluster and add up over shared memory
//   expand    Y = base + P F_i        tiles x 128 columns
//   gradient  out_i = V^T P           adapters x 128 columns, over the adapter's tokens
//
// All three read one wide matrix once and are bound by that: with r <= 128 there are at most 2 r operations to an element.
// P is rounded to bf16 between two products (the tensor cores take both operands in one type), as H is in a training pass.
// Every wait is bounded; on expiry the CTA records FFSPLIT_ERR_TIMEOUT, lets its copies and MMAs land and returns.
#include <cstring>

#include "adapter.h"
#include "epilogue.cuh"
#include "ptx.cuh"

namespace ffsp {
namespace adapter {

constexpr int TC_THREADS = 192;         // warps 0 - 3 epilogue (a row of the tile to a lane), 4 copies, 5 issues the MMAs
constexpr int COPY_WARP = 4, MMA_WARP = 5;
constexpr int BLOCK_K = 64, BLOCK64_BYTES = 64 * BLOCK_K * 2;
constexpr int A_BYTES = TOKENS * BLOCK_K * 2, B_BYTES = MAX_RANK * BLOCK_K * 2;

// ---------------------------------------------------------------------------------------------- sorting
// A block to a group: one pass counts its tokens and those of the groups before it, another writes them in their order.
constexpr int SORT_THREADS = 256, SORT_FLIGHT = 4;
// Blocks behind the groups: the entries of a tile of 256 rows.
__device__ __forceinline__ void plan_tile(const int* __restrict__ index, const Sorted& s, int tile) {
  __shared__ __align__(16) int of[EXTENSION_ROWS];
  __shared__ int ids[EXTENSION_ROWS], firsts[EXTENSION_ROWS / 32];
  const int i = threadIdx.x, lane = i & 31, warp = i >> 5;
  const long long t = static_cast<long long>(tile) * EXTENSION_ROWS + i;
  int mine = t < s.T ? __ldg(index + t) : -1;
  if (mine >= s.n) mine = -1;
  of[i] = mine;
  __syncthreads();
  bool first = mine >= 0;
#pragma unroll 4
  for (int k = 0; k < i; k += 4) {
    const int4 q = *reinterpret_cast<const int4*>(of + k);
    first = first && q.x != mine && (k + 1 >= i || q.y != mine) && (k + 2 >= i || q.z != mine) && (k + 3 >= i || q.w != mine);
  }
  const unsigned votes = __ballot_sync(0xffffffffu, first);
  if (lane == 0) firsts[warp] = __popc(votes);
  __syncthreads();
  int before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < EXTENSION_ROWS / 32; ++w) {
    if (w < warp) before += firsts[w];
    all += firsts[w];
  }
  if (first) ids[before + __popc(votes & ((1u << lane) - 1u))] = mine;
  __syncthreads();
  const bool kept = all <= s.most;
  int slot = -1;
  if (kept && mine >= 0)
    for (int k = 0; k < all; ++k) if (ids[k] == mine) slot = k;
  if (t < s.T) s.slot[t] = slot;
  if (i == 0) s.entries[tile] = kept ? all : 0;
  if (!kept) return;
  if (i < all) s.ids[static_cast<long long>(tile) * s.most + i] = ids[i];
}
static_assert(SORT_THREADS == EXTENSION_ROWS, "a thread to a row");
__global__ void __launch_bounds__(SORT_THREADS) sort_kernel(const int* __restrict__ index, Sorted s, int* status) {
  __shared__ int red[2][SORT_THREADS / 32], found[SORT_FLIGHT][SORT_THREADS / 32];
  pdl_wait();
  const int g = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (g > s.n) {
    plan_tile(index, s, g - s.n - 1);
    return;
  }
  if (s.most && g < s.n && threadIdx.x == 0) s.broken[g] = 0;
  const auto group_of = [&](int i) { return i < 0 || i >= s.n ? s.n : i; };
  int mine = 0, before = 0;
  for (long long t0 = threadIdx.x; t0 < s.T; t0 += SORT_THREADS * SORT_FLIGHT) {
    int v[SORT_FLIGHT];
#pragma unroll
    for (int k = 0; k < SORT_FLIGHT; ++k) v[k] = t0 + SORT_THREADS * k < s.T ? group_of(__ldg(index + t0 + SORT_THREADS * k)) : s.n + 1;
#pragma unroll
    for (int k = 0; k < SORT_FLIGHT; ++k) {
      mine += v[k] == g;
      before += v[k] < g;
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    mine += __shfl_xor_sync(0xffffffffu, mine, o);
    before += __shfl_xor_sync(0xffffffffu, before, o);
  }
  if (lane == 0) { red[0][warp] = mine; red[1][warp] = before; }
  __syncthreads();
  mine = before = 0;
#pragma unroll
  for (int w = 0; w < SORT_THREADS / 32; ++w) { mine += red[0][w]; before += red[1][w]; }
  if (threadIdx.x == 0) {
    s.count[g] = mine;
    s.offset[g] = before;
  }
  if (mine == 0) return;
  int at = before;
  for (long long t0 = 0; t0 < s.T; t0 += SORT_THREADS * SORT_FLIGHT) {
    unsigned votes[SORT_FLIGHT];
    bool hit[SORT_FLIGHT];
#pragma unroll
    for (int k = 0; k < SORT_FLIGHT; ++k) {
      const long long t = t0 + SORT_THREADS * k + threadIdx.x;
      const int v = t < s.T ? __ldg(index + t) : 0;
      hit[k] = t < s.T && group_of(v) == g;
      if (hit[k] && v >= s.n) record_status(status, FFSPLIT_ERR_BAD_INDEX, static_cast<int>(t), KID_ADAPTER);
    }
#pragma unroll
    for (int k = 0; k < SORT_FLIGHT; ++k) {
      votes[k] = __ballot_sync(0xffffffffu, hit[k]);
      if (lane == 0) found[k][warp] = __popc(votes[k]);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < SORT_FLIGHT; ++k) {
      int ahead = 0, all = 0;
#pragma unroll
      for (int w = 0; w < SORT_THREADS / 32; ++w) {
        if (w < warp) ahead += found[k][w];
        all += found[k][w];
      }
      if (hit[k]) s.order[at + ahead + __popc(votes[k] & ((1u << lane) - 1u))] = static_cast<int>(t0 + SORT_THREADS * k + threadIdx.x);
      at += all;
    }
    __syncthreads();
  }
}

// A row of blocks to an adapter.  In passing: zeros where the rows of the tiles' entries will be (800 KB for a tile of 24 adapters of
// rank 32: the block that plans the tile took 6 us for that alone).
constexpr int CHECK_CHUNK = 32768;      // elements
__global__ void __launch_bounds__(256) check_kernel(const __nv_bfloat16* __restrict__ F, long long each, Sorted s) {
  pdl_wait();
  const int i = blockIdx.y, tiles = static_cast<int>((s.T + EXTENSION_ROWS - 1) / EXTENSION_ROWS);
  // (as many blocks to a tile as there are, or as many tiles to a block)
  const int blocks = gridDim.x * gridDim.y, block = blockIdx.y * gridDim.x + blockIdx.x, share = blocks > tiles ? blocks / tiles : 1;
  const int entry = EXTENSION_ROWS * s.pitch / 8;
  for (int t = block / share; t < tiles; t += blocks / share) {
    uint4* Q = reinterpret_cast<uint4*>(s.Q) + static_cast<long long>(t) * s.most * entry;
    const int vectors = __ldcg(s.entries + t) * entry;      // (no more than 32 entries)
    for (int k = block % share * 256 + threadIdx.x; k < vectors; k += share * 256) Q[k] = make_uint4(0u, 0u, 0u, 0u);
  }
  if (__ldcg(s.count + i) == 0) return;
  const long long begin = static_cast<long long>(blockIdx.x) * CHECK_CHUNK, end = begin + CHECK_CHUNK < each ? begin + CHECK_CHUNK : each;
  const unsigned short* p = reinterpret_cast<const unsigned short*>(F) + i * each;
  bool bad = false;
  const int lead = static_cast<int>(((16 - (reinterpret_cast<uintptr_t>(p + begin) & 15u)) & 15u) / 2);
  const long long body = begin + lead < end ? begin + lead : end, vectors = (end - body) / 8;
  const uint4* v = reinterpret_cast<const uint4*>(p + body);
#pragma unroll 4
  for (long long k = threadIdx.x; k < vectors; k += 256) {
    const uint4 q = __ldg(v + k);
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) bad = bad || (w[j] & 0x7f80u) == 0x7f80u || (w[j] & 0x7f800000u) == 0x7f800000u;
  }
  if (threadIdx.x < 16) {      // what is left at either end
    const long long k = threadIdx.x < 8 ? begin + threadIdx.x : body + vectors * 8 + threadIdx.x - 8;
    if (k < (threadIdx.x < 8 ? body : end)) bad = bad || (__ldg(p + k) & 0x7f80u) == 0x7f80u;
  }
  if (__syncthreads_or(bad ? 1 : 0) && threadIdx.x == 0) s.broken[i] = 1;
}

struct Tile {
  int group, first, rows;     // the group (-1: no such tile), the place of its first token in the order, its tokens
};
// Tile u of groups 0 .. groups - 1, by one whole warp.
__device__ __forceinline__ Tile find_tile(const Sorted& s, int groups, int u) {
  const int lane = threadIdx.x & 31;
  for (int g0 = 0; g0 < groups; g0 += 32) {
    const int c = g0 + lane < groups ? __ldcg(s.count + g0 + lane) : 0, tiles = (c + TOKENS - 1) / TOKENS;
    int upto = tiles;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += v;
    }
    const unsigned votes = __ballot_sync(0xffffffffu, u < upto);
    if (votes) {
      const int l = __ffs(votes) - 1;
      const int j = u - (__shfl_sync(0xffffffffu, upto, l) - __shfl_sync(0xffffffffu, tiles, l));
      const int count = __shfl_sync(0xffffffffu, c, l) - j * TOKENS;
      return {g0 + l, __ldcg(s.offset + g0 + l) + j * TOKENS, count < TOKENS ? count : TOKENS};
    }
    u -= __shfl_sync(0xffffffffu, upto, 31);
  }
  return {-1, 0, 0};
}
// Tiles of the groups before g.
__device__ __forceinline__ int tiles_before(const Sorted& s, int g) {
  const int lane = threadIdx.x & 31;
  int n = 0;
  for (int i = lane; i < g; i += 32) n += (__ldcg(s.count + i) + TOKENS - 1) / TOKENS;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) n += __shfl_xor_sync(0xffffffffu, n, o);
  return n;
}

// Four rows of 64 columns from x on, one below the other at smem_dst (rows behind the tensor's last one: zeros).
__device__ __forceinline__ void gather4(const CUtensorMap* tm, uint32_t smem_dst, uint32_t bar, int x, const int* rows) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cta.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6, %7}], [%2];" ::"r"(smem_dst),
      "l"(reinterpret_cast<uint64_t>(tm)), "r"(bar), "r"(x), "r"(rows[0]), "r"(rows[1]), "r"(rows[2]), "r"(rows[3])
      : "memory");
}
__device__ __forceinline__ void load_3d(const CUtensorMap* tm, uint32_t smem_dst, uint32_t bar, int x, int y, int z) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];" ::"r"(smem_dst),
               "l"(reinterpret_cast<uint64_t>(tm)), "r"(bar), "r"(x), "r"(y), "r"(z)
               : "memory");
}
// Sixteen tokens of a tile, as a lane loads them: where they lie one after the other as one box, else four to an
// instruction (a gather takes the copy engine nearly as long for four rows as a box for sixteen: 1.4 us for 128 rows).
// Tokens of an adapter are in their order, so a stretch of them is a run if its ends are as far apart as it is long.
constexpr int ROWS = 16;
struct Rows {
  int at[ROWS];
  bool any, run;
};
__device__ __forceinline__ Rows rows_of(const Sorted& s, int first, int rows, int r0) {
  Rows r;
  r.any = r0 < rows;
  r.run = r0 + ROWS <= rows;
  r.at[0] = r.any ? __ldcg(s.order + first + r0) : static_cast<int>(s.T);      // T: behind the last row
  r.at[ROWS - 1] = r.run ? __ldcg(s.order + first + r0 + ROWS - 1) : static_cast<int>(s.T);
  r.run = r.run && r.at[ROWS - 1] == r.at[0] + ROWS - 1;
  if (r.any && !r.run) {
#pragma unroll
    for (int i = 1; i < ROWS; ++i) r.at[i] = r0 + i < rows ? __ldcg(s.order + first + r0 + i) : static_cast<int>(s.T);
  }
  return r;
}
__device__ __forceinline__ void load_2d(const CUtensorMap* tm, uint32_t smem_dst, uint32_t bar, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4}], [%2];" ::"r"(smem_dst),
               "l"(reinterpret_cast<uint64_t>(tm)), "r"(bar), "r"(x), "r"(y)
               : "memory");
}
// 64 columns from x on of the rows to smem_dst, 128 bytes each (without any: zeros).
__device__ __forceinline__ void load_rows(const CUtensorMap* box, const CUtensorMap* gather, uint32_t smem_dst, uint32_t bar, int x, const Rows& r) {
  if (r.run || !r.any) {
    load_2d(box, smem_dst, bar, x, r.at[0]);
  } else {
#pragma unroll
    for (int i = 0; i < ROWS; i += 4) gather4(gather, smem_dst + i * 128, bar, x, r.at + i);
  }
}

// What the three kernels share: barriers, tensor memory, and the way out.
struct Frame {
  uint32_t smem0;             // 1024-byte aligned
  uint64_t *full, *empty, *done, *drain;      // (drain[1]: expand's epilogue warps -> MMA)
  uint32_t tmem;
  volatile int* abort_flag;
};
constexpr int FRAME_BYTES = 256, FRAME_STAGES = 8;
template <int MMA = MMA_WARP>
__device__ __forceinline__ Frame frame_open(uint8_t* raw, int bytes, int stages, uint32_t tmem_cols, int drain_count = 1) {
  Frame f;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  f.smem0 = ptx::smem_u32(smem);
  f.full = reinterpret_cast<uint64_t*>(smem + bytes);
  f.empty = f.full + FRAME_STAGES;
  f.done = f.empty + FRAME_STAGES;
  f.drain = f.done + 1;
  uint32_t* holder = reinterpret_cast<uint32_t*>(f.drain + 2);
  f.abort_flag = reinterpret_cast<volatile int*>(holder + 1);
  if (threadIdx.x == 0) {
    for (int s = 0; s < stages; ++s) {
      ptx::mbar_init(&f.full[s], 1);
      ptx::mbar_init(&f.empty[s], 1);
    }
    ptx::mbar_init(f.done, 1);
    ptx::mbar_init(f.drain, 1);
    ptx::mbar_init(f.drain + 1, drain_count);
    *f.abort_flag = 0;
    ptx::mbar_fence_init();
  }
  if (threadIdx.x >> 5 == MMA) {
    ptx::tmem_alloc(holder, tmem_cols);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  f.tmem = *holder;
  return f;
}
// The MMA warp waits (bounded) for its MMAs, the copy warp gives its copies a bounded time to land, when giving up.
__device__ __forceinline__ void mma_gave_up(const Frame& f) {
  if (ptx::elect_one()) {
    ptx::umma_commit(f.drain);
    const long long t0 = clock64();
    while (!ptx::mbar_try_wait(f.drain, 0) && clock64() - t0 < ptx::kWaitLimitCycles / 8) {}
  }
  __syncwarp();
}
__device__ __forceinline__ void copies_gave_up() {
  const long long t0 = clock64();
  while (clock64() - t0 < ptx::kWaitLimitCycles / 64) {}
}
template <int MMA = MMA_WARP>
__device__ __forceinline__ void frame_close(const Frame& f, uint32_t tmem_cols, int* status) {
  ptx::tc_fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && *f.abort_flag) record_status(status, FFSPLIT_ERR_TIMEOUT, blockIdx.x, KID_ADAPTER);
  if (threadIdx.x >> 5 == MMA) {
    ptx::tc_fence_after();
    ptx::tmem_dealloc(f.tmem, tmem_cols);
  }
}
// One k-block of `steps` MMAs of 16.
__device__ __forceinline__ void issue(uint32_t d, uint64_t a, uint32_t a_step, uint64_t b, uint32_t b_step, uint32_t idesc, int steps, bool first) {
  for (int k = 0; k < steps; ++k) ptx::umma_bf16(d, a + k * a_step, b + k * b_step, idesc, first && k == 0 ? 0u : 1u);
}
__device__ __forceinline__ uint32_t bf16_pair(float x, float y) {
  const __nv_bfloat162 t = __floats2bfloat162_rn(x, y);
  return *reinterpret_cast<const uint32_t*>(&t);
}

// ---------------------------------------------------------------------------------------------- shrink
struct ShrinkDev {
  CUtensorMap V, V_box, V_tile, F;
  __nv_bfloat16* P;
  int kb, f_mn;               // f_mn: the rank runs along memory
  int ranges;                 // of K: no more than a cluster has CTAs
  int extends;
};
struct ShrinkParams {
  ShrinkDev job[2];
  Sorted s;
  const float* scale;
  int r, cols, pitch;         // cols: r rounded up to 16
  int stage;                  // bytes: the rows and 64 or 128 ranks
  int* status;
};
constexpr int SHRINK_STAGES = 4;
constexpr uint32_t SHRINK_TMEM = 128;
static_assert(SHRINK_STAGES * (A_BYTES + B_BYTES / 2) >= TOKENS * (MAX_RANK / 2 + 4) * 4 && SHRINK_STAGES * (A_BYTES + B_BYTES) >= TOKENS * (MAX_RANK + 4) * 4,
              "the partial sums take the place of the ring");

constexpr int MAX_RANGES = 8;

__global__ void __launch_bounds__(TC_THREADS) shrink_tc_kernel(const __grid_constant__ ShrinkParams p) {
  extern __shared__ uint8_t raw[];
  const ShrinkDev& job = p.job[blockIdx.z];
  const int share = gridDim.x, range = blockIdx.x;          // a cluster spans x; behind the last range there is nothing to add up
  if (threadIdx.x == 0) {
    ptx::prefetch_tmap(&job.V_tile);
    ptx::prefetch_tmap(&job.F);
  }
  const Frame f = frame_open(raw, SHRINK_STAGES * p.stage, SHRINK_STAGES, SHRINK_TMEM);     // (under the tail of the kernel before)
  pdl_wait();
  // in passing: the lists of the extension's tiles, now that the factors are checked
  if (p.s.most && blockIdx.x == 0 && blockIdx.z == 0 && threadIdx.x < 32 && blockIdx.y < (p.s.T + EXTENSION_ROWS - 1) / EXTENSION_ROWS) {
    const int e = threadIdx.x, at = blockIdx.y * p.s.most + e;
    const bool in = e < __ldcg(p.s.entries + blockIdx.y);   // (no more than 32)
    const int id = in ? __ldcg(p.s.ids + at) : 0;
    const bool sound = in && __ldcg(p.s.broken + id) == 0;
    const unsigned votes = __ballot_sync(0xffffffffu, sound);
    if (sound) p.s.list[blockIdx.y * p.s.most + __popc(votes & ((1u << e) - 1u))] = id | e << 16;
    if (e == 0) p.s.left[blockIdx.y] = __popc(votes);
  }
  const Tile tile = find_tile(p.s, p.s.n, blockIdx.y);
  if (tile.group < 0) {                                     // (the whole cluster)
    frame_close(f, SHRINK_TMEM, p.status);
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int per = (job.kb + job.ranges - 1) / job.ranges, k0 = range * per, k1 = k0 + per < job.kb ? k0 + per : job.kb;
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~uintptr_t(1023));
  float* part = reinterpret_cast<float*>(smem);
  const int part_pitch = p.cols + 4;
  // A tile that is one run: one box (rows behind its last token are other tokens', and their sums are not written), by the copy
  // warp.  Else every epilogue warp copies its 32 rows (one warp alone took 1.4 us for 128 rows, most of it to issue).
  const int top = __ldcg(p.s.order + tile.first);
  const bool whole = __ldcg(p.s.order + tile.first + tile.rows - 1) - top == tile.rows - 1;
  if (warp == COPY_WARP) {
    // the factor's box: 64 k x 64 ranks, one or two of them; or all ranks (as many rows as there are columns of the tile) x 64 k
    const uint32_t tx = static_cast<uint32_t>((whole ? A_BYTES : (tile.rows + ROWS - 1) / ROWS * (ROWS * 128)) + (job.f_mn ? (p.cols > 64 ? 2 : 1) * BLOCK64_BYTES : p.cols * BLOCK_K * 2));
    bool ok = true;
    for (int kb = k0, i = 0; kb < k1; ++kb, ++i) {
      const int s = i % SHRINK_STAGES;
      ok = ptx::mbar_wait_warp(&f.empty[s], ((i / SHRINK_STAGES) & 1) ^ 1, f.abort_flag);
      if (!ok) break;
      const uint32_t to = f.smem0 + s * p.stage, bar = ptx::smem_u32(&f.full[s]);
      if (ptx::elect_one()) {
        ptx::mbar_expect_tx(&f.full[s], tx);
        if (whole) load_2d(&job.V_tile, to, bar, kb * BLOCK_K, top);
        if (job.f_mn) {
          load_3d(&job.F, to + A_BYTES, bar, 0, kb * BLOCK_K, tile.group);
          if (p.cols > 64) load_3d(&job.F, to + A_BYTES + BLOCK64_BYTES, bar, 64, kb * BLOCK_K, tile.group);
        } else {
          load_3d(&job.F, to + A_BYTES, bar, kb * BLOCK_K, 0, tile.group);
        }
      }
      __syncwarp();
    }
    if (!ok) copies_gave_up();
    __syncwarp();
  } else if (warp == MMA_WARP) {
    const uint32_t idesc = ptx::umma_idesc_bf16(TOKENS, p.cols) | (job.f_mn ? 1u << 16 : 0u);
    bool ok = true;
    for (int kb = k0, i = 0; kb < k1; ++kb, ++i) {
      const int s = i % SHRINK_STAGES;
      ok = ptx::mbar_wait_warp(&f.full[s], (i / SHRINK_STAGES) & 1, f.abort_flag);
      if (!ok) break;
      ptx::tc_fence_after();
      const uint32_t at = f.smem0 + s * p.stage;
      if (ptx::elect_one()) {
        issue(f.tmem, ptx::umma_desc_k128(at), 32 >> 4, job.f_mn ? ptx::umma_desc_mn128(at + A_BYTES, BLOCK64_BYTES) : ptx::umma_desc_k128(at + A_BYTES),
              job.f_mn ? 2048 >> 4 : 32 >> 4, idesc, BLOCK_K / 16, i == 0);
        ptx::umma_commit(&f.empty[s]);
      }
      __syncwarp();
    }
    if (ok) {
      if (ptx::elect_one()) ptx::umma_commit(f.done);
      __syncwarp();
    } else {
      mma_gave_up(f);
    }
  } else {
    const bool any = k0 < k1;
    if (!whole && warp * 32 < tile.rows) {
      // (what these copies bring is counted by the copy warp, before or after them)
      const Rows rows = rows_of(p.s, tile.first, tile.rows, warp * 32 + (lane & 1) * ROWS);
      bool ok = true;
      for (int kb = k0, i = 0; kb < k1; ++kb, ++i) {
        const int s = i % SHRINK_STAGES;
        ok = ptx::mbar_wait_warp(&f.empty[s], ((i / SHRINK_STAGES) & 1) ^ 1, f.abort_flag);
        if (!ok) break;
        if (lane < 2 && rows.any)
          load_rows(&job.V_box, &job.V, f.smem0 + s * p.stage + (warp * 32 + lane * ROWS) * 128, ptx::smem_u32(&f.full[s]), kb * BLOCK_K, rows);
        __syncwarp();
      }
      if (!ok) copies_gave_up();
      __syncwarp();
    }
    if (ptx::mbar_wait(f.done, 0, f.abort_flag)) {
      ptx::tc_fence_after();
      // every copy has landed and every MMA has read it: the ring is free
      for (int c = 0; c < p.cols; c += 16) {
        float v[16];
        ptx::tmem_ld16(f.tmem + (static_cast<uint32_t>(warp * 32) << 16) + c, v);
        ptx::tmem_ld_wait();
        float4* to = reinterpret_cast<float4*>(part + (warp * 32 + lane) * part_pitch + c);
#pragma unroll
        for (int i = 0; i < 4; ++i) to[i] = any ? make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]) : make_float4(0.f, 0.f, 0.f, 0.f);
      }
    }
    __syncwarp();
  }
  __syncwarp();
  ptx::cluster_sync_all();
  // the ranges' sums, in order; every CTA of the cluster takes a share of the tile
  const float scale = p.scale ? __ldg(p.scale + tile.group) : 1.f;
  const int pairs = p.cols / 2;
  __nv_bfloat16* P = job.P + static_cast<long long>(blockIdx.y) * TOKENS * p.pitch;
  const uint32_t part0 = ptx::smem_u32(part);
  for (int e = range * TC_THREADS + threadIdx.x; e < TOKENS * pairs; e += share * TC_THREADS) {
    const int row = e / pairs, c = (e - row * pairs) * 2;
    float x = 0.f, y = 0.f;
    if (row < tile.rows) {
      // (all loads first: each is a trip to another SM)
      float a[MAX_RANGES], b[MAX_RANGES];
#pragma unroll
      for (int k = 0; k < MAX_RANGES; ++k) {
        a[k] = b[k] = 0.f;
        if (k < job.ranges) asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(a[k]), "=f"(b[k]) : "r"(ptx::map_to_cta(part0 + (row * part_pitch + c) * 4, k)));
      }
#pragma unroll
      for (int k = 0; k < MAX_RANGES; ++k) { x += a[k]; y += b[k]; }
    }
    // (zeros behind the rank, where an infinity in the row has met what the factor is filled up with: NaN, which the second
    // product would carry into every column)
    const uint32_t pair = bf16_pair(c < p.r ? scale * x : 0.f, c + 1 < p.r ? scale * y : 0.f);
    *reinterpret_cast<uint32_t*>(P + static_cast<long long>(row) * p.pitch + c) = pair;
    if (job.extends && row < tile.rows) {
      const int token = __ldcg(p.s.order + tile.first + row), slot = __ldcg(p.s.slot + token);
      if (slot >= 0)
        *reinterpret_cast<uint32_t*>(p.s.Q + ((static_cast<long long>(token / EXTENSION_ROWS) * p.s.most + slot) * EXTENSION_ROWS + token % EXTENSION_ROWS) * p.pitch + c) = pair;
    }
  }
  ptx::cluster_sync_all();      // nobody leaves while its sums are read
  frame_close(f, SHRINK_TMEM, p.status);
}

// ---------------------------------------------------------------------------------------------- expand
struct ExpandParams {
  CUtensorMap P, F;
  Sorted s;
  const __nv_bfloat16* base;
  __nv_bfloat16* Y;
  int N, r, f_mn;             // f_mn: the columns run along memory
  int blocks;                 // k-blocks of the rank: 1 or 2
  int rest;                   // rows that the extension has added are left as they are
  int late;                   // the kernel before, which gives base, was launched behind all else that is read here: waited for before base
  int* status;
};
// A CTA keeps a tile's P and goes through every gridDim.x-th block of columns: the factor's next block is on its way while
// one is added.  Two CTAs to an SM keep the loads of base going.
constexpr int EXPAND_COLS = 128, EXPAND_F = EXPAND_COLS * BLOCK_K * 2;
// eight epilogue warps: four quarters of the rows, two halves of the columns
constexpr int EXPAND_WARPS = 8, EXPAND_COPY = 8, EXPAND_MMA = 9, EXPAND_TC_THREADS = 320;
constexpr int TURN_PITCH = 36, TURN_BYTES = 32 * TURN_PITCH * 4 + 32 * 8;      // 32 columns of 32 rows, and where the rows lie
constexpr uint32_t EXPAND_TMEM = 128;

// WIDE: rows start on 8 bytes, and lie within 2^32 pieces of 8 bytes.
template <bool WIDE>
__global__ void __launch_bounds__(EXPAND_TC_THREADS, 2) expand_tc_kernel(const __grid_constant__ ExpandParams p) {
  extern __shared__ uint8_t raw[];
  if (threadIdx.x == 0) {
    ptx::prefetch_tmap(&p.P);
    ptx::prefetch_tmap(&p.F);
  }
  const Frame f = frame_open<EXPAND_MMA>(raw, p.blocks * (A_BYTES + 2 * EXPAND_F), 3, EXPAND_TMEM, EXPAND_WARPS);     // (stages 0, 1: the factor, 2: P)
  if (!p.late) pdl_wait();
  const Tile tile = find_tile(p.s, p.s.n + 1, blockIdx.y);
  const bool none = tile.group == p.s.n;
  bool leave = tile.group < 0 || (none && p.base == p.Y);
  const bool by_slot = p.rest && !leave && __ldcg(p.s.broken + tile.group) == 0;
  const auto done_before = [&](int row) { return by_slot && __ldcg(p.s.slot + __ldcg(p.s.order + tile.first + row)) >= 0; };
  if (by_slot) leave = __syncthreads_or(static_cast<int>(threadIdx.x) < tile.rows && !done_before(threadIdx.x)) == 0;
  if (leave) {
    if (p.late) pdl_wait();
    frame_close<EXPAND_MMA>(f, EXPAND_TMEM, p.status);
    return;
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int all = (p.N + EXPAND_COLS - 1) / EXPAND_COLS;
  const uint32_t factor0 = f.smem0 + p.blocks * A_BYTES;
  if (none) {
    // nothing to add
  } else if (warp == EXPAND_COPY) {
    bool ok = true;
    for (int i = 0, cb = blockIdx.x; cb < all; cb += gridDim.x, ++i) {
      const int s = i & 1;
      ok = ptx::mbar_wait_warp(&f.empty[s], ((i >> 1) & 1) ^ 1, f.abort_flag);
      if (!ok) break;
      if (ptx::elect_one()) {
        if (i == 0) {
          ptx::mbar_expect_tx(&f.full[2], p.blocks * A_BYTES);
          for (int b = 0; b < p.blocks; ++b) load_3d(&p.P, f.smem0 + b * A_BYTES, ptx::smem_u32(&f.full[2]), b * BLOCK_K, blockIdx.y * TOKENS, 0);
        }
        ptx::mbar_expect_tx(&f.full[s], p.blocks * EXPAND_F);
        const uint32_t bar = ptx::smem_u32(&f.full[s]);
        const int n0 = cb * EXPAND_COLS;
        for (int b = 0; b < p.blocks; ++b) {
          const uint32_t to = factor0 + (s * p.blocks + b) * EXPAND_F;
          if (p.f_mn) {
            load_3d(&p.F, to, bar, n0, b * BLOCK_K, tile.group);
            load_3d(&p.F, to + BLOCK64_BYTES, bar, n0 + 64, b * BLOCK_K, tile.group);
          } else {
            load_3d(&p.F, to, bar, b * BLOCK_K, n0, tile.group);
          }
        }
      }
      __syncwarp();
    }
    if (!ok) copies_gave_up();
    __syncwarp();
  } else if (warp == EXPAND_MMA) {
    const uint32_t idesc = ptx::umma_idesc_bf16(TOKENS, EXPAND_COLS) | (p.f_mn ? 1u << 16 : 0u);
    bool ok = ptx::mbar_wait_warp(&f.full[2], 0, f.abort_flag);
    for (int i = 0, cb = blockIdx.x; cb < all && ok; cb += gridDim.x, ++i) {
      const int s = i & 1;
      ok = ptx::mbar_wait_warp(&f.full[s], (i >> 1) & 1, f.abort_flag) && ptx::mbar_wait_warp(f.drain + 1, (i & 1) ^ 1, f.abort_flag);
      if (!ok) break;
      ptx::tc_fence_after();
      if (ptx::elect_one()) {
        for (int b = 0; b < p.blocks; ++b) {
          const uint32_t at = factor0 + (s * p.blocks + b) * EXPAND_F;
          const int left = (p.r - b * BLOCK_K + 15) / 16;
          issue(f.tmem, ptx::umma_desc_k128(f.smem0 + b * A_BYTES), 32 >> 4, p.f_mn ? ptx::umma_desc_mn128(at, BLOCK64_BYTES) : ptx::umma_desc_k128(at),
                p.f_mn ? 2048 >> 4 : 32 >> 4, idesc, left < 4 ? left : 4, b == 0);
        }
        ptx::umma_commit(&f.empty[s]);
        ptx::umma_commit(f.done);
      }
      __syncwarp();
    }
    if (!ok) mma_gave_up(f);
  }
  if (warp < EXPAND_WARPS) {
    // Rows of the tile lie anywhere in the batch: a warp goes along them, four rows of 32 columns to an instruction (with a row
    // to a lane, as tensor memory has them, every load and store fell into 32 lines: 1.3 TB/s).  The sums change places
    // through shared memory; base is on its way before they are complete.
    const int quarter = warp & 3, half = warp >> 2;
    const int rows = tile.rows - quarter * 32 < 32 ? tile.rows - quarter * 32 : 32;       // (may be negative)
    uint8_t* area = raw + (f.smem0 - ptx::smem_u32(raw)) + p.blocks * (A_BYTES + 2 * EXPAND_F) + FRAME_BYTES + warp * TURN_BYTES;
    float* turn = reinterpret_cast<float*>(area);
    long long* row_at = reinterpret_cast<long long*>(area + 32 * TURN_PITCH * 4);
    const int up = lane >> 3, col = (lane & 7) * 4;
    // where this lane's rows 4 k + up lie, in pieces of 8 bytes (from shared memory it was two more loads to four values)
    uint32_t piece[8];
    // (bit 4 k + up: that row is to be written)
    const uint32_t live = __ballot_sync(0xffffffffu, lane < rows && !done_before(quarter * 32 + lane));
    if (WIDE) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const int row = 4 * k + up;
        piece[k] = row < rows ? static_cast<uint32_t>(static_cast<unsigned long long>(__ldcg(p.s.order + tile.first + quarter * 32 + row)) * p.N / 4) : 0u;
      }
    } else {
      row_at[lane] = live >> lane & 1u ? static_cast<long long>(__ldcg(p.s.order + tile.first + quarter * 32 + lane)) * p.N : -1;
    }
    __syncwarp();
    const uint2* base8 = reinterpret_cast<const uint2*>(p.base);
    uint2* Y8 = reinterpret_cast<uint2*>(p.Y);
    if (p.late) pdl_wait();
    for (int i = 0, cb = blockIdx.x; cb < all; cb += gridDim.x, ++i) {
      const int c0 = cb * EXPAND_COLS + half * 64 + col;
      uint2 base[2][8];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int c = c0 + 32 * h;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          base[h][k] = make_uint2(0u, 0u);
          if (WIDE) {
            if (p.base && (live >> (4 * k + up) & 1u) && c < p.N) base[h][k] = base8[static_cast<size_t>(piece[k]) + (c >> 2)];
          } else {
            const long long at = row_at[4 * k + up];
            if (p.base && at >= 0 && c < p.N) {
              const unsigned short* q = reinterpret_cast<const unsigned short*>(p.base + at + c);
              base[h][k].x = q[0] | (c + 1 < p.N ? static_cast<uint32_t>(q[1]) << 16 : 0u);
              base[h][k].y = (c + 2 < p.N ? q[2] : 0u) | (c + 3 < p.N ? static_cast<uint32_t>(q[3]) << 16 : 0u);
            }
          }
        }
      }
      if (!none && !ptx::mbar_wait(f.done, i & 1, f.abort_flag)) break;
      ptx::tc_fence_after();
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int c = c0 + 32 * h;
        if (!none) {
          float v[32];
          ptx::tmem_ld32(f.tmem + (static_cast<uint32_t>(quarter * 32) << 16) + half * 64 + 32 * h, v);
          ptx::tmem_ld_wait();
          float4* to = reinterpret_cast<float4*>(turn + lane * TURN_PITCH);
#pragma unroll
          for (int j = 0; j < 8; ++j) to[j] = make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
        }
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float4 x = none ? make_float4(0.f, 0.f, 0.f, 0.f) : *reinterpret_cast<const float4*>(turn + (4 * k + up) * TURN_PITCH + col);
          const uint2 q = base[h][k];
          const uint32_t lo = bf16_pair(__uint_as_float(q.x << 16) + x.x, __uint_as_float(q.x & 0xffff0000u) + x.y);
          const uint32_t hi = bf16_pair(__uint_as_float(q.y << 16) + x.z, __uint_as_float(q.y & 0xffff0000u) + x.w);
          if (WIDE) {
            if ((live >> (4 * k + up) & 1u) && c < p.N) Y8[static_cast<size_t>(piece[k]) + (c >> 2)] = make_uint2(lo, hi);
          } else {
            const long long at = row_at[4 * k + up];
            if (at >= 0 && c < p.N) {
              unsigned short* o = reinterpret_cast<unsigned short*>(p.Y + at + c);
              o[0] = static_cast<unsigned short>(lo);
              if (c + 1 < p.N) o[1] = static_cast<unsigned short>(lo >> 16);
              if (c + 2 < p.N) o[2] = static_cast<unsigned short>(hi);
              if (c + 3 < p.N) o[3] = static_cast<unsigned short>(hi >> 16);
            }
          }
        }
        __syncwarp();
      }
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(f.drain + 1);      // the accumulator may be written again
    }
    __syncwarp();
  }
  frame_close<EXPAND_MMA>(f, EXPAND_TMEM, p.status);
}

// ---------------------------------------------------------------------------------------------- gradients
struct GradientDev {
  CUtensorMap V, V_box, V_tile, P;
  __nv_bfloat16* out;
  int N, rank_rows, blocks;
};
struct GradientParams {
  GradientDev job[2];
  Sorted s;
  int r, cols, wide;          // wide: r is a multiple of 8
  int apart;                  // the kernel before was launched behind all that is read here, and does not touch what is written: waited for at the end
  int stage;
  uint32_t tmem;              // columns: 128, and as many again for the sum of the parts where there may be several
  int* status;
};
constexpr int GRADIENT_STAGES = 4;
constexpr uint32_t GRADIENT_TMEM = 128;
// An adapter's tokens are summed in parts of so many k-blocks (2^18 tokens), whose sum is rounded.  Tensor cores cut what they add
// at the last place of the running sum, and where all terms have one sign 2^19 of them lose 3.5e-3 of it, 2^20 6e-3.
constexpr int GRADIENT_PART = 4096, GRADIENT_EPI_WARPS = 4;

__global__ void __launch_bounds__(TC_THREADS) gradient_tc_kernel(const __grid_constant__ GradientParams p) {
  extern __shared__ uint8_t raw[];
  const int which = static_cast<int>(blockIdx.x) >= p.job[0].blocks ? 1 : 0, i = blockIdx.y;
  const GradientDev& job = p.job[which];
  const int c0 = (blockIdx.x - (which ? p.job[0].blocks : 0)) * TOKENS;     // 128 columns of V: the rows of the tile
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    ptx::prefetch_tmap(&job.V_tile);
    ptx::prefetch_tmap(&job.P);
  }
  const Frame f = frame_open(raw, GRADIENT_STAGES * p.stage, GRADIENT_STAGES, p.tmem, GRADIENT_EPI_WARPS);
  if (!p.apart) pdl_wait();
  const int count = __ldcg(p.s.count + i), first = __ldcg(p.s.offset + i);
  const int kb = (count + BLOCK_K - 1) / BLOCK_K, parts = kb > GRADIENT_PART ? (kb + GRADIENT_PART - 1) / GRADIENT_PART : 1;
  if (warp == COPY_WARP) {
    const int tile0 = tiles_before(p.s, i);
    const uint32_t tx = A_BYTES + (p.cols > 64 ? 2 : 1) * BLOCK64_BYTES;
    const int top0 = count > 0 ? __ldcg(p.s.order + first) : 0;
    const bool run = count > 0 && __ldcg(p.s.order + first + count - 1) - top0 == count - 1;
    bool ok = true;
    for (int k = 0; k < kb; ++k) {
      const int s = k % GRADIENT_STAGES;
      // a k-block that is one run: one box for each half of the columns
      const int left = count - k * BLOCK_K, top = run ? top0 + k * BLOCK_K : 0;
      const bool whole = run && left >= BLOCK_K;
      Rows rows;
      if (!whole) rows = rows_of(p.s, first + k * BLOCK_K, left, (lane & 3) * ROWS);
      ok = ptx::mbar_wait_warp(&f.empty[s], ((k / GRADIENT_STAGES) & 1) ^ 1, f.abort_flag);
      if (!ok) break;
      const uint32_t to = f.smem0 + s * p.stage, bar = ptx::smem_u32(&f.full[s]);
      if (lane == 0) {
        ptx::mbar_expect_tx(&f.full[s], tx);
        load_3d(&job.P, to + A_BYTES, bar, 0, tile0 * TOKENS + k * BLOCK_K, 0);
        if (p.cols > 64) load_3d(&job.P, to + A_BYTES + BLOCK64_BYTES, bar, 64, tile0 * TOKENS + k * BLOCK_K, 0);
      }
      __syncwarp();
      if (whole) {
        if (lane < 2) load_2d(&job.V_tile, to + lane * BLOCK64_BYTES, bar, c0 + lane * 64, top);
      } else if (lane < 8) {
        load_rows(&job.V_box, &job.V, to + (lane >> 2) * BLOCK64_BYTES + (lane & 3) * (ROWS * 128), bar, c0 + (lane >> 2) * 64, rows);
      }
    }
    if (!ok) copies_gave_up();
    __syncwarp();
  } else if (warp == MMA_WARP) {
    const uint32_t idesc = ptx::umma_idesc_bf16(TOKENS, p.cols) | 1u << 15 | 1u << 16;
    bool ok = true;
    for (int part = 0; part < parts && ok; ++part) {
      const int begin = part * GRADIENT_PART, end = begin + GRADIENT_PART < kb ? begin + GRADIENT_PART : kb;
      if (part > 0) ok = ptx::mbar_wait_warp(f.drain + 1, (part - 1) & 1, f.abort_flag);      // (the part before has been read)
      for (int k = begin; k < end && ok; ++k) {
        const int s = k % GRADIENT_STAGES;
        ok = ptx::mbar_wait_warp(&f.full[s], (k / GRADIENT_STAGES) & 1, f.abort_flag);
        if (!ok) break;
        ptx::tc_fence_after();
        const uint32_t at = f.smem0 + s * p.stage;
        if (ptx::elect_one()) {
          issue(f.tmem, ptx::umma_desc_mn128(at, BLOCK64_BYTES), 2048 >> 4, ptx::umma_desc_mn128(at + A_BYTES, BLOCK64_BYTES), 2048 >> 4, idesc, BLOCK_K / 16, k == begin);
          ptx::umma_commit(&f.empty[s]);
        }
        __syncwarp();
      }
      if (ok) {
        if (ptx::elect_one()) ptx::umma_commit(f.done);
        __syncwarp();
      }
    }
    if (!ok) mma_gave_up(f);
  } else {
    const int col = c0 + warp * 32 + lane;
    const bool in = col < job.N;
    const uint32_t t_row = f.tmem + (static_cast<uint32_t>(warp * 32) << 16);
    // columns c .. c + 15 of the part that is complete, and of those before it
    const auto load_sum = [&](int part, int c, float* v) {
      ptx::tmem_ld16(t_row + c, v);
      ptx::tmem_ld_wait();
      if (part > 0) {
        float before[16];
        ptx::tmem_ld16(t_row + GRADIENT_TMEM + c, before);
        ptx::tmem_ld_wait();
#pragma unroll
        for (int k = 0; k < 16; ++k) v[k] += before[k];
      }
    };
    bool ok = true;
    for (int part = 0; part + 1 < parts && ok; ++part) {
      ok = ptx::mbar_wait_warp(f.done, part & 1, f.abort_flag);
      if (!ok) break;
      ptx::tc_fence_after();
      for (int c = 0; c < p.r; c += 16) {
        float v[16];
        load_sum(part, c, v);
        ptx::tmem_st16(t_row + GRADIENT_TMEM + c, v);
      }
      ptx::tmem_st_wait();
      ptx::tc_fence_before();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(f.drain + 1);
    }
    if (ok && ptx::mbar_wait(f.done, (parts - 1) & 1, f.abort_flag)) {
      ptx::tc_fence_after();
      for (int c = 0; c < p.r; c += 16) {
        float v[16];
        load_sum(parts - 1, c, v);
        if (kb == 0) {
#pragma unroll
          for (int k = 0; k < 16; ++k) v[k] = 0.f;
        }
        if (in && job.rank_rows) {
          __nv_bfloat16* out = job.out + (static_cast<long long>(i) * p.r + c) * job.N + col;
#pragma unroll
          for (int k = 0; k < 16; ++k) if (c + k < p.r) out[static_cast<long long>(k) * job.N] = __float2bfloat16_rn(v[k]);
        } else if (in) {
          __nv_bfloat16* out = job.out + (static_cast<long long>(i) * job.N + col) * p.r + c;
          if (p.wide) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const float* x = v + 8 * h;
              if (c + 8 * h < p.r)
                *reinterpret_cast<uint4*>(out + 8 * h) = make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
            }
          } else {
#pragma unroll
            for (int k = 0; k < 16; ++k) if (c + k < p.r) out[k] = __float2bfloat16_rn(v[k]);
          }
        }
        __syncwarp();
      }
    }
    __syncwarp();
  }
  frame_close(f, p.tmem, p.status);
  if (p.apart) pdl_wait();
}

// ---------------------------------------------------------------------------------------------- host side
namespace {

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

// [planes][rows][cols] with pitch ld: boxes of 64 columns x box_rows, 128-byte swizzle, zeros outside.
ffsplit_status encode(ffsplit_ctx* ctx, const void* at, long long cols, long long rows, long long planes, long long ld, int rank, int box_rows, CUtensorMap* out) {
  if (!ctx->encode_fn) {
    void* fn = nullptr;
    cudaDriverEntryPointQueryResult qres;
    const cudaError_t e = cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &qres);
    if (e != cudaSuccess || qres != cudaDriverEntryPointSuccess || !fn)
      return fail(ctx, FFSPLIT_ERR_CUDA, "cuTensorMapEncodeTiled is not available from the driver");
    ctx->encode_fn = fn;
  }
  cuuint64_t dims[3] = {static_cast<cuuint64_t>(cols), static_cast<cuuint64_t>(rows), static_cast<cuuint64_t>(planes)};
  cuuint64_t strides[2] = {static_cast<cuuint64_t>(ld) * 2, static_cast<cuuint64_t>(ld * rows) * 2};
  cuuint32_t box[3] = {BLOCK_K, static_cast<cuuint32_t>(box_rows), 1}, estr[3] = {1, 1, 1};
  const CUresult r = reinterpret_cast<EncodeTiledFn>(ctx->encode_fn)(
      out, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, static_cast<cuuint32_t>(rank), const_cast<void*>(at), dims, strides, box, estr,
      CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
  if (r != CUDA_SUCCESS) return fail(ctx, FFSPLIT_ERR_CUDA, "cuTensorMapEncodeTiled failed (" + std::to_string((int)r) + ")");
  return FFSPLIT_OK;
}
// Rows one by one, sixteen at a time, and `most` at a time.
ffsplit_status encode_rows(ffsplit_ctx* ctx, const tg::Matrix& m, int most, CUtensorMap* gather, CUtensorMap* box, CUtensorMap* tile) {
  ffsplit_status s = encode(ctx, m.p, m.cols, m.rows, 1, m.ld, 2, 1, gather);
  if (s == FFSPLIT_OK) s = encode(ctx, m.p, m.cols, m.rows, 1, m.ld, 2, ROWS, box);
  return s != FFSPLIT_OK ? s : encode(ctx, m.p, m.cols, m.rows, 1, m.ld, 2, most, tile);
}
ffsplit_status encode_factor(ffsplit_ctx* ctx, const Factor& f, int n, int box_rows, CUtensorMap* out) {
  return encode(ctx, f.m.p, f.cols, f.rows, n, f.m.ld, 3, box_rows, out);
}

inline int expand_smem(int r) { return 1024 + (r > BLOCK_K ? 2 : 1) * (A_BYTES + 2 * EXPAND_F) + FRAME_BYTES + EXPAND_WARPS * TURN_BYTES; }
inline int stage_bytes(int r) { return A_BYTES + (r > 64 ? B_BYTES : B_BYTES / 2); }
inline int smem_of(int stages, int r) { return 1024 + stages * stage_bytes(r) + FRAME_BYTES; }

// The tensor maps are made by a driver call, which needs a current context; and the kernels take more than 48 KB.
ffsplit_status set_up(ffsplit_ctx* ctx) {
  const cudaError_t bound = cudaSetDevice(ctx->device);
  if (bound != cudaSuccess) return check_cuda(ctx, bound, "cudaSetDevice");
  if (ctx->attr_adapter_set) return FFSPLIT_OK;
  cudaError_t e = cudaFuncSetAttribute(shrink_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_of(SHRINK_STAGES, MAX_RANK));
  if (e == cudaSuccess) e = cudaFuncSetAttribute(expand_tc_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, expand_smem(MAX_RANK));
  if (e == cudaSuccess) e = cudaFuncSetAttribute(expand_tc_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, expand_smem(MAX_RANK));
  if (e == cudaSuccess) e = cudaFuncSetAttribute(gradient_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_of(GRADIENT_STAGES, MAX_RANK));
  if (e != cudaSuccess) return check_cuda(ctx, e, "cudaFuncSetAttribute(adapter kernels)");
  ctx->attr_adapter_set = true;
  return FFSPLIT_OK;
}

}  // namespace

ffsplit_status launch_sort(ffsplit_ctx* ctx, const int* index, const Sorted& s, cudaStream_t st) {
  const unsigned blocks = static_cast<unsigned>(s.n + 1 + (s.most ? extension_tiles(s.T) : 0));
  const cudaError_t e = launch_pdl(sort_kernel, dim3(blocks), dim3(SORT_THREADS), 0, st, index, s, ctx->status());
  ctx->launches++;
  return check_cuda(ctx, e, "adapter::sort_kernel launch");
}

ffsplit_status launch_check(ffsplit_ctx* ctx, const void* F, long long each, const Sorted& s, cudaStream_t st) {
  const dim3 grid(static_cast<unsigned>((each + CHECK_CHUNK - 1) / CHECK_CHUNK), s.n);
  const cudaError_t e = launch_pdl(check_kernel, grid, dim3(256), 0, st, static_cast<const __nv_bfloat16*>(F), each, s);
  ctx->launches++;
  return check_cuda(ctx, e, "adapter::check_kernel launch");
}

ffsplit_status launch_shrink_tc(ffsplit_ctx* ctx, const Shrink* jobs, int n, int most_jobs, const Sorted& s, int r, const float* scale, cudaStream_t st) {
  ffsplit_status rc = set_up(ctx);
  if (rc != FFSPLIT_OK) return rc;
  ShrinkParams p;
  std::memset(&p, 0, sizeof(p));
  p.s = s; p.scale = scale; p.r = r; p.cols = round_up(r, 16); p.pitch = rank_pitch(r); p.stage = stage_bytes(r); p.status = ctx->status();
  const long long tiles = tile_bound(s.T, s.n);
  int share = 1;
  for (int i = 0; i < n; ++i) {
    ShrinkDev& d = p.job[i];
    if ((rc = encode_rows(ctx, jobs[i].V, TOKENS, &d.V, &d.V_box, &d.V_tile)) != FFSPLIT_OK) return rc;
    d.f_mn = jobs[i].F.rank_rows ? 0 : 1;
    if ((rc = encode_factor(ctx, jobs[i].F, s.n, d.f_mn ? BLOCK_K : p.cols, &d.F)) != FFSPLIT_OK) return rc;
    d.P = jobs[i].P;
    d.extends = jobs[i].extends;
    d.kb = (jobs[i].K + BLOCK_K - 1) / BLOCK_K;
    // Ranges of K: two CTAs to an SM, four k-blocks each at least (the cluster's exchange takes about as long).  By what is the
    // same whichever gradients are asked for (jobs a call may have, not those it has), so that they do not change each other's bits.
    d.ranges = 1;
    while (d.ranges < MAX_RANGES && d.ranges * tiles * most_jobs < ctx->num_sms && 8 * d.ranges <= d.kb) d.ranges *= 2;
    if (d.ranges > share) share = d.ranges;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(share, static_cast<unsigned>(tiles), n);
  cfg.blockDim = dim3(TC_THREADS);
  cfg.dynamicSmemBytes = smem_of(SHRINK_STAGES, r);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = share;
  attr[1].val.clusterDim.y = 1;
  attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, shrink_tc_kernel, p);
  ctx->launches++;
  return check_cuda(ctx, e, "adapter::shrink_tc_kernel launch");
}

ffsplit_status launch_expand_tc(ffsplit_ctx* ctx, const __nv_bfloat16* P, const Factor& F, int N, const void* base, void* Y, const Sorted& s,
                                int r, bool rest, bool late, cudaStream_t st) {
  ffsplit_status rc = set_up(ctx);
  if (rc != FFSPLIT_OK) return rc;
  ExpandParams p;
  std::memset(&p, 0, sizeof(p));
  const long long tiles = tile_bound(s.T, s.n);
  p.f_mn = F.rank_rows;
  if ((rc = encode(ctx, P, rank_pitch(r), tiles * TOKENS, 1, rank_pitch(r), 3, TOKENS, &p.P)) != FFSPLIT_OK) return rc;
  if ((rc = encode_factor(ctx, F, s.n, p.f_mn ? BLOCK_K : EXPAND_COLS, &p.F)) != FFSPLIT_OK) return rc;
  p.s = s;
  p.base = static_cast<const __nv_bfloat16*>(base); p.Y = static_cast<__nv_bfloat16*>(Y);
  p.N = N; p.r = r; p.rest = rest ? 1 : 0; p.late = late ? 1 : 0; p.status = ctx->status();
  p.blocks = r > BLOCK_K ? 2 : 1;
  // Two CTAs to an SM where there are few tiles, else four blocks of columns to a CTA: its start is paid once, and the last
  // round of CTAs stays short (fourteen blocks each, 342 CTAs on 296 places: 114 us instead of 57).
  const long long blocks = (N + EXPAND_COLS - 1) / EXPAND_COLS, fill = (2 * ctx->num_sms + tiles - 1) / tiles, four = (blocks + 3) / 4;
  // (the rest is most often nothing: CTAs that leave at once)
  const long long wanted = rest ? (fill < four ? fill : four) : fill > four ? fill : four;
  const bool wide = N % 4 == 0 && s.T * (N / 4) <= 0xffffffffll;
  const cudaError_t e = launch_pdl(wide ? expand_tc_kernel<true> : expand_tc_kernel<false>, dim3(static_cast<unsigned>(wanted < blocks ? wanted : blocks), static_cast<unsigned>(tiles)), dim3(EXPAND_TC_THREADS),
                                   expand_smem(r), st, p);
  ctx->launches++;
  return check_cuda(ctx, e, "adapter::expand_tc_kernel launch");
}

ffsplit_status launch_gradients_tc(ffsplit_ctx* ctx, const Gradient* jobs, int n, const Sorted& s, int r, bool apart, cudaStream_t st) {
  ffsplit_status rc = set_up(ctx);
  if (rc != FFSPLIT_OK) return rc;
  GradientParams p;
  std::memset(&p, 0, sizeof(p));
  p.s = s; p.r = r; p.cols = round_up(r, 16); p.wide = r % 8 == 0; p.stage = stage_bytes(r); p.apart = apart ? 1 : 0; p.status = ctx->status();
  p.tmem = s.T > static_cast<long long>(GRADIENT_PART) * BLOCK_K ? 2 * GRADIENT_TMEM : GRADIENT_TMEM;
  int blocks = 0;
  for (int i = 0; i < n; ++i) {
    GradientDev& d = p.job[i];
    if ((rc = encode_rows(ctx, jobs[i].V, BLOCK_K, &d.V, &d.V_box, &d.V_tile)) != FFSPLIT_OK) return rc;
    if ((rc = encode(ctx, jobs[i].P, rank_pitch(r), tile_bound(s.T, s.n) * TOKENS, 1, rank_pitch(r), 3, BLOCK_K, &d.P)) != FFSPLIT_OK) return rc;
    d.out = static_cast<__nv_bfloat16*>(jobs[i].out);
    d.N = jobs[i].N; d.rank_rows = jobs[i].rank_rows;
    d.blocks = (jobs[i].N + TOKENS - 1) / TOKENS;
    blocks += d.blocks;
  }
  const cudaError_t e = launch_pdl(gradient_tc_kernel, dim3(blocks, s.n), dim3(TC_THREADS), smem_of(GRADIENT_STAGES, r), st, p);
  ctx->launches++;
  return check_cuda(ctx, e, "adapter::gradient_tc_kernel launch");
}

}  // namespace adapter
}  // namespace ffsp
