// Adapters' products on the tensor cores, as adapter_tc.cu runs them.  Not part of the public ABI.
#pragma once

#include "train_gemm.h"

namespace ffsp {
namespace adapter {

constexpr int MAX_RANK = 128;
constexpr int TOKENS = 128;             // tokens of a tile: all of one adapter

// The batch sorted by adapter, tokens of one adapter in their order.  Group n holds the tokens without an adapter.
struct Sorted {
  int *count, *offset;      // [n + 1]
  int* order;               // [T]
  int n;
  long long T;
  // The adapters' part of a shared product inside that product (see tg::Extension): entries for the tiles of 256 rows that
  // have no more than `most` adapters.  most = 0: there are none.
  int most;
  int* slot;                // [T]: the entry of each token's adapter in its tile, -1: the tile has no entries
  int *entries, *ids;       // [tiles], [tiles][most]
  int *left, *list;         // the same without broken ones, as tg::Extension has them
  int* broken;              // [n]: an adapter's factor holds an infinity or NaN, which would reach all rows of a tile
  __nv_bfloat16* Q;         // [tiles][most][256][pitch]
  int pitch;
};
constexpr int EXTENSION_ROWS = 256;
inline long long extension_tiles(long long T) { return (T + EXTENSION_ROWS - 1) / EXTENSION_ROWS; }
// Tiles of all groups, group after group: no more than this.
inline long long tile_bound(long long T, int n) { return (T + TOKENS - 1) / TOKENS + (n + 1 < T ? n + 1 : T); }
inline int rank_pitch(int r) { return r <= 64 ? 64 : 128; }

// One of the two factors as an operand: [n][rows][cols], pitch ld; the rank is its rows (rank_rows) or its columns.
struct Factor {
  tg::Matrix m;             // rows = n x rows of one adapter
  int rows, cols, rank_rows;
};

ffsplit_status launch_sort(ffsplit_ctx* ctx, const int* index, const Sorted& s, cudaStream_t st);
// broken[i] of the adapters that are used, from their factors: `each` elements one after the other.
ffsplit_status launch_check(ffsplit_ctx* ctx, const void* F, long long each, const Sorted& s, cudaStream_t st);

// P = scale_i V F_i for every tile: [tiles][128][pitch] bf16, zero rows behind the last token; and into the entries of the
// extension, where the tokens have one.  Up to two at once; most_jobs: as many as calls of this kind may have.
struct Shrink {
  tg::Matrix V;             // [T, K]
  Factor F;
  __nv_bfloat16* P;
  int K;
  int extends;
};
ffsplit_status launch_shrink_tc(ffsplit_ctx* ctx, const Shrink* jobs, int n, int most_jobs, const Sorted& s, int r, const float* scale, cudaStream_t st);

// Y[t] = base[t] + P F_i: [T, N], pitch N.  rest: only the tokens that the extension leaves out.  late: base comes from the launches
// behind the shrink; what else is read here is complete when they start to leave room for this kernel.
ffsplit_status launch_expand_tc(ffsplit_ctx* ctx, const __nv_bfloat16* P, const Factor& F, int N, const void* base, void* Y, const Sorted& s,
                                int r, bool rest, bool late, cudaStream_t st);

// out_i = sum over the adapter's tokens of V[t]^T P[t] ([n][N][r], rank_rows: its transpose, [n][r][N]).  Up to two at once.
struct Gradient {
  tg::Matrix V;             // [T, N]
  const __nv_bfloat16* P;
  void* out;
  int N, rank_rows;
};
ffsplit_status launch_gradients_tc(ffsplit_ctx* ctx, const Gradient* jobs, int n, const Sorted& s, int r, bool apart, cudaStream_t st);

}  // namespace adapter
}  // namespace ffsp
