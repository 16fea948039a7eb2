// What the kernels of the paged attention share, and their launchers.
#pragma once
#include "serving_device.h"

namespace rf {

// A tile's entry in the workspace, for the launch that joins its chunks.
struct JoinTile {
  int chunks;  // 1: nothing to join
  int slot;    // of its first chunk's states
  int row;     // its first row among all packed rows (token * group + head of the group)
  int rows;
};

// One launch's work: its share of the batch, and where it keeps the states of tiles in several chunks: for slot s, KV
// head h and row r of the tile, part_m, part_l [s][h][r] and part_acc [s][h][r][d].
struct PagedArgs {
  Paged p;
  Deal deal;
  const bf16_t* q;
  const unsigned char *k, *v;
  bf16_t* o;
  Strides2 sq, so;
  float scale_log2e, v_scale;
  int causal;
  int n_tiles, n_units;  // entries of `tiles`; shares that there may be
  float *part_acc, *part_m, *part_l;  // the maximum in log2 units; the sums not normalised
  JoinTile* tiles;
};

// Writes the entry of the share's tile (or, where the batch has no such share, of one of the tiles that it does not
// have either).  One wavefront of the workgroups of KV head 0 calls it.
__device__ __forceinline__ void note_tile(const PagedArgs& a, int unit, bool found, const Share& w) {
  if (a.deal.round == 0 || (threadIdx.x & 63) != 0) return;
  if (found) {
    const int R = 1 << a.deal.rows_log2, r0 = w.tile << a.deal.rows_log2;
    if (w.chunk == 0)
      a.tiles[w.tile_index] = JoinTile{w.chunks, w.slot, w.s.row0 * a.p.group + r0, min(R, w.s.n * a.p.group - r0)};
  } else {
    // (units past the last share are at least as many as tiles past the last tile: a launch has n_tiles + target units,
    // and shares are at most `target` more than tiles; or n_tiles times the most chunks that a tile can have)
    const int64_t at = (int64_t)unit - w.all_shares + w.all_tiles;
    if (at < a.n_tiles) a.tiles[at] = JoinTile{1, 0, 0, 0};
  }
}

// Workgroups of a launch, for the shares that there may be (of few rows: whole turns over the 8 XCDs).
inline int64_t rows_blocks(const PagedArgs& a) { return ((int64_t)a.n_units + 7) / 8 * 8 * a.p.Hkv; }
inline int64_t tiles_blocks(const PagedArgs& a) { return (int64_t)a.n_units * a.p.Hkv; }

hipError_t launch_paged_rows(const PagedArgs& a, bool fp8, hipStream_t s);   // tiles of 16 or 32 rows
hipError_t launch_paged_tiles(const PagedArgs& a, bool fp8, hipStream_t s);  // tiles of 128 rows
hipError_t launch_paged_both(const PagedArgs& few, const PagedArgs& many, bool fp8, hipStream_t s);  // of 16, of 128
constexpr int kTilesRowsLog2 = 7;

}  // namespace rf
