// Host-visible argument structs and launchers of the kernels that work on rows
// ordered by expert, and of the matrix-vector kernel.
#pragma once

#include "gemv_route.hpp"
#include "kernels.hpp"

namespace mm {

constexpr int64_t kMaxExperts = 1024;  // a workgroup keeps one count per expert and wavefront in LDS
constexpr int64_t kMaxGroupedRows = (int64_t)1 << 26;

// One tile of an expert's rows: its first packed row group, and its expert (low
// 16 bits) with the number of its rows that hold a slot (high 16 bits).  Row
// group -1: no tile.
struct RowTile {
  int32_t first;
  uint32_t owner_rows;
};

// A tile's expert and rows.  A map that mm_group_rows did not fill holds anything: a
// tile that is not one (no rows, or outside of what the map and the weights hold) is
// passed over, so that the calls stay in bounds.
struct TileRows {
  int expert, rows;
};
__device__ __forceinline__ TileRows tile_rows(const RowTile& t, int most, int64_t capacity, int experts) {
  const TileRows r = {(int)(t.owner_rows & 0xFFFF), (int)(t.owner_rows >> 16)};
  const bool is = t.first >= 0 && r.rows > 0 && r.rows <= most && r.expert < experts &&
                  (int64_t)t.first * kRowGroup + r.rows <= capacity;
  return is ? r : TileRows{0, 0};
}

// Tiles of these many rows are listed.
constexpr int kTileLists = 3;
constexpr int kTileRows[kTileLists] = {32, 128, 256};

// group_rows: one workgroup of 1024 threads up to kGroupChunk slots, above one for
// every 1024 slots, at most kGroupMaxBlocks.
constexpr int64_t kGroupThreads = 1024;
constexpr int64_t kGroupChunk = 4096;
constexpr int64_t kGroupMaxBlocks = 128;

// The words (int32) of a row-group map (include/micromix.h): starts, slots and
// owners, then the tile lists and the workgroups' counts.
struct GroupLayout {
  int64_t capacity;          // packed rows
  int64_t slots, owners;     // word offsets
  int64_t tiles[kTileLists], ntiles[kTileLists];
  int64_t tile_counts;       // [kTileLists]: tiles in each list
  int64_t counts, blocks;    // [blocks, experts], only with more than one workgroup
  int64_t words;
};

inline GroupLayout group_layout(int64_t rows, int64_t experts) {
  auto round4 = [](int64_t v) { return (v + 3) / 4 * 4; };
  GroupLayout l;
  const int64_t most = experts < rows ? experts : rows;  // experts that can have rows
  l.capacity = (rows + (kRowGroup - 1) * most) / kRowGroup * kRowGroup;
  const int64_t groups = l.capacity / kRowGroup;
  l.slots = round4(experts + 1);
  l.owners = l.slots + l.capacity;
  int64_t at = l.owners + round4(groups);
  for (int k = 0; k < kTileLists; ++k) {
    l.tiles[k] = at;
    // sum over experts of ceil(their groups / groups per tile): no more than this,
    // and than the groups
    const int64_t n = groups / (kTileRows[k] / kRowGroup) + most;
    l.ntiles[k] = n < groups ? n : groups;
    at += round4(2 * l.ntiles[k]);
  }
  const int64_t b = rows <= kGroupChunk ? 1 : (rows + kGroupThreads - 1) / kGroupThreads;
  l.blocks = b > kGroupMaxBlocks ? kGroupMaxBlocks : b;
  l.tile_counts = at;
  at += round4(kTileLists);
  l.counts = at;
  if (l.blocks > 1) at += round4(l.blocks * experts);
  l.words = at;
  return l;
}

struct GroupArgs {
  const int32_t* ids;
  int64_t rows;
  int experts;
  int32_t *starts, *slots, *owners, *tile_counts, *counts;
  RowTile* tiles[kTileLists];
  int ntiles[kTileLists];
  int groups;   // row groups of the capacity
  int blocks;   // workgroups
  int turns;    // ids per thread: a wavefront takes 64 * turns consecutive slots
};
hipError_t launch_group_rows(const GroupArgs& a, const Device& dev, hipStream_t stream);

// Quantiser over packed rows: row p takes slot slots[p] (none: nothing is
// written), that is row slot / top_k of x.
struct QuantGroupedArgs {
  QuantArgs q;  // rows = rp = capacity; perm expert 0's
  int64_t perm_stride;
  uint32_t top_k;
  const int32_t *starts, *slots;
  const RowTile* tiles;  // of one row group
  int experts;
  uint32_t rows;         // slots
};
hipError_t launch_quantize_grouped(const QuantGroupedArgs& a, const Device& dev, hipStream_t stream);

// Bytes from one expert's weight to the next in each of its buffers.
struct ExpertStride {
  int64_t q[3], sc;
};

struct GemmGroupedArgs {
  GemmArgs g;  // w: expert 0; x: the packed rows
  ExpertStride next;
  const int32_t* slots;
  const RowTile* tiles[kTileLists];
  int ntiles[kTileLists];  // bounds that the host knows
  const int32_t* counts;   // [kTileLists] tiles that there are
  int64_t rows;  // slots
  int experts;
};
// tiles of bn weight rows by bm rows: 128 x 128, 256 x 128, 256 x 256 (rest: a last round that
// is at most half full in quarters, by a launch of its own)
hipError_t launch_gemm_tiled_grouped(const GemmGroupedArgs& a, int bn, int bm, bool rest, const Device& dev,
                                     hipStream_t stream);
// 64 x 32 (weights of at least 64 padded rows), else 32 x 32
hipError_t launch_gemm_split_grouped(const GemmGroupedArgs& a, bool wide, const Device& dev, hipStream_t stream);

struct GemvArgs {
  const uint16_t* x;
  int64_t ldx;
  int rows;
  int top_k;
  const int32_t* perm;
  int64_t perm_stride;
  Operand w;  // expert 0
  ExpertStride next;
  int experts;
  const int32_t* ids;  // null: every row takes weight 0
  int K;
  int nb[3], steps[3];
  uint16_t* y;
  int64_t ldy;
  int fs;
  void* workspace;  // gemv_workspace_bytes
};
hipError_t launch_gemv(const GemvArgs& a, const Device& dev, hipStream_t stream);

}  // namespace mm
