// Which tile of a product a workgroup of the LDS-tiled kernel computes.  Whole-number
// arithmetic only, no HIP: the kernels evaluate it, tests compile it by itself.
#pragma once

namespace mm {

struct GridTile {
  bool live;   // false: the workgroup has none
  int tn, tm;  // weight tile, activation tile
  int part;    // of_rest: quarter of the tile
};

// How many of nt tiles are not left to the quarters of a tile: behind whole rounds over
// `whole` CUs (0: no quarters) a last round that is at most half full.
constexpr int in_rounds(int nt, int whole) {
  const int rest = whole ? nt % whole : 0;
  return 2 * rest <= whole ? nt - rest : nt;
}

// Consecutive ones of nt tiles per XCD (workgroups are dealt to the 8 XCDs round-robin).
constexpr int tile_of_xcd(int wg, int nt) {
  const int xcd = wg & 7, k = wg >> 3;
  const int per_x = nt >> 3, extra = nt & 7;
  return xcd * per_x + (xcd < extra ? xcd : extra) + k;
}

// Tile t of tiles_n x tiles_m: groups of four weight tiles (they share an XCD's L2 at a
// time), activation tiles fastest inside a group.
constexpr GridTile tile_in_order(int t, int part, int tiles_n, int tiles_m) {
  constexpr int kGroupN = 4;
  const int grp = t / (kGroupN * tiles_m);
  const int within = t - grp * kGroupN * tiles_m;
  const int gn = tiles_n - grp * kGroupN < kGroupN ? tiles_n - grp * kGroupN : kGroupN;
  return GridTile{true, grp * kGroupN + within % gn, within / gn, part};
}

// Workgroup wg of a product over a list of activation tiles: `listed` ones have a place
// in it, `counted` is how many it says there are: any number in a map that
// mm_group_rows did not fill, so it is limited on both sides before it is used.  of_rest:
// of the launch for the quarters of the tiles that in_rounds leaves.
constexpr GridTile grouped_tile(int wg, int tiles_n, int listed, int counted, int whole, bool of_rest) {
  const int tiles_m = counted < 0 ? 0 : (counted < listed ? counted : listed);
  const int nt = tiles_n * tiles_m, rounds = in_rounds(nt, whole);
  if (of_rest) {
    const int parts = 4 * (nt - rounds);
    if (wg >= parts) return GridTile{false, 0, 0, 0};
    const int t = tile_of_xcd(wg, parts);
    return tile_in_order(rounds + (t >> 2), t & 3, tiles_n, tiles_m);
  }
  if (wg >= rounds) return GridTile{false, 0, 0, 0};
  return tile_in_order(tile_of_xcd(wg, rounds), 0, tiles_n, tiles_m);
}

}  // namespace mm
