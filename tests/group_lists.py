"""The tile lists of a row-group map (csrc/grouped.hpp): where they lie in its words, and what
they hold by their definition."""

from __future__ import annotations

import numpy as np

TILE_ROWS = (32, 128, 256)


def _round4(v: int) -> int:
    return (v + 3) // 4 * 4


def layout(rows: int, experts: int) -> dict:
    """Word offsets: tiles (three lists of two words a tile), their lengths ntiles, tile_counts, counts;
    words in all."""
    most = min(experts, rows)
    capacity = 32 * ((rows + 31 * most) // 32)
    groups = capacity // 32
    slots = _round4(experts + 1)
    owners = slots + capacity
    at, tiles, ntiles = owners + _round4(groups), [], []
    for r in TILE_ROWS:
        n = min(groups // (r // 32) + most, groups)
        tiles.append(at)
        ntiles.append(n)
        at += _round4(2 * n)
    tile_counts = at
    counts = at + _round4(len(TILE_ROWS))
    blocks = 1 if rows <= 4096 else min(-(-rows // 1024), 128)
    words = counts + (_round4(blocks * experts) if blocks > 1 else 0)
    return {"capacity": capacity, "slots": slots, "owners": owners, "tiles": tiles, "ntiles": ntiles,
            "tile_counts": tile_counts, "counts": counts, "words": words}


def lists(ids: np.ndarray, experts: int) -> list[np.ndarray]:
    """For each of TILE_ROWS int32 [tiles, 2]: a tile's first row group, and its expert with its rows
    that hold a slot above 16 bits; expert by expert."""
    valid = ids[(ids >= 0) & (ids < experts)]
    per = np.bincount(valid, minlength=experts)
    out = []
    for r in TILE_ROWS:
        tiles, first = [], 0
        for e, n in enumerate(per.tolist()):
            tiles += [(first + at // 32, e | min(n - at, r) << 16) for at in range(0, n, r)]
            first += -(-n // 32)
        out.append(np.array(tiles, np.int32).reshape(-1, 2))
    return out
