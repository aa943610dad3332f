"""The order of the LDS-tiled kernel's tiles (csrc/tile_order.hpp) compiled for the host."""

from __future__ import annotations

import functools
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "paper_2508_02343_amd", "csrc", "tile_order.hpp")
MAIN = """
#include <cstdio>
#include "%s"
int main() {
  int first, last, tiles_n, listed, counted, whole, rest;
  while (scanf("%%d %%d %%d %%d %%d %%d %%d", &first, &last, &tiles_n, &listed, &counted, &whole, &rest) == 7) {
    for (int wg = first; wg < last; ++wg) {
      const mm::GridTile t = mm::grouped_tile(wg, tiles_n, listed, counted, whole, rest != 0);
      if (t.live) printf("%%d %%d %%d ", t.tn, t.tm, t.part);
    }
    puts("");
  }
}
"""


@functools.lru_cache(maxsize=None)
def _program() -> str:
    d = tempfile.mkdtemp(prefix="mm_tiles_")
    src, exe = os.path.join(d, "order.cpp"), os.path.join(d, "order")
    with open(src, "w") as f:
        f.write(MAIN % HEADER)
    # -fwrapv: sums and products past 32 bits wrap, as they do on the GPU
    subprocess.run(["g++", "-std=c++17", "-O1", "-fwrapv", "-Wall", "-Werror", "-o", exe, src], check=True)
    return exe


def orders(requests) -> list[list[tuple[int, int, int]]]:
    """For each (workgroups, tiles_n, listed, counted, whole, of_rest) the (tn, tm, part) of the
    workgroups that have a tile."""
    lines = "\n".join(f"0 {n} {' '.join(str(int(v)) for v in r)}" for n, *r in requests)
    out = subprocess.run([_program()], input=lines, check=True, capture_output=True, text=True).stdout.splitlines()
    assert len(out) == len(requests)
    values = [[int(v) for v in line.split()] for line in out]
    return [list(zip(v[0::3], v[1::3], v[2::3])) for v in values]
