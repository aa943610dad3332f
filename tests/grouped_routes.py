"""The dispatch rule of products grouped by expert (csrc/grouped_route.hpp) compiled
for the host, and one case per compiled kernel: a CPU test states that the rule takes
that kernel, a GPU test runs each with every format set."""

from __future__ import annotations

import functools
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "paper_2508_02343_amd", "csrc", "grouped_route.hpp")
MAIN = """
#include <cstdio>
#include "%s"
int main() {
  mm::GroupedSizes z;
  long long v[6];
  while (scanf("%%lld %%lld %%lld %%d %%d %%d %%d %%lld %%lld %%lld", v, v + 1, v + 2, &z.steps[0], &z.steps[1],
               &z.steps[2], &z.cus, v + 3, v + 4, v + 5) == 10) {
    z.slots = v[0], z.experts = v[1], z.n = v[2];
    for (int k = 0; k < 3; ++k) z.ntiles[k] = v[3 + k];
    const mm::GroupedKernel k = mm::grouped_route(z);
    const char* kind = k <= mm::GroupedKernel::kSplit64x32 ? "split" : "tiled";
    bool found = false;
    for (const mm::GroupedChoice& c : mm::kGroupedChoices)
      if (c.kernel == k) {
        found = true;
        printf("%%s%%dx%%d%%s %%lld %%d\\n", kind, 32 * c.tn, 32 * c.tm,
               k == mm::GroupedKernel::kTiled256x256Rest ? "+rest" : "", (long long)(mm::ceil_div(z.n, 32 * c.tn) * z.ntiles[c.list]),
               c.threads);
      }
    if (!found) puts("none 0 0");
  }
}
"""


@functools.lru_cache(maxsize=None)
def _program() -> str:
    d = tempfile.mkdtemp(prefix="mm_grouped_")
    src, exe = os.path.join(d, "route.cpp"), os.path.join(d, "route")
    with open(src, "w") as f:
        f.write(MAIN % HEADER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-o", exe, src], check=True)
    return exe


def route(slots: int, experts: int, N: int, split, cus: int = 256) -> tuple[str, int, int]:
    """(kernel and tile, tiles in the grid, threads of a workgroup)."""
    most = min(experts, slots)
    groups = (slots + 31 * most) // 32
    ntiles = [min(groups // k + most, groups) for k in (1, 4, 8)]
    steps = [-(-(p // 32) // 4) for p in split]
    line = " ".join(str(v) for v in (slots, experts, N, *steps, cus, *ntiles))
    out = subprocess.run([_program()], input=line, check=True, capture_output=True, text=True).stdout.split()
    return out[0], int(out[1]), int(out[2])


CASES = [  # kernel, slots, experts, N, split
    ("split32x32", 13, 4, 301, (160, 96, 64)),
    ("split64x32", 2900, 3, 150, (224, 64, 96)),
    ("tiled128x128", 4000, 3, 700, (128, 64, 160)),
    ("tiled256x128", 2980, 2, 2300, (160, 64, 192)),
    ("tiled256x256", 4700, 2, 5400, (704, 160, 832)),
    ("tiled256x256+rest", 3000, 2, 5400, (1024, 160, 832)),
]
