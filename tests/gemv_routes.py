"""The matrix-vector kernel's rule (csrc/gemv_route.hpp) compiled for the host."""

from __future__ import annotations

import functools
import os
import subprocess
import tempfile

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "paper_2508_02343_amd", "csrc", "gemv_route.hpp")
MAIN = """
#include <cstdio>
#include "%s"
int main() {
  long long v[4];
  int cus, steps[3];
  while (scanf("%%lld %%lld %%lld %%lld %%d %%d %%d %%d", v, v + 1, v + 2, v + 3, &cus, steps, steps + 1, steps + 2) == 8) {
    const mm::GemvSizes z = {v[0], v[1], v[2], v[3], cus};
    const mm::GemvPlan p = mm::gemv_plan(z);
    printf("%%d %%d %%d %%lld\\n", p.tn, p.waves, p.in_lds ? 1 : 0, (long long)mm::gemv_workspace_bytes(z, steps));
  }
}
"""


@functools.lru_cache(maxsize=None)
def _program() -> str:
    d = tempfile.mkdtemp(prefix="mm_gemv_")
    src, exe = os.path.join(d, "route.cpp"), os.path.join(d, "route")
    with open(src, "w") as f:
        f.write(MAIN % HEADER)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-o", exe, src], check=True)
    return exe


def plan(rows: int, N: int, split, experts: int = 0, cus: int = 256) -> tuple[int, int, bool, int]:
    """(16-row strips per workgroup, wavefronts, x from LDS, workspace bytes); experts 0: one weight."""
    steps = [-(-(p // 32) // 4) for p in split]
    line = " ".join(str(v) for v in (rows, sum(split), N, experts, cus, *steps))
    out = subprocess.run([_program()], input=line, check=True, capture_output=True, text=True).stdout.split()
    return int(out[0]), int(out[1]), out[2] == "1", int(out[3])


# One case per compiled kernel: (strips, wavefronts, x from LDS), rows, experts (0: one weight), N.  The splits below
# take every case to several batches of steps, with the last one not full.
CASES = [
    ((1, 16, True), 1, 0, 301),
    ((1, 16, False), 9, 0, 301),
    ((2, 16, True), 1, 0, 6001),
    ((2, 16, False), 9, 0, 5003),
    ((2, 8, True), 2, 0, 9001),
    ((2, 8, False), 9, 0, 8301),
    ((2, 4, True), 1, 0, 16999),
    ((2, 4, False), 9, 0, 16411),
    ((1, 16, True), 6, 8, 301),
    ((1, 16, False), 9, 4, 301),
    ((2, 16, True), 6, 8, 1201),
    ((2, 16, False), 9, 4, 801),
    ((2, 8, True), 6, 8, 2303),
    ((2, 8, False), 9, 4, 1501),
    ((2, 4, True), 6, 8, 4001),
    ((2, 4, False), 9, 4, 2501),
]
SPLITS = [(1408, 544, 480), (1440, 0, 0), (0, 1440, 0), (0, 0, 1440)]
