"""Which kernel a product grouped by expert takes, on the CPU: the rule of
csrc/grouped_route.hpp, compiled by itself."""

import random

import pytest

from tests.grouped_routes import CASES, route


@pytest.mark.parametrize("kernel,slots,experts,N,split", CASES, ids=str)
def test_every_kernel_is_reached(kernel, slots, experts, N, split):
    assert route(slots, experts, N, split)[0] == kernel


@pytest.mark.parametrize("slots,experts,N", [(2**26, 1024, 64), (2**26, 1, 16000), (2**20, 64, 2**17), (1, 1, (1 << 31) - 1),
                                             (65536, 1024, 2**16)])
def test_grids_stay_below_the_launch_limit(slots, experts, N):
    """A launch has less than 2^32 threads."""
    kernel, tiles, threads = route(slots, experts, N, (32, 0, 0))
    assert kernel == "none" or tiles * threads < 1 << 32


def test_more_tiles_than_a_launch_takes():
    assert route(2**26, 1024, 2**24, (32, 0, 0))[0] == "none"


def test_narrow_weights_take_a_tile_they_fill():
    """A 64-row tile needs 64 padded weight rows."""
    rng = random.Random(3)
    for _ in range(200):
        slots, experts = rng.randint(1, 300), rng.randint(1, 40)
        kernel = route(slots, experts, rng.randint(1, 32), (32 * rng.randint(1, 100), 0, 32))[0]
        assert kernel == "split32x32" or kernel.startswith("tiled"), kernel


