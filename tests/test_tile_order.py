"""Which tile a workgroup of the LDS-tiled kernel takes, on the CPU: the arithmetic of
csrc/tile_order.hpp that the kernel evaluates, compiled by itself.  The number of tiles comes
from the device's map, which holds anything if mm_group_rows did not fill it."""

import pytest

from tests.tile_orders import orders

CUS = 256
COUNTS = [0, 1, 2, 3, 28, 29, 30, 57, 255, 256, 1 << 16, 1 << 20, (1 << 31) - 1, -1, -2, -28, -29, -30, -255, -256, -257,
          -(1 << 16), -(1 << 20), -(1 << 28), -(1 << 29), -(1 << 30), -(1 << 31), 0x00200005, 0x7A7A7A7A, -0x5A5A5A5B,
          0x20202020, -0x20202020] + [-(k * 0x01234567 % (1 << 31)) for k in range(1, 60)]


def _all(tiles_n, listed, counted, whole):
    """(of whole tiles, of quarters)"""
    grid = tiles_n * listed
    tiles, quarters = orders([(grid, tiles_n, listed, counted, whole, False), (2 * CUS, tiles_n, listed, counted, whole, True)])
    return tiles, quarters if whole else []


@pytest.mark.parametrize("whole", [0, CUS])
@pytest.mark.parametrize("listed", [1, 29, 300])
@pytest.mark.parametrize("tiles_n", [1, 2, 3, 4, 5, 16, 22, 56])
def test_tiles_stay_inside_the_list(tiles_n, listed, whole):
    """Whatever the count, every workgroup takes a listed tile of the product, or none."""
    requests = []
    for counted in COUNTS:
        requests.append((tiles_n * listed, tiles_n, listed, counted, whole, False))
        if whole:
            requests.append((2 * CUS, tiles_n, listed, counted, whole, True))
    for request, got in zip(requests, orders(requests)):
        bad = [t for t in got if not (0 <= t[0] < tiles_n and 0 <= t[1] < listed and 0 <= t[2] < 4)]
        assert not bad, (request, bad[:3])


@pytest.mark.parametrize("whole", [0, CUS])
@pytest.mark.parametrize("tiles_n", [1, 2, 3, 4, 5, 16, 22, 56])
def test_every_tile_once(tiles_n, whole):
    """Each of the tiles that there are once: whole, or in its four quarters."""
    for listed in (1, 29, 40):
        for counted in (0, 1, 2, 17, listed, listed + 1, (1 << 31) - 1, -1, -(1 << 30), -(1 << 31)):
            tiles, quarters = _all(tiles_n, listed, counted, whole)
            there = min(max(counted, 0), listed)
            want = sorted((n, m) for n in range(tiles_n) for m in range(there))
            parts = sorted(set(quarters))
            assert len(parts) == len(quarters)
            cut = sorted({(n, m) for n, m, _ in parts})
            assert parts == sorted((n, m, p) for n, m in cut for p in range(4))
            assert sorted([(n, m) for n, m, _ in tiles] + cut) == want, (tiles_n, listed, counted)
