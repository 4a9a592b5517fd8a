"""The sizes of the GPU tests reach every team, item and tile that the rules on
sizes can pick (the rules themselves, on the host)."""
import pytest
import torch  # noqa: F401  (its HIP runtime, before the library's)

from test_gpu_i8_tiles import TILES
from test_gpu_norm_items import ITEMS


def test_gradients_of_many_items_reach_every_team(native):
    run = native("norm_items")
    seen = set()
    for rows, C, per in ITEMS:
        for bf16 in (0, 1):
            threads, chunks, alone, items, blocks = map(int, run(rows, C, per, bf16).stdout.split())
            assert items > blocks * (256 // threads if alone else 1), (rows, C, per)
            seen.add((threads, chunks, alone))
    # every team of lanes in both manners, and the block with a row in registers
    teams = [(16, 1), (16, 2), (16, 3), (32, 2), (64, 2), (64, 3)]
    assert seen == {(*t, a) for t in teams for a in (0, 1)} | {(256, c, 0) for c in (1, 2, 4)}


def test_quantised_products_reach_every_tile(native):
    run = native("i8_pick")
    assert sorted(TILES) == list(range(10))
    for tile, sizes in TILES.items():
        assert set(map(int, run(*(v for s in sizes for v in s)).stdout.split())) == {tile}
