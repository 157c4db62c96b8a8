"""Limits of the 8-bit path: what the library accepts fits the grids that it launches (host code alone)."""
import ctypes
import random

import pytest

from paper_2504_02658_amd import api

WIDE_32x64, TILE_128x256 = 4, 8
GRID = 1 << 22          # workgroups of 512 threads: 2^31 work items


@pytest.fixture(scope="module")
def L():
    lib = api.lib()
    lib.milo_moe_w8a8_route.argtypes = [ctypes.c_int64] * 3 + [ctypes.c_int] * 2
    return lib


def grids(kernel, T, H, F, E, topk):
    """Workgroups of both grouped products: a slot for every tile of the pairs and one per expert."""
    rows, up, down = (32, 32, 64) if kernel == WIDE_32x64 else (128, 128, 256)
    slots = -(-T * topk // rows) + E
    return slots * -(-F // up), slots * -(-H // down)


def test_layers_of_many_experts_take_the_kernel_whose_grid_fits(L):
    for shape in ((17, 128, 131072, 1024, 1), (17, 64, 16384, 8192, 1)):        # just beyond with the small tiles: 2^22 and one slot's more
        assert L.milo_moe_w8a8_workspace(*shape) > 0
        assert max(grids(WIDE_32x64, *shape)) > GRID >= max(grids(TILE_128x256, *shape))
        assert L.milo_moe_w8a8_route(*shape) == TILE_128x256
    for shape in ((17, 131072, 128, 1024, 1), (17, 128, 131072, 1023, 1), (17, 64, 16384, 8191, 1)):
        assert max(grids(WIDE_32x64, *shape)) <= GRID and L.milo_moe_w8a8_route(*shape) == WIDE_32x64


def test_layers_of_more_tiles_than_a_grid_are_refused_at_once(L):
    T, H, F, topk = (1 << 19) - 64, 1 << 13, 128, 64
    shape = (T, H, F, 64, topk)
    assert grids(TILE_128x256, *shape)[1] > GRID
    need = L.milo_moe_w8a8_workspace(*shape)
    p = ctypes.c_void_p(0x10000)        # (refused before anything is launched)
    assert need == 0 and L.milo_moe_w8a8_route(*shape) == -2
    assert L.milo_moe_w8a8_forward(p, T, H, F, p, 64, p, p, topk, 0, p, p, p, 1 << 60, None) == 2
    half = (T // 2, H, F, 64, topk)
    assert grids(TILE_128x256, *half)[1] > GRID and L.milo_moe_w8a8_workspace(*half) == 0       # 64 slots more than 2^22 / 32
    less = (T // 2 - 2048, H, F, 64, topk)
    assert grids(TILE_128x256, *less)[1] <= GRID and L.milo_moe_w8a8_workspace(*less) > 0


def test_every_accepted_layer_fits_its_grids(L):
    rng = random.Random(5)
    seen = set()
    for _ in range(20000):
        side = lambda top: min(top, max(1, int(2 ** rng.uniform(0, top.bit_length())) + rng.choice((-1, 0, 0, 1))))
        E = side(65536)
        shape = (side(1 << 23), side(1 << 17), side(1 << 17), E, min(E, side(64)))
        kernel = L.milo_moe_w8a8_route(*shape)
        assert (kernel == -2) == (L.milo_moe_w8a8_workspace(*shape) == 0)
        if kernel >= 0:
            assert max(grids(kernel, *shape)) <= GRID, shape
        seen.add(kernel)
    assert seen == {-2, -1, WIDE_32x64, TILE_128x256}
