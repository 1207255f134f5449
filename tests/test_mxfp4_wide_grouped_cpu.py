"""Grouped MXFP4 products with few rows an expert and so many columns that a workgroup a tile would be more than a grid holds
(2^32 threads) take a kernel whose workgroups walk over the tiles."""
import pytest

import paper_2412_19437_amd as pkg

# workgroups of 256 threads a tile, and the tile's weight rows and rows, of the configurations without a walk
ONE_TILE_EACH = {8: (64, 32), 9: (128, 64), 10: (64, 64)}


@pytest.mark.parametrize("G,M,N", [(1023, 24 * 1023, 600_064), (64, 256, 14_950_016), (64, 64, 16_777_280), (1023, 48 * 1023, 1_500_000), (1023, 1023, 4_194_304),
                                   (1, 24, (1 << 29) - 1), (2, 40, 1 << 28)])
def test_every_grid_is_one_that_can_be_launched(G, M, N):
    config = pkg._L().ds3_gemm_mxfp4_config(G, M, N, 128, 256)
    assert 8 <= config <= 13
    if config in ONE_TILE_EACH:
        bn, bm = ONE_TILE_EACH[config]
        tiles = min(-(-M // bm) + G, M) * -(-N // bn)
        assert -(-tiles // 8) * 8 * 256 < 1 << 32
