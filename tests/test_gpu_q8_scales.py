"""The 8-bit experts (xmoe_q8.hip): scales of either sign."""
import numpy as np
import pytest
import torch

from test_gpu_q8 import ROWS, call, check, make, tile_rows

pytestmark = pytest.mark.gpu
TILES = {32: "few", 128: "middle", 256: "long"}


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("tile", TILES)
def test_scales_of_either_sign(tile, dt):
    import paper_2508_13337_amd as m
    c = make(ROWS[TILES[tile]], 384, 712, True, seed=11)
    assert tile_rows(c) == tile
    g = np.random.default_rng(5)
    for s in (c["xs"], c["ws"][0], c["ws"][1]):
        s *= g.choice(np.float32([-1, 1]), s.shape)
    assert min((s < 0).sum() for s in (c["xs"], c["ws"][0], c["ws"][1])) > 0
    check(c, call(m, c, dt), dt)
