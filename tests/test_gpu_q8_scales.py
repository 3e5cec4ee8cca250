"""The 8-bit experts (xmoe_q8.hip): scales of either sign, the accuracy of the activation's integers, small activations.

Beside the derivation in test_gpu_q8.py, u = 2^-24: A is float32 up to the rounding to its row's 127 steps.  The exponent of
silu takes 4 roundings, which move A by 4 |G| u relative to it, with |G| below 40; exp2 and the reciprocal are good to 2 u,
and the sum under it, the gate factor (4), the up factor (3), the two products, the row's scale and 127 / maximum (2) take
one u each: 4 * 40 + 17 = 177 u, 180 u bounds it."""
import numpy as np
import pytest
import torch

import test_gpu_q8 as q8
from test_gpu_q8 import ROWS, U, call, check, make, tile_rows

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


@pytest.mark.parametrize("f", [712, 1409])
@pytest.mark.parametrize("tile", TILES)
def test_the_activations_integers(tile, f, monkeypatch):
    """They differ from the oracle's only as near to a tie as float32 arithmetic is good to."""
    import paper_2508_13337_amd as m
    c = make(ROWS[TILES[tile]], 384, f, False, seed=12)
    assert tile_rows(c) == tile
    monkeypatch.setattr(q8, "NEAR", 127 * 180 * U)
    check(c, call(m, c, torch.float32), torch.float32)


@pytest.mark.parametrize("tile", TILES)
def test_small_activations(tile):
    """Rows whose largest A is 2^-120 or more keep their values, those below count as zero."""
    import paper_2508_13337_amd as m
    c = make(ROWS[TILES[tile]], 320, 272, False, seed=13)
    assert tile_rows(c) == tile
    c["xs"][:] = 2.0 ** -40         # G and U about 2^-40 * 2^-30 * the integer sum; a sum's size is near 2^15: A about 2^-111
    c["ws"][0][:] = c["ws"][1][:] = 2.0 ** -32
    c["ws"][2][:] = 2.0 ** 100
    import oracle
    index = np.arange(c["B"])
    oracle_of = lambda: oracle.expert_ffn_q8(c["x"], c["xs"], index, c["off"], *[a for p in zip(c["w"], c["ws"]) for a in p])
    most = np.abs(oracle_of()[1]).max(axis=1)
    # the row's scale acts twice (silu is linear here): every row's largest A to 2^-117, every third one's to 2^-122
    target = np.where(np.arange(c["B"]) % 3 == 1, 2.0 ** -122, 2.0 ** -117)
    c["xs"] = (c["xs"] * np.sqrt(target / most)).astype(np.float32)
    zero = np.arange(c["B"]) % 3 == 1
    got = call(m, c, torch.float32)
    assert not got[zero].any() and bool(got[~zero].any(dim=1).all())
    full = got.double().numpy()
    Y = oracle_of()[0]
    full[zero] = Y[zero]
    check(c, torch.from_numpy(full), torch.float32)
