"""A row's bits do not depend on the call's other rows, across the kernels that a call's size selects: the 8-bit experts' three
tile sizes, the narrow and the wide tiles of a layer for few tokens.  And the routing of rows longer than what it holds at a
time."""
import numpy as np
import pytest
import torch

import test_gpu_layer_few as few
from test_gpu_q8 import make, padded, tile_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,f", [(320, 448), (1000, 712), (264, 1409)])
def test_8_bit_experts(d, f, dt):
    import paper_2508_13337_amd as m
    rows = [1, 0, 33, 7, 20]
    c = make(rows, d, f, True, seed=21)
    g = np.random.default_rng(1)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    w = [t for q, s in zip(c["w"], c["ws"]) for t in (dev(padded(q)), dev(s))]
    got = {}
    for tile, more in ((32, [0, 0, 0, 0, 0]), (128, [128, 3, 64, 95, 129]), (256, [999, 130, 700, 257, 1])):
        n = np.add(rows, more)
        off = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        index = np.concatenate([np.concatenate([c["index"][c["off"][e]:c["off"][e + 1]], g.integers(0, 41, a)])
                                for e, a in enumerate(more)]).astype(np.int32)
        B = int(off[-1])
        assert tile_rows(dict(c, B=B)) == tile
        y = torch.empty((B, d), dtype=dt, device="cuda")
        ws = m.alloc_workspace(m.xmoe_workspace_bytes(m.WS_FFN_Q8_FWD, B, d, c["E"], 1, f, m.dtype_code(dt)))
        m.xmoe_expert_ffn_q8_fwd(dev(padded(c["x"])), dev(c["xs"]), dev(off), *w, y, ws, row_index=dev(index))
        # the workspace begins with the number of row tiles: the tile size that ran
        assert int(ws[:4].view(torch.int32)) == sum(-(-int(a) // tile) for a in n), tile
        got[tile] = torch.cat([y[off[e]:off[e] + a] for e, a in enumerate(rows)])
    assert torch.equal(got[32], got[128]) and torch.equal(got[32], got[256])


@pytest.mark.parametrize("d,f,E,k,E_s", [(328, 1032, 64, 6, 2), (200, 2048, 48, 4, 0), (72, 1408, 64, 6, 1)])
def test_layer_for_few_tokens(d, f, E, k, E_s):
    """8 or fewer experts with one token, all of them with 32: on either side of the rule for up's tiles, far from it."""
    import paper_2508_13337_amd as m
    c = few.make(32, d, f, E, k, E_s, "bf16", seed=4, std=0.05)
    whole, _ = few.run(m, c)
    for t in (0, 17, 31):
        one, _ = few.run(m, dict(c, x=c["x"][t:t + 1], addend=c["addend"][t:t + 1], T=1))
        assert all(torch.equal(one[n][0], whole[n][t]) for n in one), t


@pytest.mark.parametrize("name,d,E", [("bf16", 8192, 16), ("bf16", 4104, 8), ("bf16", 4097, 31), ("bf16", 13000, 10),
                                      ("f32", 8193, 7), ("f32", 5000, 12)])
def test_routing_of_long_rows(name, d, E):
    import paper_2508_13337_amd as m
    c = few.make(5, d, 16, E, 3, 1, name, seed=6, std=0.02)
    got, kernels = few.run(m, c)
    assert "layer_route_kernel" in kernels
    few.check(c, got)
