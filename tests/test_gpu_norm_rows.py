"""The norm in front of the layer (xmoe_norm.hip), row by row: the padding of 8-bit rows that hold no numbers."""
import pytest
import torch

from test_gpu_norm import EPS, data

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("d", [1, 130, 200, 1003, 2050, 5001])
def test_the_padding_of_rows_that_are_no_numbers(d, name):
    import paper_2508_13337_amd as m
    x, _, gain, _, _ = data(6, d, name)
    x[1, d // 2] = float("nan")
    x[2, 0] = float("inf")
    x[3, d - 1] = float("-inf")
    x[4] = float("nan")
    q, s = torch.full((6, m.xmoe_q8_pitch(d)), 99, dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda")
    for g in (gain, torch.full_like(gain, float("nan"))):
        m.xmoe_add_rmsnorm(x.cuda(), None, g.cuda(), EPS, None, q=q, q_scale=s)
        assert not q[:, d:].any()
        assert not torch.isfinite(s[1:5]).any()
