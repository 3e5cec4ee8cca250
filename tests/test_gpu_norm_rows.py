"""The norm in front of the layer (xmoe_norm.hip), row by row: the padding of 8-bit rows that hold no numbers, and a row's
bits beside few and beside many other rows."""
import pytest
import torch

from test_gpu_norm import DT, EPS, data

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


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("d", [70, 257, 520, 600, 1003, 1024, 1500, 2048, 2056, 4104, 8200])
def test_a_rows_bits_do_not_depend_on_the_others(d, name):
    """Few rows are spread over more threads: the sums keep their order."""
    import paper_2508_13337_amd as m
    T, few = 1029, [0, 1, 512, 1027, 1028]
    dt = DT[name]
    x, res, gain, dy, dh = (t.cuda() for t in data(T, d, name, seed=3))

    def step(x, res, dy, dh):
        t = x.shape[0]
        o = {n: torch.empty_like(x) for n in ("h", "y", "dx")}
        o.update(rstd=torch.empty(t, device="cuda"), q=torch.empty((t, m.xmoe_q8_pitch(d)), dtype=torch.int8, device="cuda"),
                 q_scale=torch.empty(t, device="cuda"))
        m.xmoe_add_rmsnorm(x, res, gain, EPS, o["h"], y=o["y"], q=o["q"], q_scale=o["q_scale"], rstd=o["rstd"])
        ws = m.alloc_workspace(m.xmoe_workspace_bytes(m.WS_ADD_RMSNORM_BWD, t, d, 0, 0, 0, m.dtype_code(dt)))
        m.xmoe_add_rmsnorm_bwd(dy, dh, o["h"], gain, o["rstd"], o["dx"], torch.empty_like(gain), ws)
        return o

    whole = step(x, res, dy, dh)
    part = step(*(t[few].contiguous() for t in (x, res, dy, dh)))
    for n in whole:
        assert torch.equal(whole[n][few], part[n]), n
