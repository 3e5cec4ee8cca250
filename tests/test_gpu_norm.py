"""The norm in front of the layer (xmoe_norm.hip): forward, 8-bit rows, backward, against the float64 oracle.

Tolerances.  u = 2^-24.  A stored result is off by half a step of its type, finfo.eps / 2 relative to it.  Before that:
r comes from a float32 sum of d squares, taken by up to 32 additions in a thread, 6 over a wave and 16 over the waves, so
it is good to (54 + 6) / 2 + 3 = 33 u, and y to two more products: 40 u.  Backward: mean(v n) is off by at most 33 u for n,
54 u for the sum and 3 u, relative to mean |v n|, i.e. 90 u; dx to 33 u + 90 u + 8 u of its terms' sizes: 160 u bounds it.
dgain adds rows: ceil(T / 512) + 2 in a block, 4 waves, ceil(512 / 16) + 16 partial rows, and n's 33 u + 2 u.
The 8-bit integers are held bit for bit to float32 steps; their values to half a step and 40 u of 127 steps."""
import numpy as np
import pytest
import torch

import oracle

pytestmark = pytest.mark.gpu
EPS, U = 1e-6, 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SHAPES = [(1, 1), (3, 7), (5, 64), (2, 513), (4, 1000), (3, 1003), (1, 2048), (2, 2056), (3, 4104), (2, 7168), (1, 8200),
          (1, 16384), (2, 16383), (1027, 70), (1030, 1003), (1025, 2048)]


def half(dt):
    return torch.finfo(dt).eps / 2


def data(T, d, name, seed=0):
    g = torch.Generator().manual_seed(seed + 1000 * T + d)
    x, res, dy, dh = (torch.randn((T, d), generator=g).to(DT[name]) for _ in range(4))
    res = (res.float() * 2).to(DT[name])
    return x, res, (1 + 0.2 * torch.randn(d, generator=g)).to(DT[name]), dy, dh


def f64(t):
    return t.double().numpy()


def guarded(shape, dtype, fill):
    """A buffer of shape + one row more, and the part that a call gets."""
    whole = torch.full((shape[0] + 1,) + tuple(shape[1:]), fill, dtype=dtype, device="cuda")
    return whole, whole[:shape[0]]


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", SHAPES)
def test_forward(T, d, name):
    import paper_2508_13337_amd as m
    x, res, gain, _, _ = data(T, d, name)
    dt = DT[name]
    h, y = guarded((T, d), dt, 7.0), guarded((T, d), dt, 7.0)
    rstd = guarded((T,), torch.float32, 7.0)
    q, s = guarded((T, m.xmoe_q8_pitch(d)), torch.int8, 99), guarded((T,), torch.float32, 7.0)
    m.xmoe_add_rmsnorm(x.cuda(), res.cuda(), gain.cuda(), EPS, h[1], y=y[1], q=q[1], q_scale=s[1], rstd=rstd[1])
    torch.cuda.synchronize()
    for whole, fill in ((h[0], 7.0), (y[0], 7.0), (rstd[0], 7.0), (s[0], 7.0), (q[0], 99)):
        assert bool((whole[T] == fill).all())
    want_h = (x.float() + res.float()).to(dt)
    assert torch.equal(h[1].cpu(), want_h)
    ref, r = oracle.add_rmsnorm(f64(want_h), f64(gain), EPS)
    assert np.all(np.abs(f64(rstd[1].cpu()) - r) <= 35 * U * r)
    assert np.all(np.abs(f64(y[1].cpu()) - ref) <= (half(dt) + 40 * U) * np.abs(ref))
    v = want_h.float().numpy() * gain.float().numpy()
    want_q, mx = oracle.quantize_rows_f32(v)
    got = q[1].cpu().numpy()
    assert np.array_equal(got[:, :d], want_q) and not got[:, d:].any()
    scale = f64(s[1].cpu())
    assert np.all(np.abs(scale - mx.astype(np.float64) * r / 127) <= 40 * U * scale)
    assert np.all(np.abs(got[:, :d] * scale[:, None] - ref) <= scale[:, None] * (0.5 + 127 * 40 * U))


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("T,d", SHAPES)
def test_backward(T, d, name):
    import paper_2508_13337_amd as m
    x, res, gain, dy, dh = data(T, d, name, seed=1)
    dt = DT[name]
    hc = (x.float() + res.float()).to(dt)
    h, rstd = hc.cuda(), torch.empty(T, device="cuda")
    y = torch.empty_like(h)
    m.xmoe_add_rmsnorm(h, None, gain.cuda(), EPS, None, y=y, rstd=rstd)
    ws = m.alloc_workspace(m.xmoe_workspace_bytes(m.WS_ADD_RMSNORM_BWD, T, d, 0, 0, 0, m.dtype_code(dt)))
    for way in (dh, None):
        dx, dg = guarded((T, d), dt, 7.0), guarded((d,), dt, 7.0)
        m.xmoe_add_rmsnorm_bwd(dy.cuda(), None if way is None else way.cuda(), h, gain.cuda(), rstd, dx[1], dg[1], ws)
        torch.cuda.synchronize()
        assert bool((dx[0][T] == 7.0).all()) and float(dg[0][d]) == 7.0
        ref, ref_g = oracle.add_rmsnorm_bwd(f64(dy), None if way is None else f64(way), f64(hc), f64(gain), EPS)
        r = oracle.add_rmsnorm(f64(hc), f64(gain), EPS)[1][:, None]
        n, v = f64(hc) * r, f64(dy) * f64(gain)
        size = r * (np.abs(v) + np.abs(n) * np.abs(v * n).mean(axis=1, keepdims=True)) + (0 if way is None else np.abs(f64(way)))
        assert np.all(np.abs(f64(dx[1].cpu()) - ref) <= half(dt) * np.abs(ref) + 160 * U * size)
        adds = -(-T // 512) + 2 + 4 + 32 + 16 + 35
        assert np.all(np.abs(f64(dg[1].cpu()) - ref_g) <= half(dt) * np.abs(ref_g) + adds * U * np.abs(f64(dy) * n).sum(axis=0))


@pytest.mark.parametrize("which", ["x", "residual"])
@pytest.mark.parametrize("T,d", [(3, 1003), (1100, 520), (2, 7168)])
def test_the_sum_may_replace_an_input(which, T, d):
    import paper_2508_13337_amd as m
    x, res, gain, _, _ = (t.cuda() for t in data(T, d, "bf16"))
    y, h, z = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    m.xmoe_add_rmsnorm(x, res, gain, EPS, h, y=y)
    m.xmoe_add_rmsnorm(x, res, gain, EPS, x if which == "x" else res, y=z)
    assert torch.equal(y, z) and torch.equal(h, x if which == "x" else res)


def test_outputs_alone_have_the_bits_of_all_together():
    import paper_2508_13337_amd as m
    x, _, gain, _, _ = (t.cuda() for t in data(9, 1400, "bf16"))
    q, s, y = torch.empty((9, m.xmoe_q8_pitch(1400)), dtype=torch.int8, device="cuda"), torch.empty(9, device="cuda"), torch.empty_like(x)
    q2, s2, y2 = torch.empty_like(q), torch.empty_like(s), torch.empty_like(y)
    m.xmoe_add_rmsnorm(x, None, gain, EPS, None, y=y, q=q, q_scale=s)
    m.xmoe_add_rmsnorm(x, None, gain, EPS, None, y=y2)
    m.xmoe_add_rmsnorm(x, None, gain, EPS, None, q=q2, q_scale=s2)
    assert torch.equal(y, y2) and torch.equal(q, q2) and torch.equal(s, s2)


@pytest.mark.parametrize("name", ["bf16", "f32"])
def test_rows_of_zeros_tiny_ones_and_what_is_no_number(name):
    import paper_2508_13337_amd as m
    d, dt = 200, DT[name]
    x = torch.randn((6, d), generator=torch.Generator().manual_seed(4)).to(dt)
    x[0] = 0
    x[1] *= 2.0 ** -125      # every |h gain| is below 2^-120
    x[2, 17] = float("inf")
    x[3, 5] = float("nan")
    x[4] *= 2.0 ** -100
    gain = torch.ones(d, dtype=dt)
    y, q = torch.empty((6, d), dtype=dt, device="cuda"), torch.empty((6, 256), dtype=torch.int8, device="cuda")
    s = torch.empty(6, device="cuda")
    m.xmoe_add_rmsnorm(x.cuda(), None, gain.cuda(), EPS, None, y=y, q=q, q_scale=s)
    y, q, s = y.cpu().float(), q.cpu()[:, :d].float(), s.cpu()
    assert not y[0].any() and not q[0].any() and s[0] == 0
    assert not q[1].any() and s[1] == 0
    assert not torch.isfinite(s[2]) and not torch.isfinite(s[3]) and torch.isnan(y[2, 17]) and torch.isnan(y[3]).all()
    want = oracle.quantize_rows_f32(x[4:].float().numpy())[0]
    assert np.array_equal(q[4:].numpy(), want) and torch.isfinite(y[4:]).all()
    ref, _ = oracle.add_rmsnorm(f64(x[5:]), f64(gain), EPS)
    assert np.all(np.abs(f64(y[5:]) - ref) <= (half(dt) + 40 * U) * np.abs(ref))


def test_no_rows():
    import paper_2508_13337_amd as m
    h = torch.empty((0, 48), dtype=torch.bfloat16, device="cuda")
    gain, dgain = torch.ones(48, dtype=torch.bfloat16, device="cuda"), torch.full((48,), 7.0, dtype=torch.bfloat16, device="cuda")
    rstd = torch.empty(0, device="cuda")
    m.xmoe_add_rmsnorm(h, None, gain, EPS, None, y=torch.empty_like(h))
    ws = m.alloc_workspace(m.xmoe_workspace_bytes(m.WS_ADD_RMSNORM_BWD, 0, 48, 0, 0, 0, m.XMOE_BF16))
    m.xmoe_add_rmsnorm_bwd(h, None, h, gain, rstd, torch.empty_like(h), dgain, ws)
    assert not dgain.any()


def test_another_stream_and_a_replayed_graph():
    import paper_2508_13337_amd as m
    x, res, gain, dy, dh = (t.cuda() for t in data(700, 1003, "bf16"))
    ws = m.alloc_workspace(m.xmoe_workspace_bytes(m.WS_ADD_RMSNORM_BWD, 700, 1003, 0, 0, 0, m.XMOE_BF16))
    o = {n: torch.empty_like(x) for n in ("h", "y", "dx")}
    o.update(dg=torch.empty_like(gain), r=torch.empty(700, device="cuda"))

    def step():
        m.xmoe_add_rmsnorm(x, res, gain, EPS, o["h"], y=o["y"], rstd=o["r"])
        m.xmoe_add_rmsnorm_bwd(dy, dh, o["h"], gain, o["r"], o["dx"], o["dg"], ws)

    step()
    want = {n: t.clone() for n, t in o.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(want[n], t) for n, t in o.items())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for turn in range(4):
        x.normal_()
        res.normal_()
        graph.replay()
        got = {n: t.clone() for n, t in o.items()}
        torch.cuda.synchronize()
        step()
        assert all(torch.equal(got[n], t) for n, t in o.items()), turn
