"""The operators as they are used together: XMoEServe (norm, then the layer for a few or for many tokens, in the storage type
or on 8-bit experts) and XMoELayer with the norm in front, forward and backward.

Each stage is compared with the oracle on the bits that the stage before it left: the norm's output element by element (its
derivation stands in test_gpu_norm.py), the layer behind it with the criteria for whole layers (gpu_util).  8-bit experts:
an integer of A is off by one at most, which is half a step and the oracle's half: 2 / 127 of the row's maximum at the very
worst for every element at once; what can happen in earnest is held by test_gpu_q8.py, and here the layer with 8-bit experts
is held to the oracle's 8-bit experts by the whole-layer criterion."""
import numpy as np
import pytest
import torch

import oracle
import xmoe_inputs as xi
from gpu_util import assert_close_chain, launched, to_dev, to_host

pytestmark = pytest.mark.gpu
EPS, U = 1e-6, 2.0 ** -24


def setup(name, T, seed=0):
    import paper_2508_13337_amd as m
    cfg = xi.CONFIGS[name].with_T(T)
    inp = xi.make_layer_inputs(cfg)
    g = torch.Generator().manual_seed(seed + T)
    dt = torch.float32 if cfg.dtype == "f32" else torch.bfloat16
    x, res = torch.randn((T, cfg.d), generator=g).to(dt), (2 * torch.randn((T, cfg.d), generator=g)).to(dt)
    gain = (1 + 0.2 * torch.randn(cfg.d, generator=g)).to(dt)
    w = {"w_router": to_dev(inp["w_router"], cfg.dtype), "norm_gain": gain.cuda(),
         "bias": None if inp["bias"] is None else torch.from_numpy(inp["bias"]).cuda()}
    for n in ("wg", "wu", "wd"):
        w[n] = m.append_shared(to_dev(inp[n], cfg.dtype), to_dev(inp["shared_" + n], cfg.dtype) if cfg.E_s else None)
    return m, cfg, inp, dt, x, res, gain, w


def check_norm(dt, x, res, gain, h, xn):
    want = x if res is None else (x.float() + res.float()).to(dt)
    assert torch.equal(h.cpu(), want)
    ref, _ = oracle.add_rmsnorm(want.double().numpy(), gain.double().numpy(), EPS)
    assert np.all(np.abs(xn.cpu().double().numpy() - ref) <= (torch.finfo(dt).eps / 2 + 40 * U) * np.abs(ref))


def with_x(inp, xn):
    return {**inp, "x": xn.float().cpu().numpy()}


@pytest.mark.parametrize("T", [1, 5, 32, 33, 300])
@pytest.mark.parametrize("name", ["mini_bf16", "mini_f32", "odd_bf16", "odd_f32", "mini_bf16_skew"])
def test_serve(name, T):
    m, cfg, inp, dt, x, res, gain, w = setup(name, 300)
    block = m.XMoEServe(300, cfg.d, cfg.E, cfg.k, cfg.f, dt, E_s=cfg.E_s, eps=EPS)
    for r in (res[:T], None):
        kernels = launched(m, lambda: block.forward(x[:T].cuda(), None if r is None else r.cuda(), w))
        out, h = block.out[:T], block.h[:T]
        assert ("layer_sum_kernel" in kernels) == (T <= 32)
        check_norm(dt, x[:T], r, gain, h, block.xn[:T])
        fwd = oracle.moe_layer_fwd(with_x(inp, block.xn[:T]), cfg.k)
        assert np.array_equal(block.topk_idx[:T].cpu().numpy(), fwd["topk_idx"])
        assert_close_chain(to_host(out), fwd["out"], cfg.dtype, f"{name} T={T}")


@pytest.mark.parametrize("T", [1, 32, 300])
@pytest.mark.parametrize("name", ["mini_bf16", "mid_bf16", "odd_bf16"])
def test_serve_on_8_bit_experts(name, T):
    m, cfg, inp, dt, x, res, gain, w = setup(name, T)
    w8 = m.quantize_experts(w)
    block = m.XMoEServe(T, cfg.d, cfg.E, cfg.k, cfg.f, dt, E_s=cfg.E_s, eps=EPS, q8=True)
    out, h = block.forward(x.cuda(), res.cuda(), w8)
    check_norm(dt, x, res, gain, h, block.xn)
    idx, topk_w, _ = oracle.route(block.logits.cpu().numpy(), cfg.k)
    assert np.array_equal(block.topk_idx.cpu().numpy(), idx)
    eri = oracle.build_eri(idx, topk_w, cfg.E)
    off = np.concatenate([eri["expert_offsets"], T * cfg.k + T * np.arange(1, cfg.E_s + 1)])
    rows = np.concatenate([eri["token_ids"], np.tile(np.arange(T), cfg.E_s)])
    v = h.float().cpu().numpy() * gain.float().numpy()
    xq = oracle.quantize_rows_f32(v)[0]
    assert np.array_equal(block.q.cpu().numpy()[:, :cfg.d], xq)
    q, s = {}, {}
    for n in "gud":
        q[n], mx = oracle.quantize_rows_f32(w["w" + n].float().cpu().numpy().transpose(0, 2, 1))
        s[n] = mx / np.float32(127)
        assert np.array_equal(w8[f"w{n}q"].cpu().numpy()[..., :q[n].shape[2]], q[n])
    Y = oracle.expert_ffn_q8(xq, block.q_scale.cpu().numpy(), rows, off, q["g"], s["g"], q["u"], s["u"], q["d"], s["d"])[0]
    B = T * cfg.k
    want = oracle.combine(Y[:B], eri["token_ids"], eri["combine_weights"], T)
    for e in range(cfg.E_s):
        want = want + Y[B + e * T:B + (e + 1) * T]
    assert_close_chain(to_host(out), want, cfg.dtype, f"{name} T={T}")
    # and what 8 bits cost against the layer itself: a percent or two of the output
    full = oracle.moe_layer_fwd(with_x(inp, block.xn), cfg.k)["out"]
    assert np.linalg.norm(to_host(out) - full) <= 0.05 * np.linalg.norm(full)


@pytest.mark.parametrize("q8", [False, True])
def test_calls_of_many_sizes_share_the_buffers(q8):
    """A prompt, decoding steps, a prompt again; the last call's results are the next one's inputs."""
    m, cfg, inp, dt, x, res, gain, w = setup("mid_bf16", 200)
    w = m.quantize_experts(w) if q8 else w
    block = m.XMoEServe(200, cfg.d, cfg.E, cfg.k, cfg.f, dt, E_s=cfg.E_s, q8=q8)
    for T in (200, 1, 32, 7, 120, 0):
        fresh = m.XMoEServe(max(T, 1), cfg.d, cfg.E, cfg.k, cfg.f, dt, E_s=cfg.E_s, q8=q8)
        a, ha = (t.clone() for t in block.forward(x[:T].cuda(), res[:T].cuda(), w))
        b, hb = (t.clone() for t in fresh.forward(x[:T].cuda(), res[:T].cuda(), w))
        assert torch.equal(a, b) and torch.equal(ha, hb), T
        a2, ha2 = block.forward(block.out[:T], block.h[:T], w)      # a second layer behind the first
        b2, hb2 = fresh.forward(b, hb, w)
        assert torch.equal(a2, b2) and torch.equal(ha2, hb2), T
    with pytest.raises(ValueError):
        block.forward(torch.zeros((201, cfg.d), dtype=dt, device="cuda"), None, w)


@pytest.mark.parametrize("q8,T", [(False, 4), (False, 100), (True, 4), (True, 100)])
def test_a_replayed_step(q8, T):
    m, cfg, inp, dt, x, res, gain, w = setup("mid_bf16", T)
    w = m.quantize_experts(w) if q8 else w
    block = m.XMoEServe(T, cfg.d, cfg.E, cfg.k, cfg.f, dt, E_s=cfg.E_s, q8=q8)
    x, res = x.cuda(), res.cuda()
    block.forward(x, res, w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        block.forward(x, res, w)
    for turn in range(4):
        x.normal_()
        res.normal_()
        graph.replay()
        got = block.out.clone(), block.h.clone()
        torch.cuda.synchronize()
        out, h = block.forward(x, res, w)
        assert torch.equal(got[0], out) and torch.equal(got[1], h), turn


@pytest.mark.parametrize("name", ["mini_bf16", "mini_f32", "odd_f32"])
def test_layer_with_the_norm(name):
    m, cfg, inp, dt, x, res, gain, w = setup(name, xi.CONFIGS[name].T)
    layer = m.XMoELayer(cfg.T, cfg.d, cfg.E, cfg.k, cfg.f, dt, E_s=cfg.E_s, norm_eps=EPS)
    grads = {"d" + n: torch.empty_like(t) for n, t in w.items() if t is not None and n != "bias"}
    dout, dh = (torch.randn((cfg.T, cfg.d), generator=torch.Generator().manual_seed(s)).to(dt) for s in (8, 9))
    xc, rc, dc, hc = x.cuda(), res.cuda(), dout.cuda(), dh.cuda()
    out = layer.forward(xc, w, residual=rc)
    dx = layer.backward(xc, w, dc, grads, dh=hc)
    torch.cuda.synchronize()
    check_norm(dt, x, res, gain, layer.h, layer.xn)
    li = {**with_x(inp, layer.xn), "dout": dout.float().numpy()}
    fwd = oracle.moe_layer_fwd(li, cfg.k)
    bwd = oracle.moe_layer_bwd(li, fwd, cfg.k)
    assert_close_chain(to_host(out), fwd["out"], cfg.dtype, "out")
    assert_close_chain(to_host(layer.dx), bwd["dx"], cfg.dtype, "dx of the layer")
    ref, ref_g = oracle.add_rmsnorm_bwd(to_host(layer.dx), dh.double().numpy(), to_host(layer.h), gain.double().numpy(), EPS)
    assert_close_chain(to_host(dx), ref, cfg.dtype, "dx")
    assert_close_chain(to_host(grads["dnorm_gain"])[None], ref_g[None], cfg.dtype, "dgain")
    # a replayed step has the bits of the eager one
    want = [out.clone(), dx.clone()] + [t.clone() for t in grads.values()]
    graph = m.capture_step(layer, xc, w, dc, grads, residual=rc, dh=hc)
    for turn in range(3):
        for t in grads.values():
            t.fill_(3.0)
        layer.out.fill_(3.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, [layer.out, layer.dx_norm] + list(grads.values()))), turn
        (torch.ones(1000, device="cuda") * 2).sum().item()      # eager work between the replays


def test_a_layer_without_the_norm_takes_no_residual():
    m, cfg, inp, dt, x, res, gain, w = setup("mini_bf16", 40)
    layer = m.XMoELayer(40, cfg.d, cfg.E, cfg.k, cfg.f, dt, E_s=cfg.E_s)
    with pytest.raises(ValueError):
        layer.forward(x.cuda(), w, residual=res.cuda())
    with pytest.raises(ValueError):
        layer.backward(x.cuda(), w, x.cuda(), {}, dh=res.cuda())
