"""A whole layer for a few tokens (xmoe_layer_few.hip) against the float64 oracle, and against the calls that it stands for.

Tolerance of out, element by element, u = 2^-24, h = half a step of the type.  A product over K terms is off by at most
(K + 8) u of the sum of its terms' sizes, in any order.  silu's slope is below 1.1, the activation and its rounding add
8 u + h of A; weights p 32 u; the sum over a token's experts (k + E_s + 2) u; the stored result h."""
import numpy as np
import pytest
import torch

import oracle
from gpu_util import launched

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
#         T   d     f    E    k  E_s
CASES = [(1, 64, 64, 8, 2, 0), (1, 2048, 192, 16, 6, 2), (2, 128, 192, 4, 4, 1), (3, 1003, 705, 16, 4, 1), (5, 50, 22, 7, 3, 2),
         (7, 7, 5, 3, 1, 0), (4, 3, 2, 5, 5, 1), (1, 1, 1, 1, 1, 0), (16, 320, 448, 64, 6, 2), (31, 72, 24, 6, 2, 0),
         (32, 64, 128, 1, 1, 1), (32, 256, 64, 12, 12, 3), (9, 520, 64, 512, 8, 0), (6, 136, 64, 300, 64, 1),
         (2, 2048, 64, 257, 8, 1), (32, 192, 320, 40, 8, 2), (13, 65, 129, 24, 3, 0),
         (3, 1000, 712, 24, 3, 1), (8, 8, 8, 4, 2, 0), (11, 40, 1032, 9, 4, 1), (32, 264, 104, 5, 2, 2), (2, 904, 2056, 6, 2, 0)]


def make(T, d, f, E, k, E_s, name, seed=0, std=0.1):
    g = torch.Generator().manual_seed(seed + 7 * T + d + 3 * f + E)
    dt = DTYPE = DT[name]
    r = lambda *s, std=1.0: (torch.randn(s, generator=g) * std).to(dt)
    return dict(x=r(T, d), w_router=r(d, E, std=d ** -0.5), bias=torch.randn(E, generator=g), wg=r(E + E_s, d, f, std=std),
                wu=r(E + E_s, d, f, std=std), wd=r(E + E_s, f, d, std=std), addend=r(T, d), T=T, d=d, f=f, E=E, k=k, E_s=E_s,
                dt=DTYPE)


def buffers(m, c):
    """Inputs on the GPU, outputs with a marked row behind each, a workspace full of noise."""
    T, E, k = c["T"], c["E"], c["k"]
    o = dict(logits=torch.full((T + 1, E), 7.0, device="cuda"), topk_idx=torch.full((T + 1, k), -7, dtype=torch.int32, device="cuda"),
             topk_w=torch.full((T + 1, k), 7.0, device="cuda"), out=torch.full((T + 1, c["d"]), 7.0, dtype=c["dt"], device="cuda"))
    dev = {n: None if c[n] is None else c[n].cuda() for n in ("x", "w_router", "bias", "wg", "wu", "wd", "addend")}
    n = m.xmoe_workspace_bytes(m.WS_LAYER_FEW_FWD, T, c["d"], E + c["E_s"], k + c["E_s"], c["f"], m.dtype_code(c["dt"]))
    ws = m.alloc_workspace(n)
    ws.random_(0, 256)
    return dev, o, ws


def call(m, dev, o, ws, T):
    m.xmoe_layer_few_fwd(dev["x"], dev["w_router"], dev["bias"], dev["wg"], dev["wu"], dev["wd"], dev["addend"], o["logits"][:T],
                         o["topk_idx"][:T], o["topk_w"][:T], o["out"][:T], ws)


def run(m, c):
    dev, o, ws = buffers(m, c)
    kernels = launched(m, lambda: call(m, dev, o, ws, c["T"]))
    o = {n: t.cpu() for n, t in o.items()}
    assert all(bool((t[c["T"]] == (-7 if n == "topk_idx" else 7)).all()) for n, t in o.items())
    return {n: t[:c["T"]] for n, t in o.items()}, kernels


def reference(c):
    """(idx, weights, out, tolerance) in float64 on the oracle's routing."""
    x = c["x"].float().numpy()
    bias = None if c["bias"] is None else c["bias"].numpy()
    logits = oracle.gate_logits_contract(x, c["w_router"].float().numpy(), bias)
    idx, w, _ = oracle.route(logits, c["k"])
    h = torch.finfo(c["dt"]).eps / 2
    gd, gf = (c["d"] + 8) * U, (c["f"] + 8) * U
    x = x.astype(np.float64)
    out = np.zeros_like(x) if c["addend"] is None else c["addend"].double().numpy()
    size, tol = np.abs(out), np.zeros_like(x)
    for e in range(c["E"] + c["E_s"]):
        t, weight = (np.nonzero((idx == e).any(axis=1))[0], None) if e < c["E"] else (np.arange(c["T"]), 1.0)
        if len(t) == 0:
            continue
        if weight is None:
            weight = np.asarray(w, np.float64)[idx == e][:, None]
        wg, wu, wd = (c[n][e].double().numpy() for n in ("wg", "wu", "wd"))
        G, Up = x[t] @ wg, x[t] @ wu
        s = oracle.silu(G)
        A = s * Up
        dA = 1.1 * gd * (np.abs(x[t]) @ np.abs(wg)) * np.abs(Up) + gd * np.abs(s) * (np.abs(x[t]) @ np.abs(wu)) + (8 * U + h) * np.abs(A)
        Y, sY = A @ wd, np.abs(A) @ np.abs(wd)
        out[t] += weight * Y
        size[t] += weight * np.abs(Y)
        tol[t] += weight * (dA @ np.abs(wd) + (gf + 32 * U) * sY)
    return logits, idx, w, out, tol + (c["k"] + c["E_s"] + 2) * U * size + h * np.abs(out)


def check(c, got):
    logits, idx, w, out, tol = reference(c)
    assert np.array_equal(got["logits"].numpy(), logits.astype(np.float32)) and np.array_equal(got["topk_idx"].numpy(), idx)
    w = np.asarray(w, np.float64)
    assert np.all(np.abs(got["topk_w"].double().numpy() - w) <= 32 * U * w + 1e-38)
    err = np.abs(got["out"].double().numpy() - out)
    assert np.all(err <= tol * 1.01), float((err / tol).max())


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("case", CASES, ids=["-".join(map(str, c)) for c in CASES])
def test_against_the_oracle(case, name):
    import paper_2508_13337_amd as m
    c = make(*case, name)
    got, kernels = run(m, c)
    check(c, got)
    matrix = name == "bf16" and c["d"] % 8 == 0 and c["f"] % 8 == 0
    assert ("layer_up_few_kernel" in kernels) == matrix and ("layer_up_alu_kernel" in kernels) != matrix, kernels


def test_no_bias_no_addend_and_the_sum_in_place():
    import paper_2508_13337_amd as m
    for name in ("bf16", "f32"):
        c = make(5, 128, 64, 8, 2, 1, name, seed=3)
        plain = dict(c, bias=None, addend=None)
        check(plain, run(m, plain)[0])
        dev, o, ws = buffers(m, c)
        call(m, dev, o, ws, 5)
        want = o["out"][:5].clone()
        m.xmoe_layer_few_fwd(dev["x"], dev["w_router"], dev["bias"], dev["wg"], dev["wu"], dev["wd"], dev["addend"],
                             o["logits"][:5], o["topk_idx"][:5], o["topk_w"][:5], dev["addend"], ws)
        assert torch.equal(dev["addend"], want)


def test_routing_has_the_bits_of_the_calls_it_stands_for():
    import paper_2508_13337_amd as m
    for case in ((16, 2048, 64, 64, 6, 0), (32, 1003, 8, 100, 5, 0), (3, 640, 64, 512, 8, 0)):
        c = make(*case, "bf16", seed=5)
        got, _ = run(m, c)
        logits = torch.empty((c["T"], c["E"]), device="cuda")
        idx = torch.empty((c["T"], c["k"]), dtype=torch.int32, device="cuda")
        w = torch.empty((c["T"], c["k"]), device="cuda")
        m.xmoe_gate_logits(c["x"].cuda(), c["w_router"].cuda(), c["bias"].cuda(), logits)
        m.xmoe_route(logits, c["k"], idx, w)
        assert torch.equal(got["logits"], logits.cpu()) and torch.equal(got["topk_idx"], idx.cpu()) and torch.equal(got["topk_w"], w.cpu())


@pytest.mark.parametrize("name,d", [("bf16", 128), ("bf16", 72), ("f32", 96)])
def test_a_tokens_bits_do_not_depend_on_the_others(name, d):
    import paper_2508_13337_amd as m
    c = make(32, d, 64, 8, 3, 1, name, seed=1)
    whole, _ = run(m, c)
    for t in (0, 13, 31):
        one, _ = run(m, dict(c, x=c["x"][t:t + 1], addend=c["addend"][t:t + 1], T=1))
        assert all(torch.equal(one[n][0], whole[n][t]) for n in one), t


@pytest.mark.parametrize("name,d", [("bf16", 128), ("f32", 100)])
def test_all_tokens_on_the_same_experts_and_experts_that_nobody_picked(name, d):
    import paper_2508_13337_amd as m
    c = make(32, d, 64, 10, 2, 0, name, seed=2)
    c["bias"][:] = -1e30
    c["bias"][3] = c["bias"][8] = 0.0
    for n in ("wg", "wu", "wd"):        # never read
        c[n][[e for e in range(10) if e not in (3, 8)]] = float("nan")
    got, _ = run(m, c)
    assert set(got["topk_idx"].flatten().tolist()) == {3, 8}
    check(c, got)


def test_no_tokens():
    import paper_2508_13337_amd as m
    c = make(1, 64, 64, 4, 2, 0, "bf16")
    c.update(x=c["x"][:0], addend=c["addend"][:0], T=0)
    _, kernels = run(m, c)
    assert not kernels


@pytest.mark.parametrize("case", [(4, 256, 128, 16, 4, 1, "bf16"), (3, 100, 37, 9, 2, 1, "f32")])
def test_another_stream_and_a_replayed_graph(case):
    import paper_2508_13337_amd as m
    c = make(*case)
    T = c["T"]
    dev, o, ws = buffers(m, c)
    call(m, dev, o, ws, T)
    want = {n: t.clone() for n, t in o.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for _ in range(3):
            call(m, dev, o, ws, T)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(want[n], t) for n, t in o.items())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(m, dev, o, ws, T)
        call(m, dev, o, ws, T)
    for turn in range(5):
        dev["x"].normal_()
        graph.replay()
        got = {n: t.clone() for n, t in o.items()}
        torch.cuda.synchronize()
        call(m, dev, o, ws, T)
        assert all(torch.equal(got[n], t) for n, t in o.items()), turn


def test_two_calls_at_once():
    """On two streams, each with its own buffers."""
    import paper_2508_13337_amd as m
    cs = [make(4, 512, 256, 32, 4, 1, "bf16", seed=s) for s in (1, 2)]
    bs = [buffers(m, c) for c in cs]
    for c, b in zip(cs, bs):
        call(m, *b, c["T"])
    torch.cuda.synchronize()
    want = [{n: t.clone() for n, t in b[1].items()} for b in bs]
    streams = [torch.cuda.Stream() for _ in cs]
    for turn in range(20):
        for c, b, s in zip(cs, bs, streams):
            with torch.cuda.stream(s):
                call(m, *b, c["T"])
    torch.cuda.synchronize()
    for w, b in zip(want, bs):
        assert all(torch.equal(w[n], t) for n, t in b[1].items())
