"""The SwiGLU experts on 8-bit integers (xmoe_q8.hip) and the weights' quantisation.

Tolerance of y, element by element, u = 2^-24.  The integer sums are exact.  A's values are float32: |G| stays below 40 here,
which is good to 8 u + 4 |G| u, in steps of the row's 8 bits at most 127 * 168 u; on the way they are rounded to 2^-16 of a
maximum that is at most the row's: 127 * 2^-16 steps.  An integer of A can therefore differ from the oracle's, by one, only
where the oracle's value lies within 127 (168 u + 2^-16) of a tie, and each such k can move the sum by |wdq[n, k]|.  Scales and
products add 16 u, the stored result half a step of its type."""
import numpy as np
import pytest
import torch

import oracle
from gpu_util import launched

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
NEAR = 127 * (168 * U + 2.0 ** -16)
ROWS = {      # mean loads up to 16, up to 160 or 384 and above: the three tile sizes
    "edges": [0, 1, 255, 256, 257, 0, 31],
    "few": [1, 0, 2, 33, 0, 64, 65] + [0] * 8,
    "middle": [1, 0, 2, 33, 0, 64, 65],
    "one long": [0, 900, 3],
    "even": [300, 257, 290],
    "single": [1],
    "long": [1300, 0, 1100, 257, 1],
}
KERNELS = {"edges": 128, "few": 32, "middle": 128, "one long": 128, "even": 128, "single": 32, "long": 256}
WIDTHS = [(1, 1), (64, 64), (130, 200), (257, 96), (1000, 712), (384, 1409)]   # d, f


def pitch(n):
    return -(-n // 128) * 128


def padded(q):
    out = np.zeros(q.shape[:-1] + (pitch(q.shape[-1]),), np.int8)
    out[..., :q.shape[-1]] = q
    return out


def make(rows, d, f, gathered, seed=0):
    g = np.random.default_rng(seed + sum(rows) + 3 * d + f)
    E, B = len(rows), sum(rows)
    T = 41 if gathered else B
    off = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    index = g.integers(0, T, B).astype(np.int32) if gathered else None
    x, xs = oracle.quantize_rows(g.standard_normal((T, d)))
    w = [oracle.quantize_rows(0.05 * g.standard_normal(s)) for s in ((E, f, d), (E, f, d), (E, d, f))]
    return dict(x=x.astype(np.int8), xs=xs.astype(np.float32), index=index, off=off,
                w=[a.astype(np.int8) for a, _ in w], ws=[s.astype(np.float32) for _, s in w], B=B, E=E, d=d, f=f)


def tile_rows(c):
    B, E, d, f = c["B"], c["E"], c["d"], c["f"]
    if B <= 16 * E:
        return 32
    if B <= 160 * E or (B <= 384 * E and (B // 256 + E) * -(-f // 128) < 256):
        return 128
    return 256 if min(pitch(d), pitch(f)) >= 256 else 128


def call(m, c, dt, B=None, fill=7.0):
    """y of one call; a marked row behind it has to stand."""
    B = c["B"] if B is None else B
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
    y = torch.full((B + 1, c["d"]), fill, dtype=dt, device="cuda")
    ws = m.alloc_workspace(m.xmoe_workspace_bytes(m.WS_FFN_Q8_FWD, B, c["d"], c["E"], 1, c["f"], m.dtype_code(dt)))
    ws.random_(0, 256)
    args = [dev(a) for a in (padded(c["x"]), c["xs"], c["off"], padded(c["w"][0]), c["ws"][0], padded(c["w"][1]), c["ws"][1],
                             padded(c["w"][2]), c["ws"][2])]
    kernels = launched(m, lambda: m.xmoe_expert_ffn_q8_fwd(*args, y[:B], ws, row_index=dev(c["index"])))
    few = "_few" if B <= 16 * c["E"] else ""
    assert kernels >= {f"q8_gateup{few}_kernel", f"q8_down{few}_kernel"}, kernels
    assert bool((y[B] == fill).all())
    return y[:B].cpu()


def check(c, got, dt):
    index = np.arange(c["B"]) if c["index"] is None else c["index"]
    Y, A, AQ, AS = oracle.expert_ffn_q8(c["x"], c["xs"], index, c["off"], c["w"][0], c["ws"][0], c["w"][1], c["ws"][1],
                                        c["w"][2], c["ws"][2])
    steps = A / np.where(AS > 0, AS, 1)[:, None]
    near = np.abs(np.abs(steps) % 1.0 - 0.5) <= NEAR
    got = got.double().numpy()
    for e in range(c["E"]):
        s = slice(c["off"][e], c["off"][e + 1])
        moved = near[s].astype(np.float64) @ np.abs(c["w"][2][e].astype(np.float64)).T
        size = np.abs(AQ[s]).astype(np.float64) @ np.abs(c["w"][2][e].astype(np.float64)).T
        tol = (torch.finfo(dt).eps / 2) * np.abs(Y[s]) + AS[s][:, None] * c["ws"][2][e] * (1.01 * moved + 16 * U * size)
        assert np.all(np.abs(got[s] - Y[s]) <= tol), (e, float((np.abs(got[s] - Y[s]) - tol).max()))


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("gathered", [False, True])
@pytest.mark.parametrize("d,f", WIDTHS)
@pytest.mark.parametrize("rows", ROWS)
def test_against_the_oracle(rows, d, f, gathered, dt):
    import paper_2508_13337_amd as m
    c = make(ROWS[rows], d, f, gathered)
    assert tile_rows(c) == (128 if rows == "long" and min(d, f) <= 128 else KERNELS[rows])
    check(c, call(m, c, dt), dt)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d,f,gathered", [(200, 2700, True), (5000, 200, False), (1700, 1900, True)])
def test_more_tiles_than_blocks(d, f, gathered, dt):
    """256-row tiles, several of them to a block: in the first product, in the second, in both."""
    import paper_2508_13337_amd as m
    c = make([2000, 700, 1, 0, 3100, 513], d, f, gathered)
    tiles = sum(-(-n // 256) for n in (2000, 700, 1, 0, 3100, 513))
    assert tile_rows(c) == 256 and max(tiles * -(-f // 128), tiles * -(-d // 256)) > 256
    check(c, call(m, c, dt), dt)


@pytest.mark.parametrize("rows,d,f", [([3, 0, 20, 1], 384, 712), ([300, 20, 257, 0], 384, 712), ([1300, 900, 700], 320, 2700)])
def test_two_calls_at_once_and_a_replayed_graph(rows, d, f):
    """Of every tile size: two streams with buffers of their own, then both calls in one graph on one workspace."""
    import paper_2508_13337_amd as m
    cs = [make(rows, d, f, True, seed=s) for s in (1, 2)]
    ws = [m.alloc_workspace(m.xmoe_workspace_bytes(m.WS_FFN_Q8_FWD, c["B"], d, c["E"], 1, f, m.XMOE_BF16)) for c in cs]
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()
    args = [[dev(a) for a in (padded(c["x"]), c["xs"], c["off"], padded(c["w"][0]), c["ws"][0], padded(c["w"][1]), c["ws"][1],
                              padded(c["w"][2]), c["ws"][2])] for c in cs]
    index = [dev(c["index"]) for c in cs]
    y = [torch.empty((c["B"], d), dtype=torch.bfloat16, device="cuda") for c in cs]
    run = lambda i, w: m.xmoe_expert_ffn_q8_fwd(*args[i], y[i], ws[w], row_index=index[i])
    for i in (0, 1):
        run(i, i)
    want = [t.clone() for t in y]
    for c, t in zip(cs, want):
        check(c, t.cpu(), torch.bfloat16)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cs]
    for turn in range(6):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                run(i, i)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, y))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(0, 0)
        run(1, 0)
    for turn in range(4):
        for t in y:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, y)), turn


def test_serving_shape():
    import paper_2508_13337_amd as m
    c = make([0, 40, 13, 600, 1, 300], 2048, 1408, True)
    check(c, call(m, c, torch.bfloat16), torch.bfloat16)


def test_a_rows_bits_do_not_depend_on_the_call():
    """The same tokens among few rows and among many."""
    import paper_2508_13337_amd as m
    few, more = [1, 0, 33, 64, 7], [300, 3, 500, 70, 1]
    c = make(few, 320, 448, True)
    many = dict(c, off=np.concatenate([[0], np.cumsum(np.add(few, more))]).astype(np.int32), B=sum(few) + sum(more))
    g = np.random.default_rng(0)
    many["index"] = np.concatenate([np.concatenate([c["index"][c["off"][e]:c["off"][e + 1]], g.integers(0, 41, n)])
                                    for e, n in enumerate(more)]).astype(np.int32)
    a, b = call(m, c, torch.bfloat16), call(m, many, torch.bfloat16)
    for e, n in enumerate(few):
        assert torch.equal(a[c["off"][e]:c["off"][e] + n], b[many["off"][e]:many["off"][e] + n]), e


@pytest.mark.parametrize("rows", [[2, 0, 9], [300, 20, 257]])
def test_rows_behind_the_last_segment_stay(rows):
    import paper_2508_13337_amd as m
    c = make(rows, 200, 136, True)
    c["index"] = np.concatenate([c["index"], np.full(50, 1 << 30, np.int32)])    # never read
    got = call(m, c, torch.bfloat16, B=c["B"] + 50)
    assert bool((got[c["B"]:] == 7.0).all())
    check(c, got[:c["B"]], torch.bfloat16)


@pytest.mark.parametrize("rows", [[3, 5], [300, 290]])
def test_rows_of_zeros_and_scales_that_are_no_number(rows):
    import paper_2508_13337_amd as m
    c = make(rows, 256, 192, False)
    clean = call(m, c, torch.bfloat16)
    c["x"][1] = 0
    c["xs"][2], c["xs"][4] = np.nan, np.inf
    got = call(m, c, torch.bfloat16)
    assert not got[1].any() and not torch.isfinite(got[2]).any() and not torch.isfinite(got[4]).any()
    rest = [i for i in range(c["B"]) if i not in (1, 2, 4)]
    assert torch.equal(got[rest], clean[rest])
    c["ws"][0][1, 7] = np.nan         # a weight column's scale: the rows of that expert
    got = call(m, c, torch.bfloat16)
    assert not torch.isfinite(got[rows[0]:]).any() and torch.equal(got[0], clean[0])


def test_the_largest_sums():
    """16384 products of 127 and -128: exact in 32 bits, and the activation overflows nothing."""
    import paper_2508_13337_amd as m
    c = make([2, 40], 16384, 64, False)
    c["x"][:] = 127
    c["w"][0][:], c["w"][1][:] = -128, 127
    c["w"][0][:, 1::2] = 127
    c["xs"][:] = 1e-4
    for s in c["ws"][:2]:
        s[:] = 1e-4
    check(c, call(m, c, torch.float32), torch.float32)


@pytest.mark.parametrize("dt", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("E,K,N", [(1, 1, 1), (3, 128, 64), (2, 200, 77), (1, 1409, 130), (2, 63, 257)])
def test_quantised_weights(E, K, N, dt):
    import paper_2508_13337_amd as m
    w = (torch.randn((E, K, N), generator=torch.Generator().manual_seed(K)) * 0.02).to(dt)
    w[0, :, N // 2] = 0
    wq = torch.full((E + 1, N, pitch(K)), 99, dtype=torch.int8, device="cuda")
    scale = torch.full((E + 1, N), 7.0, device="cuda")
    m.xmoe_quantize_weights(w.cuda(), wq[:E], scale[:E])
    torch.cuda.synchronize()
    assert bool((wq[E] == 99).all()) and bool((scale[E] == 7.0).all())
    want, mx = oracle.quantize_rows_f32(w.float().numpy().transpose(0, 2, 1))
    got = wq[:E].cpu().numpy()
    assert np.array_equal(got[..., :K], want) and not got[..., K:].any()
    assert np.array_equal(scale[:E].cpu().numpy(), mx / np.float32(127))
