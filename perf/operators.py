"""The operators of a serving step around the MoE layer, as cases that can be timed and compared: the residual's addition
with a root-mean-square norm (its 8-bit output, its backward), the SwiGLU experts' products in 8-bit integers, and a whole
MoE layer for a few tokens.  `run` computes them in plain torch, or (`own`) through the library.

Shapes are those of xmoe_inputs.CONFIGS and generic ones in between.  A case is a dict of plain values:
  what    "norm" (h = x + residual, y = norm(h) * gain), "norm_q8" (the same with y as 8-bit rows and their scales),
          "norm_train" (norm, then the gradients of x and gain), "ffn_q8" (the expert MLP on 8-bit rows and weights),
          "few" (gate, top-k, experts and weighted sum for at most 32 tokens)
  dtype   "bf16" | "f32"
  T, d    tokens, model width
  E, k, f, E_s   experts, experts per token, expert width, shared experts ("ffn_q8", "few")
  skew    steepness of the experts' load profile (0: near-uniform)
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6


def _case(name, what, dtype="bf16", T=1, d=2048, E=0, k=0, f=0, E_s=0, skew=0.0):
    c = dict(what=what, dtype=dtype, T=T, d=d, E=E, k=k, f=f, E_s=E_s, skew=skew)
    return dict(c, name=name) if name else c


def listed():
    small = dict(d=2048, E=64, k=6, f=1408, E_s=2)   # the DeepSeek-MoE-16B-shaped layer
    return [
        # in front of the MoE layer of one decoding step, 16 sequences: a launch and its latency
        _case("norm_step", "norm_q8", T=16),
        # the same while prompts are processed, at the large model's width: memory alone
        _case("norm_prompts", "norm_q8", T=4096, d=7168),
        # the norm of a training step, forward and backward
        _case("norm_train", "norm_train", T=8192),
        # full-precision training of a small model at a width that no vector divides
        _case("norm_train_odd", "norm_train", dtype="f32", T=1021, d=1003),
        # the large model's norm, served in bf16, for a batch of long prompts
        _case("norm_long", "norm", T=16384, d=7168),
        # one decoding step of 8 sequences: the active experts' 8-bit weights are read for a handful of rows
        _case("q8_step", "ffn_q8", T=8, **small),
        # the prompt of one request: a few dozen rows per expert
        _case("q8_prompt", "ffn_q8", T=509, **small),
        # the prompts of a batch: the products are bound by the matrix cores
        _case("q8_batch", "ffn_q8", T=8192, **small),
        # widths that are no multiple of any tile, a skewed load, empty experts
        _case("q8_odd", "ffn_q8", T=1501, d=1000, E=24, k=3, f=712, skew=1.25),
        # one token of one sequence: the latency of a decoding step
        _case("few_one", "few", **small),
        # a step of 16 sequences: most experts are active, with one or two rows each
        _case("few_step", "few", T=16, **small),
        # full precision at odd widths, a toy model's step
        _case("few_odd_f32", "few", dtype="f32", T=3, d=1003, E=16, k=4, f=705, E_s=1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: every family of listed() over its range, none dearer than the largest listed one."""
    while True:
        what = rng.choice(["norm", "norm_q8", "norm_train", "ffn_q8", "ffn_q8", "ffn_q8", "few", "few", "few"])
        dtype = "bf16"
        if what.startswith("norm"):
            if what != "norm_q8" and rng.random() < 0.3:
                dtype = "f32"
            c = _case("", what, dtype=dtype, T=_log(rng, 1, 32768), d=_log(rng, 64, 8192) // rng.choice([1, 1, 8, 64]))
            if rng.random() < 0.6:
                c["d"] = (c["d"] + 63) // 64 * 64
        else:
            E = rng.choice([4, 8, 16, 24, 32, 64, 96, 128, 256])
            k = rng.randint(1, min(8, E))
            step = rng.choice([64, 64, 64, 8, 8, 1])
            if what == "few" and rng.random() < 0.25:
                dtype = "f32"
            c = _case("", what, dtype=dtype, T=_log(rng, 1, 32 if what == "few" else 16384),
                      d=max(step, _log(rng, 128, 7168) // step * step), E=E, k=k,
                      f=max(step, _log(rng, 64, 2560) // step * step), E_s=rng.choice([0, 0, 1, 2]),
                      skew=rng.choice([0.0, 0.0, 0.6, 1.25]))
        w = work(c)
        if w["bytes"] <= 9.3e8 and w["flops"] <= 1.13e12 and _held(c) <= 2e10:
            return c


def _held(c):
    """Bytes that a case and its plain form hold: weights, their values in 32 bits, every expert's rows padded alike."""
    T, d, E, k, f, E_s = (c[n] for n in ("T", "d", "E", "k", "f", "E_s"))
    if c["what"].startswith("norm"):
        return 0
    if c["what"] == "few":
        return (6 * (E + E_s) + 8 * T * (k + E_s)) * d * f
    return 14 * (E + E_s) * d * f + 4 * E * (1.3 * max(_rows(c)) + 20) * (2 * d + 4 * f)


def _pitch(n):
    """Bytes of an 8-bit row of n values: a multiple of 128, the tail holds zeros."""
    return (n + 127) // 128 * 128


def _weights_q8(E, K, N, gen):
    """E matrices of K inputs and N outputs as a checkpoint in 8-bit integers holds them: [E, N, pitch(K)] with one scale
    for each output."""
    q = torch.zeros((E, N, _pitch(K)), dtype=torch.int8, device="cuda")
    scale = torch.empty((E, N), dtype=torch.float32, device="cuda")
    for e in range(E):
        w = torch.empty((N, K), device="cuda").normal_(0.0, 0.02, generator=gen)
        m = w.abs().amax(1)
        q[e, :, :K] = torch.round(w * (127.0 / m)[:, None]).to(torch.int8)
        scale[e] = m / 127.0
    return q, scale


def prepare(case, seed):
    """Weights, one batch and the buffers of its results, all on the GPU."""
    c = case
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    dt = DTYPES[c["dtype"]]
    T, d, E, k, f, E_s = (c[n] for n in ("T", "d", "E", "k", "f", "E_s"))

    def normal(shape, std=1.0, dtype=dt):
        return torch.empty(shape, dtype=dtype, device="cuda").normal_(0.0, std, generator=g)

    s = {"case": c}
    i32 = dict(dtype=torch.int32, device="cuda")
    f32 = dict(dtype=torch.float32, device="cuda")
    if c["what"].startswith("norm"):
        s["x"], s["residual"] = normal((T, d)), normal((T, d), 2.0)
        s["gain"] = (1.0 + 0.1 * normal(d, dtype=torch.float32)).to(dt)
        s["h"] = torch.empty_like(s["x"])
        if c["what"] == "norm_q8":
            s["q"], s["q_scale"] = torch.zeros((T, _pitch(d)), dtype=torch.int8, device="cuda"), torch.empty(T, **f32)
            s["values"] = torch.empty_like(s["x"])
        else:
            s["y"] = torch.empty_like(s["x"])
        if c["what"] == "norm_train":
            s["dy"], s["dh"] = normal((T, d)), normal((T, d))
            s["rstd"], s["dx"], s["dgain"] = torch.empty(T, **f32), torch.empty_like(s["x"]), torch.empty_like(s["gain"])
        return s
    bias = None
    if c["skew"]:      # bias[e] = -skew * 1.2 * ln(rank of e), ranks in random order
        rank = torch.randperm(E, generator=g, device="cuda") + 1
        bias = -c["skew"] * 1.2 * torch.log(rank.float())
    if c["what"] == "few":
        s["x"], s["residual"], s["bias"] = normal((T, d)), normal((T, d)), bias
        s["w_router"] = normal((d, E), d ** -0.5)
        for n in ("wg", "wu", "wd"):
            s[n] = normal((E + E_s,) + ((f, d) if n == "wd" else (d, f)), 0.02)
        s["logits"], s["out"] = torch.empty((T, E), **f32), torch.empty_like(s["x"])
        s["topk_idx"], s["topk_w"] = torch.empty((T, k), **i32), torch.empty((T, k), **f32)
        return s
    # the rows in the experts' order, as the routing of the batch left them; the shared experts' behind them
    logits = torch.empty((T, E), **f32).normal_(generator=g)
    idx = torch.topk(logits if bias is None else logits + bias, k, dim=1).indices.reshape(-1)
    order = torch.sort(idx, stable=True).indices
    count = torch.bincount(idx, minlength=E)
    s["offsets"] = torch.zeros(E + E_s + 1, **i32)
    s["offsets"][1:E + 1] = torch.cumsum(count, 0)
    s["offsets"][E + 1:] = T * k + T * torch.arange(1, E_s + 1, **i32)
    s["token_ids"] = torch.cat([(order // k).to(torch.int32), torch.arange(T, **i32).repeat(E_s)])
    s["most"] = int(count.max())      # the rows of the busiest expert
    x = normal((T, d), dtype=torch.float32)
    m = x.abs().amax(1)
    s["xq"] = torch.zeros((T, _pitch(d)), dtype=torch.int8, device="cuda")
    s["xq"][:, :d] = torch.round(x * (127.0 / m)[:, None]).to(torch.int8)
    s["x_scale"] = m / 127.0
    for n, (K, N) in {"g": (d, f), "u": (d, f), "d": (f, d)}.items():
        s["w%sq" % n], s["%s_scale" % n] = _weights_q8(E + E_s, K, N, g)
    s["y"] = torch.empty((T * (k + E_s), d), dtype=dt, device="cuda")
    return s


# ----------------------------------------------------------------------------------------------------------
# the plain forms
# ----------------------------------------------------------------------------------------------------------
def _norm_plain(s):
    c = s["case"]
    dt = s["x"].dtype
    h = (s["x"].float() + s["residual"].float()).to(dt)
    hf, gain = h.float(), s["gain"].float()
    r = 1.0 / torch.sqrt(hf.square().mean(1, keepdim=True) + EPS)
    if c["what"] == "norm_q8":     # the factor r scales a row and its maximum alike: the integers do not depend on it
        v = hf * gain
        m = v.abs().amax(1, keepdim=True)
        q = torch.round(v * torch.where(m > 0, 127.0 / m, 0.0))
        scale = m * r / 127.0
        return [h, (q * scale).to(dt), scale[:, 0]]
    y = (hf * r * gain).to(dt)
    if c["what"] == "norm":
        return [h, y]
    n, dy = hf * r, s["dy"].float()
    dn = dy * gain
    dx = r * (dn - n * (dn * n).mean(1, keepdim=True)) + s["dh"].float()
    return [h, y, dx.to(dt), (dy * n).sum(0).to(dt)]


def _quantised(a):
    """The values that rows of 8-bit integers with one scale stand for, nearest to a."""
    m = a.abs().amax(-1, keepdim=True)
    return torch.round(a * torch.where(m > 0, 127.0 / m, 0.0)) * (m / 127.0)


def _experts_plain(s, x, lo, hi):
    """x [experts lo to hi, rows, d] through their SwiGLU, A quantised between the products."""
    def w(n, K):
        q = s["w%sq" % n][lo:hi, :, :K].float() * s["%s_scale" % n][lo:hi, :, None]
        return q.transpose(1, 2).contiguous()
    d, f = s["case"]["d"], s["case"]["f"]
    gate, up = torch.bmm(x, w("g", d)), torch.bmm(x, w("u", d))
    return torch.bmm(_quantised(gate * torch.sigmoid(gate) * up), w("d", f))


def _ffn_q8_plain(s):
    c = s["case"]
    T, d, E, k, E_s, most = c["T"], c["d"], c["E"], c["k"], c["E_s"], s["most"]
    x = s["xq"][:, :d].float() * s["x_scale"][:, None]
    row = torch.arange(T * k, device="cuda")
    e = torch.searchsorted(s["offsets"][1:E + 1].long().contiguous(), row, right=True)
    place = e * most + row - s["offsets"].long()[e]        # every expert's rows, padded to the most that one has
    padded = torch.zeros((E * most, d), device="cuda")
    padded[place] = x[s["token_ids"][:T * k].long()]
    y = torch.empty((T * (k + E_s), d), device="cuda")
    y[:T * k] = _experts_plain(s, padded.view(E, most, d), 0, E).view(-1, d)[place]
    if E_s:
        y[T * k:] = _experts_plain(s, x.expand(E_s, T, d).contiguous(), E, E + E_s).view(-1, d)
    return [y.to(DTYPES[c["dtype"]])]


def _few_plain(s):
    c = s["case"]
    T, d, E, k, E_s = c["T"], c["d"], c["E"], c["k"], c["E_s"]
    logits = s["x"].double() @ s["w_router"].double()      # in 64 bits: two experts' logits may be close
    if s["bias"] is not None:
        logits = logits + s["bias"].double()
    idx = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :k]
    topk_w = torch.softmax(logits, 1).gather(1, idx).float()
    shared = torch.arange(E, E + E_s, device="cuda").expand(T, E_s)
    e = torch.cat([idx, shared], 1).reshape(-1)            # the experts of every token, one row each
    weight = torch.cat([topk_w, torch.ones((T, E_s), device="cuda")], 1)
    x = s["x"].float().repeat_interleave(k + E_s, 0)[:, None, :]
    gate, up = torch.bmm(x, s["wg"][e].float()), torch.bmm(x, s["wu"][e].float())
    y = torch.bmm(gate * torch.sigmoid(gate) * up, s["wd"][e].float()).view(T, k + E_s, d)
    out = (y * weight[:, :, None]).sum(1) + s["residual"].float()
    return [out.to(s["x"].dtype), idx.to(torch.int32), topk_w]


# ----------------------------------------------------------------------------------------------------------
# the library's calls
# ----------------------------------------------------------------------------------------------------------
def _workspace(s, xm, op, rows):
    """The scratch memory that a program sizes and allocates once."""
    if "ws" not in s:
        c = s["case"]
        n = xm.xmoe_workspace_bytes(op, rows, c["d"], c["E"] + c["E_s"], c["k"] + c["E_s"], c["f"],
                                    xm.dtype_code(DTYPES[c["dtype"]]))
        s["ws"] = xm.alloc_workspace(n)
    return s["ws"]


def _run_own(s):
    import paper_2508_13337_amd as xm
    c = s["case"]
    if c["what"] == "ffn_q8":
        ws = _workspace(s, xm, xm.WS_FFN_Q8_FWD, s["y"].shape[0])
        xm.xmoe_expert_ffn_q8_fwd(s["xq"], s["x_scale"], s["offsets"], s["wgq"], s["g_scale"], s["wuq"], s["u_scale"],
                                  s["wdq"], s["d_scale"], s["y"], ws, row_index=s["token_ids"])
        return [s["y"]]
    if c["what"] == "few":
        ws = _workspace(s, xm, xm.WS_LAYER_FEW_FWD, c["T"])
        xm.xmoe_layer_few_fwd(s["x"], s["w_router"], s["bias"], s["wg"], s["wu"], s["wd"], s["residual"], s["logits"],
                              s["topk_idx"], s["topk_w"], s["out"], ws)
        return [s["out"], s["topk_idx"], s["topk_w"]]
    if c["what"] == "norm_q8":
        xm.xmoe_add_rmsnorm(s["x"], s["residual"], s["gain"], EPS, s["h"], q=s["q"], q_scale=s["q_scale"])
        torch.mul(s["q"][:, :c["d"]], s["q_scale"][:, None], out=s["values"])
        return [s["h"], s["values"], s["q_scale"]]
    if c["what"] == "norm":
        xm.xmoe_add_rmsnorm(s["x"], s["residual"], s["gain"], EPS, s["h"], y=s["y"])
        return [s["h"], s["y"]]
    ws = _workspace(s, xm, xm.WS_ADD_RMSNORM_BWD, c["T"])
    xm.xmoe_add_rmsnorm(s["x"], s["residual"], s["gain"], EPS, s["h"], y=s["y"], rstd=s["rstd"])
    xm.xmoe_add_rmsnorm_bwd(s["dy"], s["dh"], s["h"], s["gain"], s["rstd"], s["dx"], s["dgain"], ws)
    return [s["h"], s["y"], s["dx"], s["dgain"]]


def run(state):
    if own:
        return _run_own(state)
    what = state["case"]["what"]
    if what == "ffn_q8":
        return _ffn_q8_plain(state)
    return _few_plain(state) if what == "few" else _norm_plain(state)


def _rows(c):
    """Expected rows of every routed expert: shares follow rank^(-1.2 skew), no expert gets a token twice."""
    share = [float(e + 1) ** (-1.2 * c["skew"]) for e in range(c["E"])]
    T, B = c["T"], c["T"] * c["k"]
    lo, hi = 0.0, B / min(share)
    for _ in range(60):
        mid = (lo + hi) / 2
        lo, hi = (mid, hi) if sum(min(T, mid * p) for p in share) < B else (lo, mid)
    return [min(T, hi * p) for p in share]


def work(case):
    c = case
    T, d, E, k, f, E_s = (c[n] for n in ("T", "d", "E", "k", "f", "E_s"))
    size = 4 if c["dtype"] == "f32" else 2
    token = T * d * size
    if c["what"] == "norm":
        return {"bytes": 4 * token + d * size, "flops": 5 * T * d}
    if c["what"] == "norm_q8":        # the 8-bit rows and the values they stand for
        return {"bytes": 4 * token + T * d + 4 * T + d * size, "flops": 7 * T * d}
    if c["what"] == "norm_train":     # x, residual, dy, dh in; h, y, dx out
        return {"bytes": 7 * token + 2 * d * size, "flops": 15 * T * d}
    # an expert is active if one of T tokens picks it, each with the probability of its share of them
    active = sum(1.0 - (1.0 - r / T) ** T for r in _rows(c)) + E_s
    flops = 6 * T * (k + E_s) * d * f
    if c["what"] == "ffn_q8":
        rows = T * (k + E_s)
        return {"bytes": active * (3 * d * f + 4 * (2 * f + d)) + T * (d + 4) + rows * (d * size + 4), "flops": flops}
    return {"bytes": (active * 3 * f + E) * d * size + 3 * token + T * (4 * E + 8 * k), "flops": flops + 2 * T * d * E}


# ----------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ----------------------------------------------------------------------------------------------------------
def _swiglu64(x, wg, wu):
    g = x @ wg
    return g / (1.0 + torch.exp(-g)) * (x @ wu)


def exact(case, seed):
    s, c = prepare(case, seed), case
    T, d, E, k, f, E_s = (c[n] for n in ("T", "d", "E", "k", "f", "E_s"))
    if c["what"].startswith("norm"):
        h = (s["x"].double() + s["residual"].double()).to(DTYPES[c["dtype"]])      # the stored sum is what is normalised
        x, gain = h.double(), s["gain"].double()
        rms = torch.sqrt((x * x).sum(1) / d + EPS)[:, None]
        y = x / rms * gain
        if c["what"] == "norm":
            return [None, y]
        if c["what"] == "norm_q8":
            step = y.abs().max(1, keepdim=True).values / 127
            return [None, torch.round(y / step) * step, step[:, 0]]
        # y_i = g_i x_i / rms:  d y_j / d x_i = g_j (delta_ij / rms - x_i x_j / (d rms^3))
        dy = s["dy"].double()
        inner = (dy * gain * x).sum(1, keepdim=True)
        dx = dy * gain / rms - x * inner / (d * rms ** 3) + s["dh"].double()
        return [None, y, dx, (dy * x / rms).sum(0)]
    if c["what"] == "few":
        x = s["x"].double()
        logits = x @ s["w_router"].double() + (0 if s["bias"] is None else s["bias"].double())
        p = torch.exp(logits - logits.max(1, keepdim=True).values)
        p = p / p.sum(1, keepdim=True)
        out, chosen = s["residual"].double(), torch.zeros((T, k), dtype=torch.float64, device="cuda")
        for t in range(T):
            best = sorted(range(E), key=lambda e, row=logits[t].tolist(): (-row[e], e))[:k]
            for j, e in enumerate(best):
                chosen[t, j] = p[t, e]
            for e in best + list(range(E, E + E_s)):
                a = _swiglu64(x[t], s["wg"][e].double(), s["wu"][e].double())
                out[t] += (p[t, e] if e < E else 1.0) * (a @ s["wd"][e].double())
        return [out, None, chosen]
    y = torch.empty((T * (k + E_s), d), dtype=torch.float32, device="cuda")        # bf16 results need no more
    ends = s["offsets"].tolist()
    x = s["xq"][:, :d].double() * s["x_scale"].double()[:, None]
    for e in range(E + E_s):
        rows = slice(ends[e], ends[e + 1])
        if ends[e] == ends[e + 1]:
            continue
        w = [(s["w%sq" % n][e].double() * s["%s_scale" % n][e].double()[:, None]).t() for n in "gud"]
        a = _swiglu64(x[s["token_ids"][rows].long()], w[0][:d], w[1][:d])
        step = a.abs().max(1, keepdim=True).values / 127
        step = torch.where(step > 0, step, 1.0)
        y[rows] = ((torch.round(a / step) * step) @ w[2][:f]).float()
    return [y]
