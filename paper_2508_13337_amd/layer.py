"""One padding-free MoE layer as a sequence of libxmoe calls (Listing 1's call(): gating -> PFT construction
-> dispatch -> mlp -> combine, then the mirrored backward).  This class only owns the device buffers and the
order of the calls; all arithmetic happens inside the HIP kernels."""
from __future__ import annotations

from typing import Optional

import torch

from . import api


def append_shared(w_routed: torch.Tensor, w_shared: Optional[torch.Tensor]) -> torch.Tensor:
    """Weights of the E routed experts followed by those of the E_s shared experts, [E+E_s, ...]: the layout the
    layer hands to the expert-MLP calls.  Pure data movement."""
    if w_shared is None or w_shared.shape[0] == 0:
        return w_routed
    return torch.cat([w_routed, w_shared], dim=0).contiguous()


class XMoELayer:
    """Buffers and call order for one layer of T tokens; weights are passed in by the caller.

    The gather of dispatch is fused into the expert MLP's operand loads: the MLP reads x through token_ids, and no
    [B,d] copy of the tokens exists.  The backward of combine is fused the same way (fuse_combine_bwd, the default):
    the MLP's backward reads dOut through token_ids and scales by combine_weights, so no [B,d] gradient of the expert
    outputs exists, and it also returns the gradient of every row's combine weight (dy_row_scale_grad), which
    xmoe_route_bwd_rows takes from there: the expert outputs Y are then read by the forward combine only
    and nothing but G and U is held between forward and backward.  (Without fuse_combine_bwd, xmoe_combine_bwd
    reads Y back for the weights' gradient and writes dY, and xmoe_dispatch copies dOut into the shared experts'
    dY rows.)
    norm_eps: None, or the layer starts with a root-mean-square norm: forward(x, w, residual) adds the residual (optional)
    into self.h, normalises that with w["norm_gain"] into self.xn, and the layer runs on xn; backward also takes the
    gradient dh that reaches h by other ways and gives grads["dnorm_gain"] and the gradient of x (and of the residual).
    Shared experts (every token, weight 1) run inside the same grouped-GEMM launches as the routed ones: they are
    experts E .. E+E_s-1 whose segments are rows [B + s*T, B + (s+1)*T) and read x[0..T-1], so the tail of
    expert_offsets and of token_ids is constant and written once here."""

    def __init__(self, T: int, d: int, E: int, k: int, f: int, dtype: torch.dtype, E_s: int = 0, device="cuda",
                 max_token_count: Optional[int] = None, fuse_combine_bwd: bool = True, norm_eps: Optional[float] = None):
        self.T, self.d, self.E, self.k, self.f, self.E_s = T, d, E, k, f, E_s
        self.norm_eps = norm_eps
        self.fuse_combine_bwd = fuse_combine_bwd
        # None: dropless.  Else the per-expert capacity of the token-dropping PFT construction; the number of
        # retained rows is then known on the device only, and xmoe_append_shared_segments continues the index arrays
        # with the shared experts' segments behind them, every step.
        self.max_token_count = max_token_count
        self.dtype, self.device = dtype, device
        B = T * k
        R = B + E_s * T          # rows of the expert MLP
        Ea = E + E_s             # experts of the expert MLP
        self.B, self.R, self.Ea = B, R, Ea
        dt = api.dtype_code(dtype)
        i32 = dict(dtype=torch.int32, device=device)
        f32 = dict(dtype=torch.float32, device=device)
        act = dict(dtype=dtype, device=device)
        self.logits = torch.empty((T, E), **f32)
        self.topk_idx = torch.empty((T, k), **i32)
        self.topk_w = torch.empty((T, k), **f32)
        self.tokens_per_expert = torch.empty(E, **i32)
        self.offsets_all = torch.empty(Ea + 1, **i32)
        self.token_ids_all = torch.empty(R, **i32)
        if E_s > 0:
            self.offsets_all[E + 1:] = B + T * torch.arange(1, E_s + 1, **i32)
            self.token_ids_all[B:] = torch.arange(T, **i32).repeat(E_s)
        self.expert_offsets = self.offsets_all[:E + 1]
        self.token_ids = self.token_ids_all[:B]
        self.expert_ids = torch.empty(B, **i32)
        # combine weight of every row of the expert MLP: the ERI-array for the routed rows, 1 for a shared expert's
        self.combine_weights_all = torch.ones(R, **f32)
        self.combine_weights = self.combine_weights_all[:B]
        self.row_of_slot = torch.empty(B, **i32)
        self.g = torch.empty((R, f), **act)
        self.u = torch.empty((R, f), **act)
        self.y = torch.empty((R, d), **act)
        self.out = torch.empty((T, d), **act)
        # backward
        self.dy = None if fuse_combine_bwd else torch.empty((R, d), **act)
        self.row_grad = torch.empty(R, **f32) if fuse_combine_bwd else None   # gradient of every row's combine weight
        self.dw = torch.empty((T, k), **f32)
        self.dxd = torch.empty((R, d), **act)
        self.dlogits = torch.empty((T, E), **f32)
        self.dx_gate = torch.empty((T, d), **act)
        self.dx = torch.empty((T, d), **act)
        ws = max(api.xmoe_workspace_bytes(api.WS_BUILD_ERI, T, d, E, k, f, dt),
                 api.xmoe_workspace_bytes(api.WS_FFN_FWD, R, d, Ea, k, f, dt),
                 api.xmoe_workspace_bytes(api.WS_FFN_BWD, R, d, Ea, k, f, dt),
                 api.xmoe_workspace_bytes(api.WS_GATE_BWD, T, d, E, k, f, dt))
        if max_token_count is not None:
            ws = max(ws, api.xmoe_workspace_bytes(api.WS_BUILD_ERI_CAPPED, T, d, E, k, f, dt))
        if norm_eps is not None:
            ws = max(ws, api.xmoe_workspace_bytes(api.WS_ADD_RMSNORM_BWD, T, d, E, k, f, dt))
            self.h, self.xn = torch.empty((T, d), **act), torch.empty((T, d), **act)
            self.rstd = torch.empty(T, **f32)
            self.dx_norm = torch.empty((T, d), **act)
        self.ws = api.alloc_workspace(ws, device)

    # weights: dict with w_router [d,E], bias [E]|None, wg/wu [E+E_s,d,f], wd [E+E_s,f,d] (routed experts first,
    # see append_shared), norm_gain [d] with norm_eps
    def forward(self, x: torch.Tensor, w: dict, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
        if self.norm_eps is not None:
            api.xmoe_add_rmsnorm(x, residual, w["norm_gain"], self.norm_eps, self.h, y=self.xn, rstd=self.rstd)
            x = self.xn
        elif residual is not None:
            raise ValueError("a residual is added by the norm: the layer has none (norm_eps)")
        api.xmoe_gate_logits(x, w["w_router"], w.get("bias"), self.logits)
        api.xmoe_route(self.logits, self.k, self.topk_idx, self.topk_w)
        B, E, T, E_s = self.B, self.E, self.T, self.E_s
        if self.max_token_count is None:
            api.xmoe_build_eri(self.topk_idx, self.topk_w, E, self.tokens_per_expert, self.expert_offsets,
                               self.token_ids, self.expert_ids, self.combine_weights, self.row_of_slot, self.ws)
        else:
            api.xmoe_build_eri_capped(self.topk_idx, self.topk_w, E, self.max_token_count, self.tokens_per_expert,
                                      self.expert_offsets, self.token_ids, self.expert_ids, self.combine_weights,
                                      self.row_of_slot, self.ws)
            if E_s > 0:   # the shared experts' segments start behind the retained rows, a count only the device has
                api.xmoe_append_shared_segments(self.offsets_all, self.token_ids_all, self.combine_weights_all, T, E,
                                                E_s)
        api.xmoe_expert_ffn_fwd(x, self.offsets_all, w["wg"], w["wu"], w["wd"], self.g, self.u, self.y,
                                self.ws, row_index=self.token_ids_all)
        y, y_shared, kw = self._row_args(self.y)
        api.xmoe_combine(y, self.row_of_slot, self.topk_w, y_shared, None, self.k, self.out, **kw)
        return self.out

    def _row_args(self, rows: torch.Tensor):
        """How xmoe_combine / xmoe_dispatch_bwd find the routed and the shared experts' rows in `rows` [R,d]:
        (routed rows, shared rows, keyword arguments)."""
        B, E, E_s = self.B, self.E, self.E_s
        if E_s == 0:
            return rows[:B], None, {}
        if self.max_token_count is None:
            return rows[:B], rows[B:], {}
        # the shared segments start behind the retained rows: their first row is expert_offsets[E], on the device
        return rows, rows, {"shared_row0": self.offsets_all[E:E + 1], "n_shared": E_s}

    def backward(self, x: torch.Tensor, w: dict, dout: torch.Tensor, grads: dict,
                 dh: Optional[torch.Tensor] = None) -> torch.Tensor:
        """grads: preallocated dw_router, dwg, dwu, dwd in the layouts of the weights (with norm_eps: dnorm_gain too).
        dh: None, or the gradient that reaches the normalised sum by other ways (norm_eps)."""
        B = self.B
        if self.norm_eps is not None:
            x = self.xn
        elif dh is not None:
            raise ValueError("dh is the gradient of the norm's sum: the layer has no norm (norm_eps)")
        if self.fuse_combine_bwd:
            api.xmoe_expert_ffn_bwd(x, self.g, self.u, dout, self.offsets_all, w["wg"], w["wu"], w["wd"],
                                    self.dxd, grads["dwg"], grads["dwu"], grads["dwd"], self.ws,
                                    row_index=self.token_ids_all, dy_row_index=self.token_ids_all,
                                    dy_row_scale=self.combine_weights_all, dy_row_scale_grad=self.row_grad)
            api.xmoe_route_bwd_rows(self.logits, self.topk_idx, self.row_grad, self.row_of_slot, self.dw, self.dlogits)
        else:
            if self.E_s > 0:   # dY of a shared expert's rows is dout itself
                if self.max_token_count is None:
                    api.xmoe_dispatch(dout, self.token_ids_all[B:], self.dy[B:])
                else:          # their first row is known on the device only: every row, the routed ones overwritten next
                    api.xmoe_dispatch(dout, self.token_ids_all, self.dy)
            api.xmoe_combine_bwd(dout, self.y[:B], self.row_of_slot, self.topk_w, self.dy[:B], self.dw)
            api.xmoe_expert_ffn_bwd(x, self.g, self.u, self.dy, self.offsets_all, w["wg"], w["wu"], w["wd"],
                                    self.dxd, grads["dwg"], grads["dwu"], grads["dwd"], self.ws,
                                    row_index=self.token_ids_all)
            api.xmoe_route_bwd(self.logits, self.topk_idx, self.dw, self.dlogits)
        api.xmoe_gate_logits_bwd(x, w["w_router"], self.dlogits, grads["dw_router"], self.dx_gate, self.ws)
        dxd, dxd_shared, kw = self._row_args(self.dxd)
        api.xmoe_dispatch_bwd(dxd, self.row_of_slot, dxd_shared, self.dx_gate, self.k, self.dx, **kw)
        if self.norm_eps is None:
            return self.dx
        api.xmoe_add_rmsnorm_bwd(self.dx, dh, self.h, w["norm_gain"], self.rstd, self.dx_norm, grads["dnorm_gain"], self.ws)
        return self.dx_norm


def capture_step(layer, x: torch.Tensor, w: dict, dout: torch.Tensor, grads: dict, residual: Optional[torch.Tensor] = None,
                 dh: Optional[torch.Tensor] = None) -> "torch.cuda.CUDAGraph":
    """Records one forward + backward of `layer` (either class; residual, dh: for one with a norm) into a HIP graph and
    returns it; `graph.replay()` then runs the step with one launch instead of two dozen.  The library's calls only
    enqueue kernels on the current stream (no allocation, no synchronisation, no memset nodes: counters are cleared by
    kernels), so they can be captured as they are.  All tensors are captured by address: refill x, dout and the weights
    in place."""
    more = {} if residual is None else {"residual": residual}
    more_bwd = {} if dh is None else {"dh": dh}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):          # warm-up outside the capture (first-use initialisation of the library)
        layer.forward(x, w, **more)
        layer.backward(x, w, dout, grads, **more_bwd)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer.forward(x, w, **more)
        layer.backward(x, w, dout, grads, **more_bwd)
    return graph


def quantize_experts(w: dict) -> dict:
    """The weights of XMoEServe with 8-bit experts: wg, wu, wd replaced by wgq, wuq, wdq and their scales.  Done once."""
    out = {n: t for n, t in w.items() if n not in ("wg", "wu", "wd")}
    for n in ("g", "u", "d"):
        E, K, N = w["w" + n].shape
        out[f"w{n}q"] = torch.empty((E, N, api.xmoe_q8_pitch(K)), dtype=torch.int8, device=w["w" + n].device)
        out[f"{n}_scale"] = torch.empty((E, N), dtype=torch.float32, device=w["w" + n].device)
        api.xmoe_quantize_weights(w["w" + n], out[f"w{n}q"], out[f"{n}_scale"])
    return out


class XMoEServe:
    """The MoE block of a serving step, forward only, for up to T tokens a call: h = x + residual, the norm, the layer.  Buffers
    and call order.  Up to FEW_TOKENS tokens take xmoe_layer_few_fwd; more, the layer's calls; with q8 the experts run on
    8-bit rows, which the norm makes, and 8-bit weights (quantize_experts): faster from a few tokens on (d 2048, f 1408, 6 of 64
    experts + 2, us, bf16 | 8-bit: 1 token 51 | 73, 2 tokens 68 | 74, 8 tokens 136 | 102, 1024 360 | 236), as they always take
    the layer's calls.  Shared experts as in XMoELayer."""

    def __init__(self, T: int, d: int, E: int, k: int, f: int, dtype: torch.dtype, E_s: int = 0, eps: float = 1e-6,
                 q8: bool = False, device="cuda"):
        self.T, self.d, self.E, self.k, self.f, self.E_s, self.eps, self.q8 = T, d, E, k, f, E_s, eps, q8
        R, Ea, few = T * (k + E_s), E + E_s, min(T, api.FEW_TOKENS)
        dt = api.dtype_code(dtype)
        i32 = dict(dtype=torch.int32, device=device)
        f32 = dict(dtype=torch.float32, device=device)
        act = dict(dtype=dtype, device=device)
        self.h, self.xn, self.out = (torch.empty((T, d), **act) for _ in range(3))
        self.logits = torch.empty((T, E), **f32)
        self.topk_idx, self.topk_w = torch.empty((T, k), **i32), torch.empty((T, k), **f32)
        self.tokens_per_expert, self.offsets = torch.empty(E, **i32), torch.empty(Ea + 1, **i32)
        self.token_ids, self.combine_weights = torch.empty(R, **i32), torch.empty(R, **f32)
        self.expert_ids, self.row_of_slot = torch.empty(T * k, **i32), torch.empty(T * k, **i32)
        ws = [api.xmoe_workspace_bytes(api.WS_BUILD_ERI, T, d, E, k, f, dt)]
        if q8:
            self.q = torch.empty((T, api.xmoe_q8_pitch(d)), dtype=torch.int8, device=device)
            self.q_scale = torch.empty(T, **f32)
            ws.append(api.xmoe_workspace_bytes(api.WS_FFN_Q8_FWD, R, d, Ea, k, f, dt))
        else:
            ws.append(api.xmoe_workspace_bytes(api.WS_LAYER_FEW_FWD, few, d, Ea, k + E_s, f, dt))
        if q8 or T > api.FEW_TOKENS:
            self.y = torch.empty((R, d), **act)
            if not q8:
                self.g, self.u = torch.empty((R, f), **act), torch.empty((R, f), **act)
                ws.append(api.xmoe_workspace_bytes(api.WS_FFN_FWD, R, d, Ea, k, f, dt))
        self.ws = api.alloc_workspace(max(ws), device)

    # weights: norm_gain [d], w_router [d,E], bias [E]|None, wg/wu [E+E_s,d,f], wd [E+E_s,f,d] or what quantize_experts made
    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor], w: dict):
        """(out, h): the layer's output for x [t,d], t <= T, and the sum that the next residual is.  Both are buffers of this
        object, and the next call's."""
        t, E, k, E_s = x.shape[0], self.E, self.k, self.E_s
        if t > self.T:
            raise ValueError(f"{t} tokens: this block has buffers for {self.T}")
        if t == 0:
            return self.out[:0], self.h[:0]
        B, R = t * k, t * (k + E_s)
        h, xn, out = self.h[:t], self.xn[:t], self.out[:t]
        logits, idx, topk_w = self.logits[:t], self.topk_idx[:t], self.topk_w[:t]
        q = dict(q=self.q[:t], q_scale=self.q_scale[:t]) if self.q8 else {}
        api.xmoe_add_rmsnorm(x, residual, w["norm_gain"], self.eps, h, y=xn, **q)
        if not self.q8 and t <= api.FEW_TOKENS:
            api.xmoe_layer_few_fwd(xn, w["w_router"], w.get("bias"), w["wg"], w["wu"], w["wd"], None, logits, idx, topk_w,
                                   out, self.ws)
            return out, h
        api.xmoe_gate_logits(xn, w["w_router"], w.get("bias"), logits)
        api.xmoe_route(logits, k, idx, topk_w)
        token_ids, combine_weights, row_of_slot = self.token_ids[:R], self.combine_weights[:R], self.row_of_slot[:B]
        api.xmoe_build_eri(idx, topk_w, E, self.tokens_per_expert, self.offsets[:E + 1], token_ids[:B], self.expert_ids[:B],
                           combine_weights[:B], row_of_slot, self.ws)
        if E_s > 0:
            api.xmoe_append_shared_segments(self.offsets, token_ids, combine_weights, t, E, E_s)
        y = self.y[:R]
        if self.q8:
            api.xmoe_expert_ffn_q8_fwd(self.q[:t], self.q_scale[:t], self.offsets, w["wgq"], w["g_scale"], w["wuq"],
                                       w["u_scale"], w["wdq"], w["d_scale"], y, self.ws, row_index=token_ids)
        else:
            api.xmoe_expert_ffn_fwd(xn, self.offsets, w["wg"], w["wu"], w["wd"], self.g[:R], self.u[:R], y, self.ws,
                                    row_index=token_ids)
        api.xmoe_combine(y[:B], row_of_slot, topk_w, y[B:] if E_s else None, None, k, out)
        return out, h


class XMoE2Layer:
    """The same layer with the paper's own expert, Y = act(X W1) W2 (Listing 1's call(tokens, k, max_token_count,
    w1, w2)).  Buffers and call order only; dropless; the gather of dispatch is fused into the expert MLP's loads."""

    def __init__(self, T: int, d: int, E: int, k: int, f: int, dtype: torch.dtype, act: str = "gelu", device="cuda",
                 fuse_combine_bwd: bool = True):
        self.T, self.d, self.E, self.k, self.f, self.act = T, d, E, k, f, act
        self.fuse_combine_bwd = fuse_combine_bwd
        B = T * k
        self.B = B
        dt = api.dtype_code(dtype)
        i32 = dict(dtype=torch.int32, device=device)
        f32 = dict(dtype=torch.float32, device=device)
        tt = dict(dtype=dtype, device=device)
        self.logits = torch.empty((T, E), **f32)
        self.topk_idx = torch.empty((T, k), **i32)
        self.topk_w = torch.empty((T, k), **f32)
        self.tokens_per_expert = torch.empty(E, **i32)
        self.expert_offsets = torch.empty(E + 1, **i32)
        self.token_ids = torch.empty(B, **i32)
        self.expert_ids = torch.empty(B, **i32)
        self.combine_weights = torch.empty(B, **f32)
        self.row_of_slot = torch.empty(B, **i32)
        self.h = torch.empty((B, f), **tt)
        self.y = torch.empty((B, d), **tt)
        self.out = torch.empty((T, d), **tt)
        self.dy = None if fuse_combine_bwd else torch.empty((B, d), **tt)
        self.row_grad = torch.empty(B, **f32) if fuse_combine_bwd else None
        self.dw = torch.empty((T, k), **f32)
        self.dxd = torch.empty((B, d), **tt)
        self.dlogits = torch.empty((T, E), **f32)
        self.dx_gate = torch.empty((T, d), **tt)
        self.dx = torch.empty((T, d), **tt)
        ws = max(api.xmoe_workspace_bytes(api.WS_BUILD_ERI, T, d, E, k, f, dt),
                 api.xmoe_workspace_bytes(api.WS_MLP2_FWD, B, d, E, k, f, dt),
                 api.xmoe_workspace_bytes(api.WS_MLP2_BWD, B, d, E, k, f, dt),
                 api.xmoe_workspace_bytes(api.WS_GATE_BWD, T, d, E, k, f, dt))
        self.ws = api.alloc_workspace(ws, device)

    # weights: dict with w_router [d,E], bias [E]|None, w1 [E,d,f], w2 [E,f,d]
    def forward(self, x: torch.Tensor, w: dict) -> torch.Tensor:
        api.xmoe_gate_logits(x, w["w_router"], w.get("bias"), self.logits)
        api.xmoe_route(self.logits, self.k, self.topk_idx, self.topk_w)
        api.xmoe_build_eri(self.topk_idx, self.topk_w, self.E, self.tokens_per_expert, self.expert_offsets,
                           self.token_ids, self.expert_ids, self.combine_weights, self.row_of_slot, self.ws)
        api.xmoe_expert_mlp2_fwd(x, self.expert_offsets, w["w1"], w["w2"], self.act, self.h, self.y, self.ws,
                                 row_index=self.token_ids)
        api.xmoe_combine(self.y, self.row_of_slot, self.topk_w, None, None, self.k, self.out)
        return self.out

    def backward(self, x: torch.Tensor, w: dict, dout: torch.Tensor, grads: dict) -> torch.Tensor:
        """grads: preallocated dw_router, dw1, dw2 in the layouts of the weights."""
        if self.fuse_combine_bwd:   # dY is never written and Y is not read back (see XMoELayer)
            api.xmoe_expert_mlp2_bwd(x, self.h, dout, self.expert_offsets, w["w1"], w["w2"], self.act, self.dxd,
                                     grads["dw1"], grads["dw2"], self.ws, row_index=self.token_ids,
                                     dy_row_index=self.token_ids, dy_row_scale=self.combine_weights,
                                     dy_row_scale_grad=self.row_grad)
            api.xmoe_route_bwd_rows(self.logits, self.topk_idx, self.row_grad, self.row_of_slot, self.dw, self.dlogits)
        else:
            api.xmoe_combine_bwd(dout, self.y, self.row_of_slot, self.topk_w, self.dy, self.dw)
            api.xmoe_expert_mlp2_bwd(x, self.h, self.dy, self.expert_offsets, w["w1"], w["w2"], self.act, self.dxd,
                                     grads["dw1"], grads["dw2"], self.ws, row_index=self.token_ids)
            api.xmoe_route_bwd(self.logits, self.topk_idx, self.dw, self.dlogits)
        api.xmoe_gate_logits_bwd(x, w["w_router"], self.dlogits, grads["dw_router"], self.dx_gate, self.ws)
        api.xmoe_dispatch_bwd(self.dxd, self.row_of_slot, None, self.dx_gate, self.k, self.dx)
        return self.dx
