"""CPU oracle of what stands around the layer in a serving step: the residual's addition with a root-mean-square norm and
its backward, rows and weights in 8-bit integers, and the SwiGLU experts on them.

TEST INFRASTRUCTURE ONLY, like moe_oracle.py: float64 numpy, one step after the other, nothing of the HIP library."""
from __future__ import annotations

import numpy as np

from .moe_oracle import silu

__all__ = ["add_rmsnorm", "add_rmsnorm_bwd", "quantize_rows", "quantize_rows_f32", "expert_ffn_q8"]


def add_rmsnorm(h, gain, eps: float):
    """(y, r) of rows h [T, d] (the stored sum of x and the residual): r = 1 / sqrt(mean h^2 + eps), y = h r gain."""
    h = np.asarray(h, np.float64)
    r = 1.0 / np.sqrt((h * h).mean(axis=1) + eps)
    return h * r[:, None] * np.asarray(gain, np.float64), r


def add_rmsnorm_bwd(dy, dh, h, gain, eps: float):
    """(dx, dgain) by the quotient rule: y_j = g_j h_j / s with s = sqrt(mean h^2 + eps), so
    dy_j / dh_i = g_j (delta_ij / s - h_i h_j / (d s^3))."""
    dy, h, gain = (np.asarray(a, np.float64) for a in (dy, h, gain))
    d = h.shape[1]
    s = np.sqrt((h * h).mean(axis=1, keepdims=True) + eps)
    dx = dy * gain / s - h * (dy * gain * h).sum(axis=1, keepdims=True) / (d * s ** 3)
    if dh is not None:
        dx = dx + np.asarray(dh, np.float64)
    return dx, (dy * h / s).sum(axis=0)


def quantize_rows(v):
    """(integers, scale) of rows v [..., n] in float64: scale = max |v| / 127, integers = v / scale to the nearest, ties to
    even; a row of zeros has scale 0."""
    v = np.asarray(v, np.float64)
    m = np.abs(v).max(axis=-1)
    q = np.rint(v * np.where(m > 0, 127.0 / np.where(m > 0, m, 1.0), 0.0)[..., None])
    return q.astype(np.int64), m / 127.0


def quantize_rows_f32(v):
    """The integers as the library defines them, bit for bit: v float32, each step rounded to float32.  Rows whose maximum
    is below 2^-120 count as zero.  (integers, maximum)."""
    v = np.ascontiguousarray(v, np.float32)
    m = np.abs(v).max(axis=-1)
    none = m < np.float32(2.0 ** -120)
    inv = np.where(none, np.float32(0), np.float32(127) / np.where(none, np.float32(1), m)).astype(np.float32)
    return np.rint(v * inv[..., None]).astype(np.int8), np.where(none, np.float32(0), m)


def expert_ffn_q8(xq, x_scale, rows, expert_offsets, wgq, g_scale, wuq, u_scale, wdq, d_scale):
    """(Y, A, its integers, its scales): row i of the experts' input is x_scale * xq of row rows[i].  Weights [E, N, K] with
    one scale per output n; the integer sums are exact, the activation is quantised by rows between the products."""
    xq, wgq, wuq, wdq = (np.asarray(a).astype(np.float64) for a in (xq, wgq, wuq, wdq))   # sums below 2^53 are exact
    x_scale, g_scale, u_scale, d_scale = (np.asarray(a, np.float64) for a in (x_scale, g_scale, u_scale, d_scale))
    E, d, f = wgq.shape[0], wdq.shape[1], wgq.shape[1]
    B = int(expert_offsets[-1])
    Y, A = np.zeros((B, d)), np.zeros((B, f))
    AQ, AS = np.zeros((B, f), np.int64), np.zeros(B)
    for e in range(E):
        s = slice(int(expert_offsets[e]), int(expert_offsets[e + 1]))
        r = np.asarray(rows)[s]
        if len(r) == 0:
            continue
        G = (xq[r] @ wgq[e].T) * x_scale[r][:, None] * g_scale[e]
        U = (xq[r] @ wuq[e].T) * x_scale[r][:, None] * u_scale[e]
        A[s] = silu(G) * U
        AQ[s], AS[s] = quantize_rows(A[s])
        Y[s] = (AQ[s] @ wdq[e].T) * AS[s][:, None] * d_scale[e]
    return Y, A, AQ, AS
