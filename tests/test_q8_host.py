"""Refusals of the 8-bit entry points: each on the host, before anything is enqueued (no GPU)."""
import ctypes

import pytest

from test_norm_host import lib  # noqa: F401  (the library, built if it is not there)

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
P, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(4104)      # never dereferenced on the host
ARGS = dict(xq=P, x_scale=P, row_index=None, off=P, B=32, E=4, d=64, f=32, wgq=P, g_scale=P, wuq=P, u_scale=P, wdq=P,
            d_scale=P, y=P, dt=1, ws=P, ws_bytes=1 << 24)


def ffn(lib, **kw):  # noqa: F811
    return lib.xmoe_expert_ffn_q8_fwd(*{**ARGS, **kw}.values(), None)


def test_experts(lib):  # noqa: F811
    assert ffn(lib, dt=2) == UNSUPPORTED and ffn(lib, E=513) == UNSUPPORTED
    assert ffn(lib, d=65537) == UNSUPPORTED and ffn(lib, f=65537) == UNSUPPORTED
    for n, v in dict(B=-1, E=0, d=0, f=0).items():
        assert ffn(lib, **{n: v}) == INVALID, n
    for n in ("xq", "x_scale", "off", "wgq", "g_scale", "wuq", "u_scale", "wdq", "d_scale", "y"):
        assert ffn(lib, **{n: None}) == INVALID, n
    for n in ("xq", "wgq", "wuq", "wdq"):
        assert ffn(lib, **{n: ODD}) == INVALID, n
    assert ffn(lib, B=1 << 26) == INVALID
    assert ffn(lib, ws=None) == WORKSPACE and ffn(lib, ws=ODD) == WORKSPACE
    need = lib.xmoe_workspace_bytes(17, 32, 64, 4, 1, 32, 1)
    assert need >= 32 * 128 * 3 and need % 256 == 0 and ffn(lib, ws_bytes=need - 1) == WORKSPACE
    assert ffn(lib, B=0, xq=None, y=None, ws=None) == OK


def test_quantising_weights(lib):  # noqa: F811
    def call(w=P, E=2, K=64, N=32, dt=1, wq=P, scale=P):
        return lib.xmoe_quantize_weights(w, E, K, N, dt, wq, scale, None)
    assert call(dt=9) == UNSUPPORTED and call(K=65537) == UNSUPPORTED and call(E=65536) == UNSUPPORTED
    assert call(E=0) == INVALID and call(K=0) == INVALID and call(N=0) == INVALID
    assert call(w=None) == INVALID and call(wq=None) == INVALID and call(scale=None) == INVALID and call(wq=ODD) == INVALID
