"""Refusals of the norm's entry points: each on the host, before anything is enqueued (no GPU)."""
import ctypes

import pytest

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
P = ctypes.c_void_p(4096)      # never dereferenced on the host


@pytest.fixture(scope="module")
def lib():
    import os

    from paper_2508_13337_amd import _lib
    if not os.path.exists(_lib.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return _lib.lib()


def fwd(lib, x=P, residual=None, gain=P, T=4, d=64, eps=1e-6, dt=1, h=None, y=P, q=None, q_scale=None, rstd=None):
    return lib.xmoe_add_rmsnorm(x, residual, gain, T, d, eps, dt, h, y, q, q_scale, rstd, None)


def bwd(lib, dy=P, dh=None, h=P, gain=P, rstd=P, T=4, d=64, dt=1, dx=P, dgain=P, ws=P, ws_bytes=1 << 20):
    return lib.xmoe_add_rmsnorm_bwd(dy, dh, h, gain, rstd, T, d, dt, dx, dgain, ws, ws_bytes, None)


def test_forward_refusals(lib):
    assert fwd(lib, dt=2) == UNSUPPORTED and fwd(lib, d=16385) == UNSUPPORTED
    assert fwd(lib, d=0) == INVALID and fwd(lib, T=-1) == INVALID
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        assert fwd(lib, eps=eps) == INVALID
    assert fwd(lib, x=None) == INVALID and fwd(lib, gain=None) == INVALID
    assert fwd(lib, y=None) == INVALID                                   # nothing asked for
    assert fwd(lib, q=P) == INVALID and fwd(lib, q_scale=P) == INVALID   # integers without scales, scales without integers
    assert fwd(lib, residual=P) == INVALID                               # a sum with nowhere to go
    assert fwd(lib, q=ctypes.c_void_p(4100), q_scale=P) == INVALID       # 8-bit rows start at 16 bytes
    assert fwd(lib, T=0) == OK


def test_backward_refusals(lib):
    assert bwd(lib, dt=7) == UNSUPPORTED and bwd(lib, d=1 << 20) == UNSUPPORTED and bwd(lib, d=0) == INVALID
    for n in ("dy", "h", "gain", "rstd", "dx", "dgain"):
        assert bwd(lib, **{n: None}) == INVALID, n
    assert bwd(lib, ws=None) == WORKSPACE and bwd(lib, ws=ctypes.c_void_p(4100)) == WORKSPACE
    need = lib.xmoe_workspace_bytes(16, 4, 64, 0, 0, 0, 1)
    assert need >= 4 * 64 * 4 and need % 256 == 0 and bwd(lib, ws_bytes=need - 1) == WORKSPACE
    # one partial row for each of a bounded number of blocks
    for d in (64, 2048):
        assert lib.xmoe_workspace_bytes(16, 1 << 20, d, 0, 0, 0, 1) == lib.xmoe_workspace_bytes(16, 1024, d, 0, 0, 0, 0)


def test_pitch(lib):
    assert [lib.xmoe_q8_pitch(n) for n in (1, 127, 128, 129, 1408, 16384)] == [128, 128, 128, 256, 1408, 16384]
