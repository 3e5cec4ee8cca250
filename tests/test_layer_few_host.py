"""Refusals of xmoe_layer_few_fwd: each on the host, before anything is enqueued (no GPU)."""
import ctypes

from test_norm_host import lib  # noqa: F401  (the library, built if it is not there)

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3
P, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(4104)      # never dereferenced on the host
ARGS = dict(x=P, w_router=P, bias=None, wg=P, wu=P, wd=P, addend=None, T=4, d=64, E=8, E_s=1, k=2, f=32, dt=1, logits=P,
            topk_idx=P, topk_w=P, out=P, ws=P, ws_bytes=1 << 24)


def test_refusals(lib):  # noqa: F811
    def call(**kw):
        return lib.xmoe_layer_few_fwd(*{**ARGS, **kw}.values(), None)
    assert call(dt=5) == UNSUPPORTED and call(T=33) == UNSUPPORTED and call(E=513) == UNSUPPORTED
    assert call(E=512, E_s=1) == UNSUPPORTED and call(E=100, k=65) == UNSUPPORTED
    assert call(d=65537) == UNSUPPORTED and call(f=65537) == UNSUPPORTED
    for n, v in dict(T=-1, d=0, E=0, E_s=-1, k=0, f=0).items():
        assert call(**{n: v}) == INVALID, n
    assert call(k=9) == INVALID
    for n in ("x", "w_router", "wg", "wu", "wd", "logits", "topk_idx", "topk_w", "out"):
        assert call(**{n: None}) == INVALID, n
    assert call(ws=None) == WORKSPACE and call(ws=ODD) == WORKSPACE
    need = lib.xmoe_workspace_bytes(18, 4, 64, 9, 3, 32, 1)
    assert need >= 4 * 3 * (32 * 2 + 64 * 4) and need % 256 == 0 and call(ws_bytes=need - 1) == WORKSPACE
    assert call(T=0, x=None, out=None, logits=None, topk_idx=None, topk_w=None, ws=None) == OK
