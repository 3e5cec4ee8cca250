"""The largest sizes of xmoe_quantize_weights: refused on the host, before anything is enqueued (no GPU)."""
import ctypes

from test_norm_host import lib  # noqa: F401  (the library, built if it is not there)

INVALID, UNSUPPORTED = 1, 2
P = ctypes.c_void_p(4096)      # never dereferenced on the host


def test_columns(lib):  # noqa: F811
    def call(N, w=P):
        return lib.xmoe_quantize_weights(w, 1, 1, N, 1, P, P, None)
    for n in ((1 << 30) - 63, 1 << 30, (1 << 31) - 1):
        assert call(n) == UNSUPPORTED, n
    assert call((1 << 30) - 64, w=None) == INVALID      # a size that is taken: the pointer is what is refused
