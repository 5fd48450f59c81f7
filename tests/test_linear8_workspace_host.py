"""What the norm and clipping calls ask of the workspace (no GPU needed)."""
import ctypes

import paper_2607_17572_amd as pk
from paper_2607_17572_amd import api
from test_capi_host import _lib_or_skip

P = 1 << 20  # a fake, aligned device address: never dereferenced


def test_clipping_needs_a_few_kilobytes_whatever_the_model():
    L = _lib_or_skip()
    n = ctypes.c_size_t()
    assert L.jagg_grad_norm_bytes(None) == 1
    assert L.jagg_grad_norm_bytes(ctypes.byref(n)) == 0 and 0 < n.value <= 1 << 16
    for name in ("tiny", "block"):
        h = ctypes.c_void_p()
        c = pk.config(name).c()
        assert L.jagg_ctx_create(ctypes.byref(c), None, ctypes.byref(h)) == 0
        try:
            g = (api._Grad * 1)(api._Grad(P, 8, 0))
            for bound in (None, n.value - 1):
                assert L.jagg_ctx_set_workspace(h, None if bound is None else P, bound or 0) == 0
                assert L.jagg_grad_norm(h, g, 1, 0, P) == 1 and b"jagg_grad_norm_bytes" in L.jagg_last_error()
                assert L.jagg_grad_clip(h, g, None, 1, 0, 1.0, P) == 1 and b"jagg_grad_norm_bytes" in L.jagg_last_error()
        finally:
            L.jagg_ctx_destroy(h)
