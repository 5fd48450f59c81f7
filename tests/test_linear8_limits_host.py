"""Sizes that no launch can take (2^32 threads and more) are refused on the host, without a
launch (no GPU needed)."""
import ctypes

import pytest

import paper_2607_17572_amd as pk
from paper_2607_17572_amd import api
from test_capi_host import _lib_or_skip

P = 1 << 20  # a fake, aligned device address: never dereferenced
UNSUPPORTED = 4
MOST = 2 ** 31 - 1


@pytest.fixture()
def ctx():
    L = _lib_or_skip()
    h = ctypes.c_void_p()
    c = pk.config("tiny").c()
    assert L.jagg_ctx_create(ctypes.byref(c), None, ctypes.byref(h)) == 0
    yield L, h
    L.jagg_ctx_destroy(h)


def m8(rows, k):
    return ctypes.byref(api._Mat8(P, P, -(-k // 128) * 128, rows, k, 0))


@pytest.mark.parametrize("rows,cols", [(2 ** 26, 128), (MOST, 1), (MOST - 2, 2048), (2 ** 24, 2049), (2 ** 24, 8192), (2 ** 22, 8193),
                                       (MOST, 32768)])
@pytest.mark.parametrize("dt", [0, 1])
def test_norm(ctx, rows, cols, dt):
    L, h = ctx
    assert L.jagg_rmsnorm8(h, P, cols, None, 0, P, rows, cols, dt, 1e-6, None, 0, m8(rows, cols), P) == UNSUPPORTED
    assert b"rows" in L.jagg_last_error()


@pytest.mark.parametrize("rows,cols", [(2 ** 31 - 127, 1), (MOST, 1), (2 ** 30, 129), (4096 * 128, 4096 * 128)])
def test_quantiser(ctx, rows, cols):
    L, h = ctx
    for tile in (0, 1):
        assert L.jagg_quantize8(h, P, cols, rows, cols, 0, None, None, tile, m8(rows, cols), None) == UNSUPPORTED


@pytest.mark.parametrize("m,n,k", [(1, 2 ** 27, 128), (16, MOST, 1), (2 ** 31 - 200, 1, 1), (MOST, 64, 128), (17, MOST, 128),
                                   (2 ** 30, 2 ** 20, 128), (MOST, MOST, 4096)])
@pytest.mark.parametrize("dt", [0, 1])
def test_product(ctx, m, n, k, dt):
    L, h = ctx
    assert L.jagg_matmul8(h, m8(m, k), m8(n, k), None, P, n, dt, 0.0) == UNSUPPORTED
