"""Host-side checks of the 8-bit and clipping calls (no GPU needed): every argument
error is found before a launch, in the C ABI and in the binding."""
import ctypes

import pytest
import torch

import paper_2607_17572_amd as pk
from paper_2607_17572_amd import api
from test_capi_host import _lib_or_skip

P = 1 << 20  # a fake, aligned device address: never dereferenced
NAN, INF = float("nan"), float("inf")


@pytest.fixture(autouse=True)
def fp32_default():
    """Another test file sets fp64 as the default type."""
    was = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(was)


@pytest.fixture()
def ctx():
    L = _lib_or_skip()
    h = ctypes.c_void_p()
    c = pk.config("tiny").c()
    assert L.jagg_ctx_create(ctypes.byref(c), None, ctypes.byref(h)) == 0
    yield L, h
    L.jagg_ctx_destroy(h)


def m8(n_rows, n_k, **kw):
    d = dict(q=P, scale=P, ld=-(-n_k // 128) * 128, rows=n_rows, k=n_k, fmt=0)
    d.update(kw)
    return ctypes.byref(api._Mat8(*[d[n] for n in ("q", "scale", "ld", "rows", "k", "fmt")]))


def test_sizes_of_an_8bit_matrix():
    L = _lib_or_skip()
    n = [ctypes.c_size_t() for _ in range(3)]
    r = [ctypes.byref(x) for x in n]
    for rows, k, want in ((1, 1, (128, 128, 4)), (3, 128, (128, 384, 12)), (5, 513, (640, 3200, 40))):
        assert L.jagg_mat8_bytes(rows, k, *r) == 0
        assert tuple(x.value for x in n) == want
    assert L.jagg_mat8_bytes(0, 1, *r) == 1 and L.jagg_mat8_bytes(1, 0, *r) == 1 and L.jagg_mat8_bytes(1, 1, None, *r[1:]) == 1


BAD_MAT = [dict(q=None), dict(scale=None), dict(q=P + 8), dict(scale=P + 2), dict(fmt=2), dict(ld=100), dict(ld=192),
           dict(ld=128), dict(ld=(1 << 22) + 128)]


@pytest.mark.parametrize("bad", BAD_MAT + [dict(rows=0), dict(k=0), dict(rows=9), dict(k=200)])
def test_quantize8_refuses_a_bad_matrix(ctx, bad):
    L, h = ctx
    for a in ((m8(8, 256, **bad), None), (None, m8(8, 256, **bad))):
        rows, cols = (8, 256) if a[0] is not None else (256, 8)
        assert L.jagg_quantize8(h, P, 256, rows, cols, 1, None, None, 0, *a) == 1


@pytest.mark.parametrize("bad", [dict(x=None), dict(x=P + 1), dict(ldx=255), dict(rows=0), dict(cols=0), dict(dt=2),
                                 dict(rm=P + 2), dict(cm=P + 1), dict(tile=2), dict(out=None, out_t=None),
                                 dict(out_t=m8(256, 8, fmt=1)), dict(out_t=m8(8, 256))])
def test_quantize8_refuses_bad_arguments(ctx, bad):
    L, h = ctx
    d = dict(x=P, ldx=256, rows=8, cols=256, dt=1, rm=None, cm=None, tile=0, out=m8(8, 256), out_t=None)
    d.update(bad)
    assert L.jagg_quantize8(h, *d.values()) == 1
    assert L.jagg_quantize8(None, *d.values()) == 1


@pytest.mark.parametrize("bad,rc", [(b, 1) for b in BAD_MAT if "fmt" not in b] + [
    (dict(k=255), 1), (dict(rows=0), 1)])
def test_matmul8_refuses_a_bad_operand(ctx, bad, rc):
    L, h = ctx
    assert L.jagg_matmul8(h, m8(8, 256, **bad), m8(16, 256), None, P, 16, 0, 0.0) == rc
    assert L.jagg_matmul8(h, m8(8, 256), m8(16, 256, **bad), None, P, 16, 0, 0.0) == rc


def test_matmul8_refuses_bad_arguments(ctx):
    L, h = ctx
    a, b = m8(8, 256), m8(16, 256)
    assert L.jagg_matmul8(None, a, b, None, P, 16, 0, 0.0) == 1
    assert L.jagg_matmul8(h, None, b, None, P, 16, 0, 0.0) == 1
    assert L.jagg_matmul8(h, a, None, None, P, 16, 0, 0.0) == 1
    assert L.jagg_matmul8(h, a, b, None, None, 16, 0, 0.0) == 1
    assert L.jagg_matmul8(h, a, b, None, P + 2, 16, 0, 0.0) == 1       # fp32 result at an odd address
    assert L.jagg_matmul8(h, a, b, P + 1, P, 16, 1, 0.0) == 1          # bias
    assert L.jagg_matmul8(h, a, b, None, P, 15, 0, 0.0) == 1           # row stride
    assert L.jagg_matmul8(h, a, b, None, P, 16, 2, 0.0) == 1           # dtype
    assert L.jagg_matmul8(h, a, b, None, P, 16, 0, 0.5) == 1           # beta
    assert L.jagg_matmul8(h, a, b, None, P, 16, 0, NAN) == 1
    assert L.jagg_matmul8(h, a, m8(16, 256, fmt=1), None, P, 16, 0, 0.0) == 4  # right operand E5M2
    assert b"E4M3" in L.jagg_last_error()


def test_matmul8_workspace(ctx):
    """A long contraction over a small result needs one, few rows and large results none."""
    L, h = ctx
    n = ctypes.c_size_t()

    def need(*a):
        assert L.jagg_matmul8_bytes(*a, ctypes.byref(n)) == 0
        return n.value

    assert need(37, 4096, 12288, 1) >= 2 * 37 * 4096 * 4 and need(512, 512, 9216, 0) >= 2 * 512 * 512 * 4
    assert need(1, 4096, 12288, 1) == need(16, 4096, 12288, 0) == need(9216, 16384, 4096, 1) == need(100, 100, 100, 1) == 0
    bytes_ = need(37, 4096, 12288, 1)
    args = (m8(37, 12288), m8(4096, 12288), None, P, 4096, 1, 0.0)
    assert L.jagg_matmul8(h, *args) == 1 and b"jagg_matmul8_bytes" in L.jagg_last_error()
    assert L.jagg_ctx_set_workspace(h, P, bytes_ - 1) == 0
    assert L.jagg_matmul8(h, *args) == 1 and b"jagg_matmul8_bytes" in L.jagg_last_error()
    assert L.jagg_matmul8_bytes(0, 1, 1, 0, ctypes.byref(n)) == 1 and L.jagg_matmul8_bytes(1, 1, 1, 2, ctypes.byref(n)) == 1
    assert L.jagg_matmul8_bytes(1, 1, 1, 0, None) == 1


NORM = dict(x=P, ldx=256, r=None, ldr=0, gain=P, rows=8, cols=256, dt=1, eps=1e-6, h=None, ldh=0, y=m8(8, 256), rstd=P)


@pytest.mark.parametrize("bad,rc", [
    (dict(x=None), 1), (dict(gain=None), 1), (dict(y=None), 1), (dict(rows=0), 1), (dict(cols=0), 1), (dict(dt=3), 1),
    (dict(ldx=255), 1), (dict(r=P, ldr=255), 1), (dict(h=P, ldh=0), 1), (dict(eps=-1.0), 1), (dict(eps=NAN), 1),
    (dict(eps=INF), 1), (dict(x=P + 1), 1), (dict(gain=P + 1), 1), (dict(r=P + 1, ldr=256), 1), (dict(h=P + 1, ldh=256), 1),
    (dict(rstd=P + 2), 1), (dict(y=m8(8, 255)), 1), (dict(y=m8(9, 256)), 1), (dict(y=m8(8, 256, fmt=1)), 4),
    (dict(cols=32769, ldx=32769, y=m8(8, 32769)), 4)])
def test_rmsnorm8_refuses_bad_arguments(ctx, bad, rc):
    L, h = ctx
    assert L.jagg_rmsnorm8(h, *{**NORM, **bad}.values()) == rc
    assert L.jagg_rmsnorm8(None, *{**NORM, **bad}.values()) == 1


GRAD = dict(dy=P, lddy=256, h=P, ldh=256, rstd=P, gain=P, dh=None, lddh=0, rows=8, cols=256, dt=1, dx=P, lddx=256,
            dgain=P, gdt=0, beta=0.0)


@pytest.mark.parametrize("bad,rc", [
    (dict(dy=None), 1), (dict(h=None), 1), (dict(rstd=None), 1), (dict(gain=None), 1), (dict(dx=None), 1),
    (dict(dgain=None), 1), (dict(rows=0), 1), (dict(cols=0), 1), (dict(dt=3), 1), (dict(gdt=3), 1), (dict(beta=2.0), 1),
    (dict(lddy=255), 1), (dict(ldh=255), 1), (dict(lddx=255), 1), (dict(dh=P, lddh=255), 1), (dict(dy=P + 1), 1),
    (dict(dx=P + 1), 1), (dict(dgain=P + 2), 1), (dict(rstd=P + 1), 1),
    (dict(cols=32769, lddy=32769, ldh=32769, lddx=32769), 4)])
def test_rmsnorm8_grad_refuses_bad_arguments(ctx, bad, rc):
    L, h = ctx
    assert L.jagg_rmsnorm8_grad(h, *{**GRAD, **bad}.values()) == rc
    assert b"workspace" not in L.jagg_last_error()


def test_rmsnorm8_grad_needs_its_workspace(ctx):
    L, h = ctx
    n = ctypes.c_size_t()
    assert L.jagg_rmsnorm8_grad(h, *GRAD.values()) == 1 and b"workspace" in L.jagg_last_error()
    assert L.jagg_rmsnorm8_grad_bytes(8, 256, ctypes.byref(n)) == 0 and n.value >= 256 * 4
    assert L.jagg_ctx_set_workspace(h, P, n.value - 1) == 0
    assert L.jagg_rmsnorm8_grad(h, *GRAD.values()) == 1 and b"workspace" in L.jagg_last_error()
    assert L.jagg_rmsnorm8_grad_bytes(0, 256, ctypes.byref(n)) == 1 and L.jagg_rmsnorm8_grad_bytes(8, 256, None) == 1


def gl(*entries):
    return (api._Grad * len(entries))(*[api._Grad(*e) for e in entries])


def test_gradient_lists_are_checked(ctx):
    L, h = ctx
    ok = gl((P, 8, 0), (P + 64, 8, 1))
    for bad in (gl((None, 8, 0)), gl((P + 2, 8, 0)), gl((P + 1, 8, 1)), gl((P, 8, 2))):
        assert L.jagg_grad_norm(h, bad, 1, 0, P) == 1
        assert L.jagg_grad_clip(h, bad, None, 1, 0, 1.0, P) == 1
        assert L.jagg_grad_clip(h, gl((P, 8, 0)), bad, 1, 0, 1.0, P) == 1
        assert b"workspace" not in L.jagg_last_error()
    for call in (lambda *a: L.jagg_grad_norm(*a), lambda h, g, n, o, out: L.jagg_grad_clip(h, g, None, n, o, 1.0, out)):
        assert call(None, ok, 2, 0, P) == 1 and call(h, None, 2, 0, P) == 1 and call(h, ok, 2, 0, None) == 1
        assert call(h, ok, 0, 0, P) == 1 and call(h, ok, 2, 2, P) == 1 and call(h, ok, 2, 0, P + 4) == 1
        assert b"workspace" not in L.jagg_last_error()
        assert call(h, ok, 2, 0, P) == 1 and b"workspace" in L.jagg_last_error()
        assert call(h, gl((None, 0, 0)), 1, 0, P) == 1 and b"workspace" in L.jagg_last_error()  # an empty tensor is fine
    assert L.jagg_grad_clip(h, ok, gl((P, 8, 0), (P, 9, 1)), 2, 0, 1.0, P) == 1   # another size
    assert L.jagg_grad_clip(h, ok, gl((P, 8, 1), (P, 8, 1)), 2, 0, 1.0, P) == 1   # in place with another dtype
    for m in (-1.0, NAN, INF):
        assert L.jagg_grad_clip(h, ok, None, 2, 0, m, P) == 1 and b"max_norm" in L.jagg_last_error()


def test_the_binding_checks_shapes_strides_and_types():
    cpu = torch.device("cpu")
    x = torch.zeros(4, 6)
    p = x.data_ptr()
    assert api._rows(x, "x", 4, 6, torch.float32, cpu) == (p, 6)
    assert api._rows(x[:, :5], "x", 4, 5, torch.float32, cpu) == (p, 6)
    assert api._rows(x[:1, 2:], "x", 1, 4, torch.float32, cpu) == (p + 8, 4)
    assert api._vec(x[0], "v", 6, torch.float32, cpu) == p
    assert api._vec(x[0, :1], "v", 1, torch.float32, cpu) == p
    for bad in (lambda: api._rows(x.t(), "x", 6, 4, torch.float32, cpu), lambda: api._rows(x, "x", 4, 5, torch.float32, cpu),
                lambda: api._rows(x, "x", 4, 6, torch.bfloat16, cpu), lambda: api._rows(x[0], "x", 1, 6, torch.float32, cpu),
                lambda: api._rows(x[:1].expand(4, 6), "x", 4, 6, torch.float32, cpu),
                lambda: api._rows(x, "x", 4, 6, torch.float32, torch.device("cuda", 0)),
                lambda: api._vec(x[:, 0], "v", 4, torch.float32, cpu), lambda: api._vec(x, "v", 24, torch.float32, cpu),
                lambda: api._dtype_of(x.double(), "x"), lambda: pk.GradList([x]), lambda: pk.GradList([])):
        with pytest.raises(pk.JaggError) as e:
            bad()
        assert e.value.status == 1
