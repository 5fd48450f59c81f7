"""Matrices and gradient lists whose memory moved are refused, and one whose tensors were
given other memory works on the memory that it keeps: nothing is read from or written
to memory that may be another's by now."""
import pytest
import torch

import paper_2607_17572_amd as pk

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


@pytest.fixture(autouse=True)
def fp32_default():
    """Another test file sets fp64 as the default type."""
    was = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(was)


@pytest.fixture(scope="module")
def ctx():
    return pk.Context(pk.config("tiny"))


def set_(t):
    t.set_(torch.zeros_like(t))


def data(t):
    t.data = torch.zeros_like(t)


def resize(t):
    t.resize_(4 * t.numel())


def storage(t):
    t.untyped_storage().resize_(8 * t.untyped_storage().nbytes())


@pytest.mark.parametrize("move", [set_, data])
def test_a_gradient_list_keeps_its_memory(ctx, move):
    n = 1 << 20
    t = torch.full((n,), 3.0, device="cuda")
    src, at = pk.GradList([t]), t.data_ptr()
    out = torch.empty(2, dtype=torch.float64, device="cuda")
    move(t)
    junk = [torch.full((n,), 5.0, device="cuda") for _ in range(8)]  # would take what was freed
    assert at not in [j.data_ptr() for j in junk]
    ctx.clip_grads(src, 1.0, out)
    assert float(out[0]) == 3.0 * n ** 0.5
    assert all(bool((j == 5).all()) for j in junk) and not bool(t.any())


@pytest.mark.parametrize("move", [resize, storage])
def test_a_gradient_list(ctx, move):
    ts = [torch.full((n,), 3.0, device="cuda") for n in (700, 5, 3000)]
    keep = [t.view(-1) for t in ts]  # the old memory stays the test's
    out = torch.empty(2, dtype=torch.float64, device="cuda")
    src, dst = pk.GradList(ts), pk.GradList([torch.zeros_like(t) for t in ts])
    ctx.clip_grads(src, 1.0, out, dst=dst)
    move(ts[1])
    for call in (lambda: ctx.clip_grads(src, 1.0, out), lambda: ctx.clip_grads(src, 1.0, out, dst=dst),
                 lambda: ctx.clip_grads(dst, 1.0, out, dst=src), lambda: ctx.grad_norm(src, out[:1])):
        with pytest.raises(pk.JaggError):
            call()
    assert all(bool((k == 3).all()) for k in (keep[0], keep[2]))
    ctx.clip_grads([ts[0], ts[2]], 1.0, out)  # a new list takes them as they are


@pytest.mark.parametrize("which", ["q", "scale"])
@pytest.mark.parametrize("how", ["storage", "replaced"])
def test_a_matrix(ctx, which, how):
    x = torch.randn(8, 256, device="cuda")
    g, out = torch.ones(256, device="cuda"), torch.empty(8, 8, device="cuda")
    a, b = pk.Mat8(8, 256), pk.Mat8(8, 256)
    ctx.quantize8(x, a)
    ctx.quantize8(x, b)
    ctx.matmul8(a, b, out)
    if how == "storage":
        storage(getattr(a, which))
    else:
        setattr(a, which, getattr(a, which).clone())
    for call in (lambda: ctx.quantize8(x, a), lambda: ctx.quantize8(x.t().contiguous(), out_t=a), lambda: ctx.matmul8(a, b, out),
                 lambda: ctx.matmul8(b, a, out), lambda: ctx.rmsnorm8(x, g, a)):
        with pytest.raises(pk.JaggError):
            call()
    ctx.matmul8(b, b, out)
