"""The workspace that the 8-bit and clipping calls bind: as large as they need, within its
bounds, and no longer than a captured graph may need it."""
import ctypes

import pytest
import torch

import paper_2607_17572_amd as pk

pytestmark = pytest.mark.gpu

DB = torch.float64


@pytest.fixture(autouse=True)
def fp32_default():
    """Another test file sets fp64 as the default type."""
    was = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(was)


def test_clipping_binds_no_models_workspace():
    """A context of a large model: the norm and the clip take kilobytes, and stay in them."""
    ctx = pk.Context(pk.config("block"))
    t, out = torch.ones(300000, device="cuda"), torch.empty(2, dtype=DB, device="cuda")
    was = torch.cuda.memory_allocated()
    ctx.grad_norm([t], out[:1])
    assert float(out[0]) == 300000 ** 0.5
    ctx.clip_grads([t], 1.0, out, ord=float("inf"))
    assert out.tolist() == [1.0, 1.0]
    assert torch.cuda.memory_allocated() - was < 1 << 20
    n = ctypes.c_size_t()
    assert pk.lib().jagg_grad_norm_bytes(ctypes.byref(n)) == 0
    full = torch.full((n.value + 8192,), 0xA5, dtype=torch.uint8, device="cuda")
    assert full.data_ptr() % 256 == 0
    assert pk.lib().jagg_ctx_set_workspace(ctx._h, full.data_ptr() + 4096, n.value) == 0
    big = torch.ones(5000000, device="cuda")  # more chunks than partial results
    for o in (2, float("inf")):
        ctx.clip_grads([big, t], 1.0, out, dst=[torch.empty_like(big), torch.empty_like(t)], ord=o)
        assert float(out[0]) == (5300000 ** 0.5 if o == 2 else 1.0)
    assert bool((full[:4096] == 0xA5).all()) and bool((full[-4096:] == 0xA5).all())


def test_only_a_captured_workspace_outlives_its_successor():
    """A graph's workspace stays when a larger one is bound; those before and after it,
    which no graph holds, are freed."""
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx = pk.Context(pk.config("tiny"), stream=s)
        t, out = torch.full((1000,), 2.0, device="cuda"), torch.empty(2, dtype=DB, device="cuda")
        dst = torch.empty_like(t)
        ctx._ensure_bytes(1 << 16)
        ctx._ensure_bytes(1 << 20)
        ctx.clip_grads([t], 1.0, out, dst=[dst])
        s.synchronize()
        want = dst.clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            ctx.clip_grads([t], 1.0, out, dst=[dst])
        held = ctx._ws
        was = torch.cuda.memory_allocated()
        for mb in (64, 128, 256):
            ctx._ensure_bytes(mb << 20)
            ctx.clip_grads([t], 1.0, out, dst=[dst])  # eager use in between
        assert ctx._ws_of_graphs == [held]
        assert torch.cuda.memory_allocated() - was <= (256 << 20) + (1 << 21)
        for _ in range(3):
            dst.zero_()
            g.replay()
            s.synchronize()
            assert torch.equal(dst, want)
        with torch.cuda.graph(torch.cuda.CUDAGraph(), stream=s):
            ctx.clip_grads([t], 1.0, out, dst=[dst])
        ctx._ensure_bytes(300 << 20)
        assert len(ctx._ws_of_graphs) == 2
