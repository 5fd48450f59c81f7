"""Gradient clipping by factors at the end of fp32's range and past it."""
import numpy as np
import pytest
import torch

import paper_2607_17572_amd as pk
from oracle import linear8 as o8

pytestmark = pytest.mark.gpu

BF, FP, DB = torch.bfloat16, torch.float32, torch.float64


@pytest.fixture(autouse=True)
def fp32_default():
    """Another test file sets fp64 as the default type."""
    was = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(was)


@pytest.mark.parametrize("large,max_norm", [(1e30, 1e-20), (1e38, 1e-3), (1e30, 2.0 ** -27), (1e20, 1e-18), (1e36, 1e-44), (2.0, 0.0)])
@pytest.mark.parametrize("src", [BF, FP])
@pytest.mark.parametrize("sizes", [[5, 3000], [40000, 17]])
def test_small_factors(large, max_norm, src, sizes):
    """The factor is rounded to fp32 where that holds it (2^-24) and not below 2^-126, the
    product to fp32 (2^-24, or half of 2^-149), that to bf16 (2^-8, or half of 2^-133); no
    element is lost while the factor is not 0."""
    print(f"case: clip {large} {max_norm} {src} {sizes}", flush=True)
    ctx = pk.Context(pk.config("tiny"))
    g = torch.Generator().manual_seed(1)
    ts = [(torch.rand(n, generator=g) * large).to(src).cuda() for n in sizes]
    want = [t.double().cpu().numpy() for t in ts]
    norm = o8.grad_norm(want)
    c = o8.clip_factor(norm, max_norm)
    assert c < 1
    out = torch.empty(2, dtype=DB, device="cuda")
    for dt in (FP, BF):
        dst = [torch.full(t.shape, 3.0, dtype=dt, device="cuda") for t in ts]
        ctx.clip_grads(ts, max_norm, out, dst=dst)
        assert abs(float(out[1]) - c) <= 1e-12 * c
        for d, w in zip(dst, want):
            tol = (2 * 2.0 ** -24 + (2.0 ** -8 if dt is BF else 0)) * w * c + 2.0 ** -150 + (2.0 ** -134 if dt is BF else 0)
            assert (np.abs(d.double().cpu().numpy() - w * c) <= tol * (1 + 1e-6)).all()
    keep = [t.clone() for t in ts]
    ctx.clip_grads(ts, max_norm, out)  # in place: the same values
    same = [torch.empty_like(t) for t in ts]
    ctx.clip_grads(keep, max_norm, out, dst=same)
    assert all(torch.equal(a, b) for a, b in zip(ts, same))
