"""Pins of the 8-bit and clipping oracle (CPU): the formats against torch's 8-bit
casts, the block scales against their defining inequality, the RMS norm and its
gradient against torch autograd and central differences, clipping against
torch.nn.utils.clip_grad_norm_."""
import numpy as np
import pytest
import torch

from oracle import linear8 as o8

T8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_values_and_rounding_of_the_formats(fmt):
    table = o8.table8(fmt)
    want = torch.arange(256, dtype=torch.uint8).view(T8[fmt]).double().numpy()
    assert np.array_equal(table, want, equal_nan=True)
    rs = np.random.default_rng(1)
    v = np.concatenate([rs.standard_normal(20000) * 10.0 ** rs.uniform(-6, 2, 20000), table[np.isfinite(table)]])
    mid = np.sort(table[np.isfinite(table)])
    v = np.concatenate([v, (mid[1:] + mid[:-1]) / 2])  # every tie
    v = v[np.abs(v) <= o8.MOST[fmt]].astype(np.float32)
    assert np.array_equal(o8.round8(v, fmt), torch.from_numpy(v).to(T8[fmt]).double().numpy())


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_block_scales_are_the_least_that_hold_the_block(fmt):
    rs = np.random.default_rng(2)
    a = np.concatenate([rs.uniform(0.1, 1, 500) * 2.0 ** rs.integers(-120, 120, 500),
                        o8.MOST[fmt] * 2.0 ** np.arange(-20, 20), np.nextafter(o8.MOST[fmt], 1e9) * 2.0 ** np.arange(-20, 20)])
    s = o8.scale_bytes(a, fmt)
    assert (a <= o8.MOST[fmt] * 2.0 ** (s - 127)).all() and (a > o8.MOST[fmt] * 2.0 ** (s - 128))[s > 0].all()
    assert list(o8.scale_bytes(np.array([0.0, np.inf, np.nan, 2.0 ** -149]), fmt)) == [0, 255, 255, 0]


def test_norm_and_its_gradient():
    rs = np.random.default_rng(3)
    h, g, dy, eps = rs.standard_normal((5, 37)), rs.standard_normal(37), rs.standard_normal((5, 37)), 1e-3
    rstd, y = o8.rmsnorm(h, g, eps)
    th, tg = torch.from_numpy(h).requires_grad_(), torch.from_numpy(g).requires_grad_()
    ty = torch.nn.functional.rms_norm(th, (37,), tg, eps)
    ty.backward(torch.from_numpy(dy))
    assert np.abs(ty.detach().numpy() - y).max() < 1e-13
    dh, dg = o8.rmsnorm_grad(dy, h, g, eps)
    assert np.abs(th.grad.numpy() - dh).max() < 1e-13 and np.abs(tg.grad.numpy() - dg).max() < 1e-13
    # central differences of <y, dy>: step 1e-5, third derivatives of order 10
    for _ in range(4):
        u, w, d = rs.standard_normal(h.shape), rs.standard_normal(37), 1e-5
        f = [(o8.rmsnorm(h + k * d * u, g + k * d * w, eps)[1] * dy).sum() for k in (1, -1)]
        assert abs((f[0] - f[1]) / (2 * d) - (dh * u).sum() - (dg * w).sum()) < 1e-7


@pytest.mark.parametrize("ord", [2, float("inf")])
def test_clipping_against_torch(ord):
    rs = np.random.default_rng(4)
    ts = [rs.standard_normal(n) for n in (1, 7, 300)]
    params = [torch.nn.Parameter(torch.zeros(t.size, dtype=torch.float64)) for t in ts]
    for p, t in zip(params, ts):
        p.grad = torch.from_numpy(t.copy())
    norm = torch.nn.utils.clip_grad_norm_(params, 0.75, norm_type=ord)
    got = o8.grad_norm(ts, ord)
    assert abs(got - float(norm)) < 1e-12
    c = o8.clip_factor(got, 0.75)
    # torch divides by norm + 1e-6
    assert max(np.abs(p.grad.numpy() - t * c).max() for p, t in zip(params, ts)) < 1e-5
    assert o8.clip_factor(0.5, 0.75) == o8.clip_factor(np.inf, 0.75) == o8.clip_factor(np.nan, 0.75) == 1.0
