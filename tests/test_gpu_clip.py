"""Global gradient norm and clipping on the GPU against the fp64 oracle: lists of one to
hundreds of tensors, either dtype, odd sizes and addresses, in place and into a copy,
norms that are not finite, graphs."""
import numpy as np
import pytest
import torch

import paper_2607_17572_amd as pk
from oracle import linear8 as o8

pytestmark = pytest.mark.gpu

BF, FP, DB = torch.bfloat16, torch.float32, torch.float64
INF = float("inf")


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


def say(*a):
    print(*a, flush=True)


def grads(seed, sizes, dts, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(scale * torch.randn(n, generator=g)).to(dts[i % len(dts)]).cuda() for i, n in enumerate(sizes)]


def f64(t):
    return t.double().cpu().numpy()


LISTS = {
    "one": [1], "small": [5, 8, 0, 13], "chunks": [8191, 8192, 8193, 40000], "empty first": [0, 3],
    "many": [(7 * i) % 900 for i in range(300)], "one long": [3000001], "rising": [2 ** i for i in range(21)],
}


@pytest.mark.parametrize("name", LISTS)
@pytest.mark.parametrize("dts", [[BF], [FP], [BF, FP]], ids=["bf16", "fp32", "both"])
@pytest.mark.parametrize("ord", [2, INF])
def test_norm_and_clip(ctx, name, dts, ord):
    """The norm is a sum of squares in fp64 (relative error far below 1e-12); the factor
    is rounded to fp32, the product once more, and once to the copy's type."""
    say(f"case: clip {name} {dts} {ord}")
    ts = grads(1, LISTS[name], dts)
    want = [f64(t) for t in ts]
    norm = o8.grad_norm(want, ord)
    out = torch.empty(2, dtype=DB, device="cuda")
    ctx.grad_norm(ts, out[:1], ord=ord)
    assert abs(float(out[0]) - norm) <= 1e-12 * norm
    for max_norm in (0.37 * norm, norm * 2, 0.0):
        c = o8.clip_factor(norm, max_norm)
        for dst_dt in (BF, FP):
            dst = [torch.full(t.shape, 3.0, dtype=dst_dt, device="cuda") for t in ts]
            ctx.clip_grads(ts, max_norm, out, dst=dst, ord=ord)
            got = f64(out)
            assert abs(got[0] - norm) <= 1e-12 * norm and abs(got[1] - c) <= 1e-12
            for t, d, w in zip(ts, dst, want):
                assert np.array_equal(f64(t), w)
                tol = 2 * 2.0 ** -24 + (2.0 ** -8 if dst_dt is BF else 0)
                assert (np.abs(f64(d) - w * c) <= tol * np.abs(w * c) + 1e-45).all()
    keep = [t.clone() for t in ts]
    ctx.clip_grads(ts, norm * 2, out, ord=ord)
    assert all(torch.equal(a, b) for a, b in zip(ts, keep))
    ctx.clip_grads(ts, 0.37 * norm, out, ord=ord)
    same = [torch.empty_like(t) for t in ts]
    ctx.clip_grads(keep, 0.37 * norm, out, dst=same, ord=ord)
    assert all(torch.equal(a, b) for a, b in zip(ts, same))  # in place or not: the same bits
    if norm:
        assert abs(o8.grad_norm([f64(t) for t in ts], ord) / (0.37 * norm) - 1) <= 2.0 ** -8


@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("off", range(1, 9))
def test_tensors_at_any_address_and_the_space_between(ctx, dt, off):
    """Views at odd offsets of one buffer: neighbours that touch, gaps that hold NaN and
    stay as they are."""
    sizes, at, views = [17, 1, 4099, 300, 8192, 9], off, []
    flat = torch.full((30000,), float("nan"), dtype=dt, device="cuda")
    for i, n in enumerate(sizes):
        flat[at:at + n] = grads(i, [n], [dt])[0]
        views.append(flat[at:at + n])
        at += n + (0 if i % 2 else off)
    want = [f64(v) for v in views]
    norm = o8.grad_norm(want)
    out = torch.empty(2, dtype=DB, device="cuda")
    into = torch.full((30000,), 5.0, device="cuda")
    ctx.clip_grads(views, 1.5, out, dst=[into[2 * i + sum(sizes[:i]):][:n] for i, n in enumerate(sizes)])
    for i, (n, w) in enumerate(zip(sizes, want)):
        got = f64(into[2 * i + sum(sizes[:i]):][:n])
        assert (np.abs(got - w * 1.5 / norm) <= 2.0 ** -22 * np.abs(w)).all()
    assert int((into == 5.0).sum()) == 30000 - sum(sizes)
    ctx.clip_grads(views, 1.5, out)
    assert abs(float(out[0]) - norm) <= 1e-12 * norm
    assert int(flat.isnan().sum()) == 30000 - sum(sizes)
    for v, w in zip(views, want):
        tol = 2.0 ** -22 + (2.0 ** -8 if dt is BF else 0)
        assert (np.abs(f64(v) - w * 1.5 / norm) <= tol * np.abs(w)).all()


@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("ord", [2, INF])
@pytest.mark.parametrize("bad", [INF, -INF, float("nan")])
def test_a_norm_that_is_not_finite_leaves_the_gradients(ctx, dt, ord, bad):
    ts = grads(2, [100, 9000, 3], [dt])
    ts[1][8999] = bad
    keep = [t.clone() for t in ts]
    out = torch.empty(2, dtype=DB, device="cuda")
    ctx.clip_grads(ts, 1.0, out, ord=ord)
    assert float(out[1]) == 1.0 and not np.isfinite(float(out[0]))
    assert np.isnan(float(out[0])) == np.isnan(bad)
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(ts, keep))


def test_squares_that_leave_fp32_do_not_leave_the_norm(ctx):
    for v in (1e30, 1e-30):
        t = torch.full((1000,), v, device="cuda")
        out = torch.empty(2, dtype=DB, device="cuda")
        ctx.clip_grads([t], v, out)
        x = float(np.float32(v))
        assert abs(float(out[0]) / (x * 1000 ** 0.5) - 1) < 1e-12
        assert abs(float(t.double().norm()) / v - 1) < 2.0 ** -22


def test_a_models_flat_gradient(ctx):
    """dtheta as the VJP writes it, whole (zeros in its padding) or tensor by tensor."""
    lay, n = ctx.layout, ctx.n_params
    flat = torch.zeros(n, device="cuda")
    for i, (_, at, c, _, _) in enumerate(lay):
        flat[at:at + c] = grads(i, [c], [FP])[0]
    out = torch.empty(2, dtype=DB, device="cuda")
    a, b = torch.empty(n, device="cuda"), torch.zeros(n, device="cuda")
    ctx.clip_grads(flat, 1.0, out, dst=a)
    one = out.clone()
    ctx.clip_grads(pk.GradList([flat[o:o + c] for _, o, c, _, _ in lay]), 1.0, out,
                   dst=pk.GradList([b[o:o + c] for _, o, c, _, _ in lay]))
    assert abs(float(one[0] / out[0]) - 1) < 1e-12
    assert float((a - b).abs().max()) <= 2.0 ** -23 * float(a.abs().max())


def test_replays_of_a_captured_clip():
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx = pk.Context(pk.config("tiny"), stream=s)
        ts = grads(3, [70000, 9, 33333], [FP])
        out, dst = torch.empty(2, dtype=DB, device="cuda"), [torch.empty_like(t) for t in ts]
        src = pk.GradList(ts)
        ctx.clip_grads(src, 2.0, out, dst=dst)
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            ctx.clip_grads(src, 2.0, out, dst=dst)
        other = grads(4, [500000], [BF])
        for i in range(4):
            for t in ts:
                t.mul_(1.0 - 0.3 * i)
            ctx.clip_grads(src, 2.0, out, dst=dst)
            s.synchronize()
            want = [d.clone() for d in dst] + [out.clone()]
            for d in dst + [out]:
                d.zero_()
            ctx.grad_norm(other, torch.empty(1, dtype=DB, device="cuda"))
            g.replay()
            s.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(dst + [out], want))


def test_elements_past_32_bits(ctx):
    """4.4 billion bf16 elements: the last ones count and are scaled."""
    n = (1 << 32) + (1 << 27) + 5
    t = torch.zeros(n, dtype=BF, device="cuda")
    t[0], t[-1], t[(1 << 32) + 1] = 3.0, 4.0, 12.0
    out = torch.empty(2, dtype=DB, device="cuda")
    ctx.clip_grads([t], 6.5, out)
    assert float(out[0]) == 13.0 and float(out[1]) == 0.5
    assert (float(t[0]), float(t[-1]), float(t[(1 << 32) + 1])) == (1.5, 2.0, 6.0)


def test_binding_refuses_bad_lists(ctx):
    t, out = torch.zeros(64, device="cuda"), torch.empty(2, dtype=DB, device="cuda")
    for bad in (lambda: ctx.clip_grads([t, t], 1.0, out), lambda: ctx.clip_grads([t[:40], t[30:]], 1.0, out),
                lambda: ctx.clip_grads([t], 1.0, out[:1]), lambda: ctx.clip_grads([t], 1.0, out.float()),
                lambda: ctx.clip_grads([t], -1.0, out), lambda: ctx.clip_grads([t], float("nan"), out),
                lambda: ctx.clip_grads([t], 1.0, out, ord=1), lambda: ctx.clip_grads([t.double()], 1.0, out),
                lambda: ctx.clip_grads([t[::2]], 1.0, out), lambda: ctx.clip_grads([t.cpu()], 1.0, out),
                lambda: ctx.clip_grads([], 1.0, out), lambda: ctx.clip_grads([t], 1.0, out, dst=[t, t[:0]]),
                lambda: ctx.clip_grads([t], 1.0, out, dst=[torch.zeros(63, device="cuda")]),
                lambda: ctx.clip_grads([t[:32]], 1.0, out, dst=[t[16:48]]),
                lambda: ctx.clip_grads([t[:32], t[32:]], 1.0, out, dst=[t[32:], t[:32]]),
                lambda: ctx.clip_grads([t], 1.0, out, dst=[t.view(BF)[:64]])):
        with pytest.raises(pk.JaggError):
            bad()
