"""The timed workloads of the 8-bit and clipping operators (perf/operators.py) under
other streams than the one that was current first."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def fp32_default():
    """Another test file sets fp64 as the default type."""
    was = torch.get_default_dtype()
    torch.set_default_dtype(torch.float32)
    yield
    torch.set_default_dtype(was)


@pytest.fixture()
def ops():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf", "operators.py")
    spec = importlib.util.spec_from_file_location("operators", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    m.own = True
    return m


def test_calls_go_to_the_current_stream(ops):
    """One context for each stream, and the calls' results are there for work queued on
    that stream without a wait in between; a capture holds them."""
    first, other = torch.cuda.current_stream(), torch.cuda.Stream()
    _, here = ops._context()
    assert here.stream == first and ops._context()[1] is here
    with torch.cuda.stream(other):
        _, there = ops._context()
        assert there is not here and there.stream == other
    assert ops._context()[1] is here
    names = ("clip_tiny", "norm_token", "norm_grad_ragged", "quant_tile_ragged", "product_rows37")
    for case in [c for c in ops.listed() if c["name"] in names]:
        print("case:", case["name"], flush=True)
        want = [t.clone() for t in ops.run(ops.prepare(case, 3))]
        torch.cuda.synchronize()
        with torch.cuda.stream(other):
            state = ops.prepare(case, 3)
            got = [t.clone() for t in ops.run(state)]
            other.synchronize()
            assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want))
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=other):
                out = ops.run(state)
            for _ in range(3):
                for t in out:
                    t.view(torch.uint8).zero_()
                g.replay()
                other.synchronize()
                assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(out, want))
