"""The bytes behind an 8-bit matrix's last column are zeros, as bytes: for negative and
non-finite factors, for blocks that are NaN, in rows, transposed rows and tiles."""
import pytest
import torch

import paper_2607_17572_amd as pk

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32
INF, NAN = float("inf"), float("nan")


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


def matrix(rows, k, fmt=pk.E4M3):
    m = pk.Mat8(rows, k, fmt)
    m.q.fill_(0xA5)
    m.scale.fill_(0xA5)
    return m


def check(m):
    """Zero bytes behind column k, up to the next multiple of 128; no scale behind the last block."""
    assert not bool(m.q[:, m.k:].any())
    s = m.scale.permute(1, 0, 2).reshape(m.rows, -1)
    assert not bool(s[:, -(-m.k // 128):].any())


@pytest.mark.parametrize("rows,cols", [(1, 1), (133, 391), (128, 7), (9, 640), (300, 129)])
@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("tile", [False, True])
@pytest.mark.parametrize("factors", ["none", "negative", "inf", "nan"])
def test_quantiser(ctx, rows, cols, dt, tile, factors):
    print(f"case: padding {rows}x{cols} {dt} tile={tile} {factors}", flush=True)
    g = torch.Generator().manual_seed(rows + cols)
    x = torch.randn(rows, cols, generator=g)
    x[rows // 2, cols // 2], x[-1, -1] = INF, NAN
    x = x.to(dt).cuda()
    v = {"none": None, "negative": -1.5, "inf": -INF, "nan": NAN}[factors]
    rm = None if v is None else torch.full((rows,), v, device="cuda")
    cm = None if v is None else torch.full((cols,), v, dtype=dt, device="cuda")
    for fmt in (pk.E4M3, pk.E5M2):
        for r, c in ((None, None), (rm, None), (None, cm), (rm, cm)):
            out, out_t = matrix(rows, cols, fmt), matrix(cols, rows, fmt)
            ctx.quantize8(x, out, out_t, tile=tile, row_mul=r, col_mul=c)
            check(out)
            check(out_t)


@pytest.mark.parametrize("cols", [1, 130, 700, 1000, 2051, 5000, 9001, 20000])
@pytest.mark.parametrize("dt", [BF, FP])
def test_norm(ctx, cols, dt):
    print(f"case: padding norm {cols} {dt}", flush=True)
    x = torch.randn(4, cols, generator=torch.Generator().manual_seed(cols))
    x[1, cols // 2], x[2, -1], x[3] = NAN, INF, 0
    y = matrix(4, cols)
    ctx.rmsnorm8(x.to(dt).cuda(), torch.full((cols,), -1.0, dtype=dt, device="cuda"), y, eps=0.0)
    check(y)
