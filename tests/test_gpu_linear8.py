"""8-bit linear-layer operators on the GPU against the fp64 oracle: block
quantisation (bit for bit), the product (exactly, on operands whose sums fit fp32;
within the bound of its summation otherwise), the residual RMS norm and its
gradient, odd sizes, strides, non-finite values, buffers' margins, graphs and
streams."""
import numpy as np
import pytest
import torch

import paper_2607_17572_amd as pk
from oracle import linear8 as o8

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float32
FMT = {"e4m3": pk.E4M3, "e5m2": pk.E5M2}
MARGIN = 4096


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


def rand(seed, *shape, spread=0.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(*shape, generator=g)
    if spread:
        x = x * torch.exp(spread * torch.randn(*shape, generator=g))
    return x


def f64(t):
    return t.detach().double().cpu().numpy()


def guarded(nbytes):
    """(all bytes, the middle nbytes) of a buffer with a pattern on both sides."""
    full = torch.full((nbytes + 2 * MARGIN,), 0xA5, dtype=torch.uint8, device="cuda")
    return full, full[MARGIN:MARGIN + nbytes]


def intact(full):
    return bool((full[:MARGIN] == 0xA5).all()) and bool((full[-MARGIN:] == 0xA5).all())


def guarded_mat(rows, k, fmt="e4m3"):
    ld, words = -(-k // 128) * 128, -(-k // 512)
    fq, q = guarded(rows * ld)
    fs, s = guarded(words * rows * 4)
    return pk.Mat8(rows, k, FMT[fmt], q=q.view(rows, ld), scale=s.view(words, rows, 4)), (fq, fs)


def unpack(m):
    """(values [rows][ld], exponent bytes [rows][4 ceil(k/512)]) of a Mat8."""
    q = o8.table8("e5m2" if m.fmt else "e4m3")[m.q.cpu().numpy()]
    return q, m.scale.cpu().numpy().transpose(1, 0, 2).reshape(m.rows, -1).astype(np.int64)


def check_mat(m, y, fmt, tile=1):
    """m holds y (fp64 values of fp32 numbers) bit for bit, with zero padding."""
    q, s = unpack(m)
    wq, ws = o8.quantize8(y, fmt, tile)
    nb = ws.shape[1]
    assert np.array_equal(s[:, :nb], ws) and not s[:, nb:].any()
    assert np.array_equal(q[:, :m.k], wq, equal_nan=True)
    assert not np.nan_to_num(q[:, m.k:]).any()


# ------------------------------------------------------------------ quantiser
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 700), (3, 128), (129, 127), (128, 512), (260, 641), (7, 1030), (515, 9)])
@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("tile", [False, True])
def test_quantize8_bit_for_bit(ctx, rows, cols, dt, fmt, tile):
    say(f"case: quantize8 {rows}x{cols} {dt} {fmt} tile={tile}")
    x = rand(rows + cols, rows, cols, spread=2.0).to(dt)
    if rows > 1:
        x[rows // 2] = 0  # a row of zeros
    out, g1 = guarded_mat(rows, cols, fmt)
    out_t, g2 = guarded_mat(cols, rows, fmt)
    xd = x.cuda()
    ctx.quantize8(xd, out, out_t, tile=tile)
    check_mat(out, f64(x), fmt, 128 if tile else 1)
    check_mat(out_t, f64(x).T, fmt, 128 if tile else 1)
    assert all(intact(g) for g in g1 + g2)
    one, t_one = pk.Mat8(rows, cols, FMT[fmt]), pk.Mat8(cols, rows, FMT[fmt])
    ctx.quantize8(xd, out=one, tile=tile)  # each form alone gives the same bytes
    ctx.quantize8(xd, out_t=t_one, tile=tile)
    for a, b in ((one, out), (t_one, out_t)):
        assert torch.equal(a.q, b.q) and torch.equal(a.scale, b.scale)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
def test_quantize8_extremes(ctx, fmt):
    """Every exponent of fp32, ties, subnormal blocks, the largest finite value."""
    x = torch.zeros(300, 256)
    for i in range(276):
        x[i, :128] = rand(i, 128) * 2.0 ** (i - 149 if i < 149 else i - 150)
    x[276, 0] = torch.finfo(FP).max
    x[277, 5] = 2.0 ** -149
    x[278] = torch.arange(256) / 16.0  # many ties
    x[279, :] = float(o8.MOST[fmt])
    x[280, :] = float(np.nextafter(np.float32(o8.MOST[fmt]), np.float32(1e9)))
    x = torch.where(torch.isfinite(x), x, torch.ones(()))
    out, out_t = pk.Mat8(300, 256, FMT[fmt]), pk.Mat8(256, 300, FMT[fmt])
    ctx.quantize8(x.cuda(), out, out_t)
    check_mat(out, f64(x), fmt)
    check_mat(out_t, f64(x).T, fmt)


@pytest.mark.parametrize("tile", [False, True])
def test_quantize8_non_finite_blocks_are_nan(ctx, tile):
    x = rand(5, 140, 300)
    x[3, 7], x[130, 290], x[139, 200] = float("inf"), float("nan"), float("-inf")
    out, out_t = pk.Mat8(140, 300), pk.Mat8(300, 140)
    ctx.quantize8(x.cuda(), out, out_t, tile=tile)
    for m, y in ((out, f64(x)), (out_t, f64(x).T)):
        q, s = unpack(m)
        wq, ws = o8.quantize8(y, "e4m3", 128 if tile else 1)
        assert (ws == 255).any() and np.array_equal(s[:, :ws.shape[1]], ws)
        assert np.array_equal(q[:, :m.k], wq, equal_nan=True)


@pytest.mark.parametrize("dt", [BF, FP])
def test_quantize8_multipliers_strides_and_odd_addresses(ctx, dt):
    rows, cols = 133, 391
    big = rand(6, rows, cols + 13).to(dt).cuda()
    x = big[:, 5:5 + cols]  # rows at addresses that are multiples of the element only
    rm, cm = rand(7, rows).cuda(), rand(8, cols).to(dt).cuda()
    y = (x.float() * rm[:, None]) * cm.float()
    out, out_t = pk.Mat8(rows, cols), pk.Mat8(cols, rows)
    ctx.quantize8(x, out, out_t, row_mul=rm, col_mul=cm)
    check_mat(out, f64(y), "e4m3")
    check_mat(out_t, f64(y).T, "e4m3")


# -------------------------------------------------------------------- product
def whole_mat(seed, rows, k, fmt, spread=3):
    """An 8-bit matrix of small whole numbers with scales 2^0 .. 2^spread, so that sums
    of products fit fp32; (Mat8, fp64 values)."""
    g = np.random.default_rng(seed)
    v = g.integers(-3, 4, (rows, k)).astype(np.float64)
    s = 127 + g.integers(0, spread + 1, (rows, -(-k // 128)))
    ld, words = -(-k // 128) * 128, -(-k // 512)
    table = o8.table8(fmt)
    code = np.array([int(np.nonzero(table == x)[0][0]) for x in range(-3, 4)])
    q = np.zeros((rows, ld), dtype=np.uint8)
    q[:, :k] = code[(v + 3).astype(int)]
    sc = np.zeros((rows, words * 4), dtype=np.uint8)
    sc[:, :s.shape[1]] = s
    sc = np.ascontiguousarray(sc.reshape(rows, words, 4).transpose(1, 0, 2))
    m = pk.Mat8(rows, k, FMT[fmt], q=torch.from_numpy(q).cuda(), scale=torch.from_numpy(sc).cuda())
    return m, o8.values8(v, s)


SIZES = [(1, 1, 1), (1, 64, 128), (1, 515, 1000), (2, 40, 4096), (7, 1000, 513), (16, 96, 640), (17, 130, 64), (33, 257, 2049),
         (64, 64, 64), (65, 63, 129), (100, 300, 127), (128, 128, 1024), (130, 511, 777), (257, 255, 300), (300, 1030, 1152),
         (513, 520, 4224), (1, 4100, 260), (37, 700, 5000), (520, 1, 1300), (1030, 33, 260)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dt", [BF, FP])
def test_matmul8_exact_on_whole_numbers(ctx, m, n, k, dt):
    fmt = "e5m2" if (m + n + k) % 2 else "e4m3"
    say(f"case: matmul8 {m}x{n}x{k} {fmt} {dt}")
    a, va = whole_mat(m, m, k, fmt)
    b, vb = whole_mat(n + 1, n, k, "e4m3")
    want = va @ vb.T
    assert np.abs(va).sum(1).max() * np.abs(vb).max() < 2 ** 24  # every partial sum is exact in fp32
    full, mid = guarded(m * n * (2 if dt is BF else 4))
    out = mid.view(dt).view(m, n)
    ctx.matmul8(a, b, out)
    exact = torch.from_numpy(want)
    assert torch.equal(out.cpu(), exact.to(dt)) and intact(full)
    # bias and accumulation, into rows of a wider buffer: the columns beside are not written
    wide = torch.full((m, n + 3), 7.0, dtype=dt, device="cuda")
    wide[:, 1:n + 1] = 2.0
    bias = torch.arange(n, dtype=FP).remainder(5).to(dt).cuda()
    ctx.matmul8(a, b, wide[:, 1:n + 1], bias=bias, beta=1.0)
    want2 = (exact + bias.double().cpu() + 2.0).to(dt)
    assert torch.equal(wide[:, 1:n + 1].cpu(), want2)
    assert bool((wide[:, 0] == 7).all()) and bool((wide[:, n + 1:] == 7).all())
    ctx.matmul8(a, b, wide[:, 1:n + 1], bias=bias)
    assert torch.equal(wide[:, 1:n + 1].cpu(), (exact + bias.double().cpu()).to(dt))


@pytest.mark.parametrize("m,n,k", [(17, 131, 9000), (40, 515, 12288), (129, 257, 8001), (640, 300, 7000), (1100, 70, 15000)])
@pytest.mark.parametrize("dt", [BF, FP])
def test_matmul8_with_a_split_contraction(m, n, k, dt):
    """Few tiles and a long k: sums of each split, joined in order; the workspace holds
    NaN before."""
    say(f"case: matmul8 split {m}x{n}x{k} {dt}")
    ctx = pk.Context(pk.config("tiny"))
    a, va = whole_mat(m, m, k, "e5m2", 1)
    b, vb = whole_mat(n + 1, n, k, "e4m3", 1)
    out = torch.full((m, n + 2), 3.0, dtype=dt, device="cuda")
    bias = torch.arange(n, dtype=FP).remainder(7).to(dt).cuda()
    ctx.matmul8(a, b, out[:, 1:n + 1])
    ctx._ensure_bytes(1)  # (129 rows in bf16 need none: four groups of k in a workgroup)
    ctx._ws.view(torch.uint8).fill_(0xFF)
    ctx.matmul8(a, b, out[:, 1:n + 1], bias=bias)
    want = torch.from_numpy(va @ vb.T) + bias.double().cpu()
    assert torch.equal(out[:, 1:n + 1].cpu(), want.to(dt))
    out[:, 1:n + 1] = 2.0
    ctx.matmul8(a, b, out[:, 1:n + 1], bias=bias, beta=1.0)
    assert torch.equal(out[:, 1:n + 1].cpu(), (want + 2).to(dt))
    assert bool((out[:, 0] == 3).all()) and bool((out[:, n + 1] == 3).all())


@pytest.mark.parametrize("m,n,k,fmt", [(17, 4096, 4096, "e4m3"), (33, 1030, 4000, "e5m2"), (63, 31, 5100, "e4m3"),
                                       (64, 2049, 2300, "e5m2"), (133, 333, 5249, "e4m3"), (600, 33, 3100, "e5m2"),
                                       (33, 9000, 4096, "e4m3"), (20, 33, 1537, "e5m2")])
@pytest.mark.parametrize("dt", [BF, FP])
def test_matmul8_few_rows_and_a_long_k(ctx, m, n, k, fmt, dt):
    """Tiles of 64 x 32 whose four groups of waves share k, some of them with nothing left
    of it: whole numbers, exactly."""
    say(f"case: matmul8 few rows {m}x{n}x{k} {fmt} {dt}")
    a, va = whole_mat(m, m, k, fmt, 1)
    b, vb = whole_mat(n + 1, n, k, "e4m3", 1)
    assert np.abs(va).sum(1).max() * np.abs(vb).max() < 2 ** 24
    want = torch.from_numpy(va @ vb.T)
    bias = torch.arange(n, dtype=FP).remainder(5).to(dt).cuda()
    out = torch.full((m + 2, n + 3), 7.0, dtype=dt, device="cuda")
    mid = out[1:m + 1, 1:n + 1]
    ctx.matmul8(a, b, mid, bias=bias)
    assert torch.equal(mid.cpu(), (want + bias.double().cpu()).to(dt))
    ctx.matmul8(a, b, mid, beta=1.0)
    again = ((want + bias.double().cpu()).to(dt).double() + want).to(dt)
    assert torch.equal(mid.cpu(), again)
    out[1:m + 1, 1:n + 1] = 7
    assert bool((out == 7).all())


@pytest.mark.parametrize("m,n,k,fmt", [(4096, 4096, 500, "e4m3"), (5000, 5000, 2048, "e5m2"), (5000, 5001, 1990, "e4m3"),
                                       (8200, 8200, 512, "e4m3"), (16000, 2056, 1024, "e5m2")])
def test_matmul8_with_more_tiles_than_compute_units(ctx, m, n, k, fmt):
    """bf16 results: a workgroup goes from tile to tile.  Rows of a wider buffer; a bias at
    an odd place and accumulation (which take a workgroup per tile) give the same."""
    say(f"case: matmul8 many tiles {m}x{n}x{k} {fmt}")
    a, va = whole_mat(m, m, k, fmt, 1)
    b, vb = whole_mat(n + 1, n, k, "e4m3", 1)
    assert np.abs(va).sum(1).max() * np.abs(vb).max() < 2 ** 24
    want = torch.from_numpy(va.astype(np.float32) @ vb.astype(np.float32).T)  # whole numbers below 2^24: exact
    bias = torch.arange(n + 1, dtype=FP).remainder(5).to(BF).cuda()
    out = torch.full((m, n + 3), 7.0, dtype=BF, device="cuda")
    mid = out[:, 1:n + 1]
    ctx.matmul8(a, b, mid)
    assert torch.equal(mid.cpu(), want.to(BF))
    for at in (0, 1):
        mid.fill_(3)
        ctx.matmul8(a, b, mid, bias=bias[at:at + n])
        wanted = (want + bias[at:at + n].float().cpu()).to(BF)
        assert torch.equal(mid.cpu(), wanted), at
    mid.fill_(2)
    ctx.matmul8(a, b, mid, bias=bias[1:], beta=1.0)
    assert torch.equal(mid.cpu(), (want + bias[1:].float().cpu() + 2).to(BF))
    assert bool((out[:, 0] == 7).all()) and bool((out[:, n + 1:] == 7).all())


@pytest.mark.parametrize("m,n,k,fmt", [(1, 300, 3000, "e4m3"), (5, 129, 8200, "e5m2"), (40, 200, 2000, "e4m3"),
                                       (200, 333, 2500, "e5m2"), (600, 700, 1100, "e4m3")])
def test_matmul8_on_quantised_values(ctx, m, n, k, fmt):
    """fp32 sums: a product is exact, each of at most 64 additions inside an
    instruction and of K/64 + 64 between them is off by at most 2^-23 (a truncated
    fp32) of the sum of magnitudes so far."""
    say(f"case: matmul8 {m}x{n}x{k} {fmt} quantised")
    a, b = pk.Mat8(m, k, FMT[fmt]), pk.Mat8(n, k)
    ctx.quantize8((rand(m, m, k, spread=1.5) * 1e-3).cuda(), a)
    ctx.quantize8(rand(n, n, k).cuda(), b, tile=True)
    va, vb = (o8.values8(unpack(x)[0][:, :k], unpack(x)[1]) for x in (a, b))
    out = torch.empty(m, n, device="cuda")
    ctx.matmul8(a, b, out)
    bound = (k / 64 + 128) * 2.0 ** -23 * (np.abs(va) @ np.abs(vb).T)
    err = np.abs(f64(out) - va @ vb.T)
    assert (err <= bound).all(), (err / bound).max()
    again = torch.empty_like(out)
    ctx.matmul8(a, b, again)
    assert torch.equal(out, again)


def test_matmul8_without_a_bias_after_one_with(ctx):
    """Nothing of a call's bias is left on the chip for the next one; a replayed graph of
    both gives the same."""
    m, n, k = 5000, 5000, 2048
    a, va = whole_mat(m, m, k, "e4m3", 0)
    b, vb = whole_mat(n + 1, n, k, "e4m3", 0)
    want = torch.from_numpy(va.astype(np.float32) @ vb.astype(np.float32).T)
    bias = torch.full((n,), 2.0 ** 20, dtype=BF, device="cuda")
    with_, without = torch.empty(m, n, dtype=BF, device="cuda"), torch.empty(m, n, dtype=BF, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        c = pk.Context(pk.config("tiny"), stream=s)

        def both():
            c.matmul8(a, b, with_, bias=bias)
            c.matmul8(a, b, without)
        both()
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            both()
        for i in range(4):
            if i:
                with_.fill_(1)
                without.fill_(1)
                g.replay()
            s.synchronize()
            assert torch.equal(without.cpu(), want.to(BF)), i
            assert torch.equal(with_.cpu(), (want + 2.0 ** 20).to(BF)), i


def test_matmul8_carries_nan_and_zero_blocks(ctx):
    m, n, k = 70, 50, 700
    x, w = rand(1, m, k), rand(2, n, k)
    x[5, 300], x[9] = float("inf"), 0
    a, b = pk.Mat8(m, k), pk.Mat8(n, k)
    ctx.quantize8(x.cuda(), a)
    ctx.quantize8(w.cuda(), b)
    out = torch.empty(m, n, device="cuda")
    ctx.matmul8(a, b, out)
    assert bool(out[5].isnan().all()) and bool((out[9] == 0).all())
    assert not bool(out[:5].isnan().any()) and not bool(out[6:].isnan().any())


@pytest.mark.parametrize("m,n,k", [(3, 40, 700), (70, 50, 700), (200, 300, 1500), (2100, 2100, 400), (4200, 4200, 300), (40, 300, 9000)])
@pytest.mark.parametrize("dt", [BF, FP])
def test_matmul8_takes_exponent_255_as_nan_and_0_as_the_least(ctx, m, n, k, dt):
    """Whatever the bytes of a block are: exponent 255 makes its row (or column) of the
    result NaN; exponent 0 scales by 2^-127."""
    say(f"case: matmul8 exponents {m}x{n}x{k} {dt}")
    a, va = whole_mat(m, m, k, "e4m3", 0)
    b, vb = whole_mat(n, n, k, "e4m3", 0)
    a.scale[0, 2, 1], b.scale[0, 7, 0] = 255, 255
    a.scale[:, 0, :] = 0
    b.scale[:, 5, :] = 254  # 2^127 (2^-127) = 1
    out = torch.empty(m, n, dtype=dt, device="cuda")
    ctx.matmul8(a, b, out)
    got = f64(out)
    # (column 5 of the other rows is whole numbers times 2^127: past fp32's largest, 2^128)
    rest = np.delete(got, 5, axis=1)
    assert np.isnan(got[2]).all() and np.isnan(got[:, 7]).all() and np.isnan(rest).sum() == m + n - 2
    fine = [i for i in range(min(m, 60)) if i not in (0, 2)]
    cols = [j for j in range(min(n, 60)) if j not in (5, 7)]
    assert np.array_equal(got[np.ix_(fine, cols)], f64(torch.from_numpy(va[fine] @ vb[cols].T).to(dt)))
    if dt is BF:
        assert got[0, 5] == f64(torch.tensor(float(va[0] @ vb[5])).to(dt))


@pytest.mark.parametrize("m", [2, 33, 300000])
def test_matmul8_operands_past_4_gib(ctx, m):
    """Offsets of the last rows lie past 32 bits: on the left with many rows, on the
    right with few."""
    rows, k = 300000, 16000
    say(f"case: matmul8 past 4 GiB, {m} rows")
    ld = 16000 // 128 * 128
    assert rows * ld > 2 ** 32
    code = torch.tensor(sorted({int(np.nonzero(o8.table8("e4m3") == x)[0][0]) for x in (-1, 0, 1)}), dtype=torch.uint8,
                        device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    q = torch.empty(rows, ld, dtype=torch.uint8, device="cuda")
    for i in range(0, rows, 30000):
        q[i:i + 30000] = code[torch.randint(0, 3, (30000, ld), generator=g, device="cuda")]
    sc = torch.full((-(-k // 512), rows, 4), 127, dtype=torch.uint8, device="cuda")
    sc[-1, :, 1:] = 0  # 125 blocks
    big = pk.Mat8(rows, k, q=q, scale=sc)
    small, vs = whole_mat(9, 24 if m == rows else m, k, "e4m3", 1)
    a, b = (big, small) if m == rows else (small, big)
    out = torch.empty(a.rows, b.rows, device="cuda")
    ctx.matmul8(a, b, out)
    at = torch.tensor([0, 1, 150001, 268434, 268436, 299998, 299999])
    vb = o8.table8("e4m3")[q[at.cuda()].cpu().numpy()]
    want = vb @ vs.T if m == rows else vs @ vb.T
    got = out[at.cuda()] if m == rows else out[:, at.cuda()]
    assert np.array_equal(f64(got), want)


# ----------------------------------------------------------------------- norm
NORM_SIZES = [(1, 1), (1, 130), (3, 512), (5, 1000), (70, 513), (9, 2048), (4, 2051), (3, 4096), (5, 5000), (2, 8192), (2, 9001),
              (3, 16384), (2, 20000), (1, 32768)]


@pytest.mark.parametrize("rows,cols", NORM_SIZES)
@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("residual", [False, True])
def test_rmsnorm8(ctx, rows, cols, dt, residual):
    """h exactly; rstd: a sum of squares of depth at most 32 + 6 + 16 additions, two more
    operations and a halving by the root: 2^-24 (54 / 2 + 5); y: within half a step
    of 8 bits plus the fp32 error of (h rstd) gain."""
    say(f"case: rmsnorm8 {rows}x{cols} {dt} residual={residual}")
    eps, fe = 1e-5, (54 / 2 + 5) * 2.0 ** -24
    x, r, g = rand(1, rows, cols, spread=1.0).to(dt), rand(2, rows, cols).to(dt), (1 + 0.3 * rand(3, cols)).to(dt)
    if rows > 2:
        x[1] = 0
        r[1] = 0
    full, mid = guarded(rows * cols * x.element_size())
    h, rstd = mid.view(dt).view(rows, cols), torch.empty(rows, device="cuda")
    y, gy = guarded_mat(rows, cols)
    ctx.rmsnorm8(x.cuda(), g.cuda(), y, residual=r.cuda() if residual else None, h=h, rstd=rstd, eps=eps)
    wh = (x.float() + r.float()).to(dt) if residual else x
    assert torch.equal(h.cpu(), wh) and intact(full) and all(intact(t) for t in gy)
    wr, wy = o8.rmsnorm(f64(wh), f64(g), eps)
    assert (np.abs(f64(rstd) / wr - 1) <= fe).all()
    q, s = unpack(y)
    nb = -(-cols // 128)
    got = o8.values8(q[:, :cols], s)
    step = np.repeat(np.ldexp(1.0, s[:, :nb] - 127), 128, axis=1)[:, :cols]
    assert (np.abs(got - wy) <= np.maximum(2.0 ** -4 * np.abs(wy), 2.0 ** -10 * step) * (1 + 1e-3) + (fe + 2.0 ** -22) * np.abs(wy)).all()
    pad = np.zeros((rows, nb * 128))
    pad[:, :cols] = np.abs(wy)
    amax, e = pad.reshape(rows, nb, 128).max(2), fe + 2.0 ** -22
    top = np.ldexp(448.0, s[:, :nb] - 127)
    assert (amax * (1 - e) <= top).all() and (amax * (1 + e) > top / 2)[s[:, :nb] > 0].all()
    assert not s[:, nb:].any() and not q[:, cols:].any()
    # the quantiser with the same factors makes the same bytes
    two = pk.Mat8(rows, cols)
    ctx.quantize8(h, two, row_mul=rstd, col_mul=g.cuda())
    assert torch.equal(two.q, y.q) and torch.equal(two.scale, y.scale)


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 130), (3, 512), (70, 513), (2500, 96), (600, 2051), (5, 5000), (3, 9001), (2, 32768)])
@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("add,beta", [(False, 0.0), (True, 1.0)])
def test_rmsnorm8_grad(ctx, rows, cols, dt, add, beta):
    """fp32: the mean's sum has depth at most 54, eight more operations; a column sum
    adds at most rows / 512 + 600 numbers.  One rounding to the output's type."""
    say(f"case: rmsnorm8_grad {rows}x{cols} {dt} add={add}")
    eps = 1e-5
    h, dy, dh = rand(1, rows, cols, spread=1.0).to(dt), rand(2, rows, cols).to(dt), rand(3, rows, cols).to(dt)
    g = (1 + 0.3 * rand(4, cols)).to(dt)
    wr, _ = o8.rmsnorm(f64(h), f64(g), eps)
    rstd = torch.from_numpy(wr).float()
    full, mid = guarded(rows * cols * h.element_size())
    dx = mid.view(dt).view(rows, cols)
    fg, mg = guarded(cols * 4)
    dgain = mg.view(FP)
    dgain.copy_(rand(5, cols))
    was = f64(dgain)
    ctx.rmsnorm8_grad(dy.cuda(), h.cuda(), rstd.cuda(), g.cuda(), dx, dgain, dh=dh.cuda() if add else None, beta=beta)
    wx, wg = o8.rmsnorm_grad(f64(dy), f64(h), f64(g), eps)
    n, a = np.abs(f64(h) * wr[:, None]), np.abs(f64(dy) * f64(g))
    size = wr[:, None] * (a + n * (a * n).mean(1, keepdims=True))
    if add:
        wx, size = wx + f64(dh), size + np.abs(f64(dh))
    tol = 62 * 2.0 ** -24 * size + (2.0 ** -8 if dt is BF else 0) * np.abs(wx)
    assert (np.abs(f64(dx) - wx) <= tol).all() and intact(full)
    gtol = (rows / 512 + 610) * 2.0 ** -24 * ((np.abs(f64(dy)) * n).sum(0) + beta * np.abs(was))
    assert (np.abs(f64(dgain) - wg - beta * was) <= gtol).all() and intact(fg)


@pytest.mark.parametrize("dt", [BF, FP])
def test_norm_in_place_and_strided(ctx, dt):
    rows, cols = 37, 1111
    buf = [rand(i, rows, cols + 9).to(dt).cuda() for i in range(4)]
    x, r, dy, dh = (b[:, 3:3 + cols] for b in buf)
    g = (1 + 0.3 * rand(4, cols)).to(dt).cuda()
    rstd = torch.empty(rows, device="cuda")
    y1, y2 = pk.Mat8(rows, cols), pk.Mat8(rows, cols)
    h = torch.empty(rows, cols, dtype=dt, device="cuda")
    ctx.rmsnorm8(x.contiguous(), g, y1, residual=r.contiguous(), h=h, rstd=rstd)
    dx, dg = torch.empty_like(h), torch.empty(cols, dtype=dt, device="cuda")
    ctx.rmsnorm8_grad(dy.contiguous(), h, rstd, g, dx, dg, dh=dh.contiguous())
    ctx.rmsnorm8(x, g, y2, residual=r, h=x)  # the residual stream updated in place, in a wider buffer
    assert torch.equal(x, h) and torch.equal(y1.q, y2.q) and torch.equal(y1.scale, y2.scale)
    edge = buf[0][:, :3].clone(), buf[0][:, 3 + cols:].clone()
    dg2 = torch.empty_like(dg)
    ctx.rmsnorm8_grad(dy, x, rstd, g, dh, dg2, dh=dh)  # the gradient stream updated in place
    assert torch.equal(dh, dx) and torch.equal(dg, dg2)
    assert torch.equal(edge[0], buf[0][:, :3]) and torch.equal(edge[1], buf[0][:, 3 + cols:])


def test_norm_of_a_row_with_nan_touches_no_other_row(ctx):
    x, g = rand(1, 6, 700), torch.ones(700)
    x[2, 3], x[4, 699] = float("nan"), float("inf")
    y, rstd = pk.Mat8(6, 700), torch.empty(6, device="cuda")
    ctx.rmsnorm8(x.cuda(), g.cuda(), y, rstd=rstd)
    q, s = unpack(y)
    assert np.isnan(q[2, :700]).all() and not np.isnan(q[[0, 1, 3, 5]]).any()
    assert (s[2, :6] == 255).all() and (s[4, 5] == 255) and (s[[0, 1, 3, 5]] < 255).all()


# ------------------------------------------------------------------- together
def layer(ctx, t, out):
    """One 8-bit layer's training step: norm, forward, both backward products, the
    norm's backward, and the clip of its gradients."""
    ctx.rmsnorm8(t["x"], t["gain"], out["y"], residual=t["r"], h=out["h"], rstd=out["rstd"])
    ctx.matmul8(out["y"], t["w8"], out["o"])
    ctx.quantize8(t["do"], out["d8"], out["d8t"])
    ctx.matmul8(out["d8"], t["w8t"], out["dy"])
    ctx.quantize8(out["h"], out_t=out["yt"], row_mul=out["rstd"], col_mul=t["gain"])
    ctx.matmul8(out["d8t"], out["yt"], out["dw"])
    ctx.rmsnorm8_grad(out["dy"], out["h"], out["rstd"], t["gain"], out["dx"], out["dgain"], dh=t["dh"])
    ctx.clip_grads([out["dw"], out["dgain"]], 0.25, out["clip"])


def layer_state(M, D, F):
    dev = dict(device="cuda")
    t = dict(x=rand(1, M, D).to(BF), r=rand(2, M, D).to(BF), gain=(1 + 0.2 * rand(3, D)).to(BF),
             w=(rand(4, F, D) * D ** -0.5).to(BF), do=(rand(5, M, F) * 1e-2).to(BF), dh=(rand(6, M, D) * 1e-2).to(BF))
    t = {k: v.cuda() for k, v in t.items()}
    out = dict(y=pk.Mat8(M, D), h=torch.empty(M, D, dtype=BF, **dev), rstd=torch.empty(M, **dev),
               o=torch.empty(M, F, dtype=BF, **dev), d8=pk.Mat8(M, F, pk.E5M2), d8t=pk.Mat8(F, M, pk.E5M2),
               dy=torch.empty(M, D, dtype=BF, **dev), yt=pk.Mat8(D, M), dw=torch.empty(F, D, **dev),
               dx=torch.empty(M, D, dtype=BF, **dev), dgain=torch.empty(D, **dev),
               clip=torch.empty(2, dtype=torch.float64, **dev))
    return t, out


def weights(ctx, t):
    F, D = t["w"].shape
    t["w8"], t["w8t"] = pk.Mat8(F, D), pk.Mat8(D, F)
    ctx.quantize8(t["w"], t["w8"], t["w8t"], tile=True)


def test_a_layers_step_against_fp64(ctx):
    """The whole chain against the exact gradients of the unquantised layer: each 8-bit
    operand is off by at most 2^-4 of each value (E5M2: 2^-3), with signs that
    differ, so a product of two such operands stays within 2^-4 + 2^-3 of the result's
    norm times the ratio of the operands' magnitudes to the result (1 in the mean for
    independent roundings)."""
    M, D, F = 300, 520, 777
    t, out = layer_state(M, D, F)
    weights(ctx, t)
    layer(ctx, t, out)
    x = {k: f64(v) for k, v in t.items() if torch.is_tensor(v)}
    h = f64((t["x"].float() + t["r"].float()).to(BF))
    rstd, y = o8.rmsnorm(h, x["gain"], 1e-6)
    dy = x["do"] @ x["w"]
    dh, dg = o8.rmsnorm_grad(dy, h, x["gain"], 1e-6)
    dw = x["do"].T @ y
    norm = o8.grad_norm([dw, dg])
    c = o8.clip_factor(norm, 0.25)
    assert c < 1

    def rel(a, b):
        return np.linalg.norm(f64(a) - b) / np.linalg.norm(b)

    assert rel(out["o"], y @ x["w"].T) < 2.0 ** -4 * 2
    assert rel(out["dy"], dy) < 2.0 ** -3 + 2.0 ** -4
    assert rel(out["dx"], dh + x["dh"]) < 2.0 ** -3 + 2.0 ** -4
    assert rel(out["dw"], dw * c) < 2.0 ** -3 + 2.0 ** -4
    assert rel(out["dgain"], dg * c) < 2.0 ** -3 + 2.0 ** -4
    got = f64(out["clip"])
    assert abs(got[0] / norm - 1) < 2.0 ** -3 and abs(got[1] * got[0] - 0.25) < 1e-12


def test_a_layers_step_in_a_graph():
    """Captured on a stream of its own, replayed between eager steps of other data: every
    replay gives the eager bits."""
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx = pk.Context(pk.config("tiny"), stream=s)
        t, out = layer_state(130, 260, 390)
        weights(ctx, t)
        layer(ctx, t, out)  # also binds the workspace
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            layer(ctx, t, out)
        t2, out2 = layer_state(64, 700, 100)
        weights(ctx, t2)
        for i in range(4):
            for k, v in (("x", 10), ("do", 20), ("dh", 30)):
                t[k].copy_(rand(v + i, *t[k].shape).to(BF) * (1 if k == "x" else 1e-2))
            layer(ctx, t, out)
            s.synchronize()
            want = {k: (v.q.clone() if isinstance(v, pk.Mat8) else v.clone()) for k, v in out.items()}
            for v in out.values():
                (v.q if isinstance(v, pk.Mat8) else v).zero_()
            layer(ctx, t2, out2)  # eager work on the same workspace
            g.replay()
            s.synchronize()
            for k, v in out.items():
                assert torch.equal(v.q if isinstance(v, pk.Mat8) else v, want[k]), (i, k)


def test_a_first_call_inside_a_capture():
    """A context whose first calls are captured (its workspace is made and grows there),
    then used eagerly and replayed."""
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        one, two = (pk.Context(pk.config("tiny"), stream=s) for _ in range(2))
        t, out = layer_state(333, 520, 1000)
        big = layer_state(2000, 3000, 256)
        other = layer_state(50, 4000, 64)
        for st in (t, big[0], other[0]):
            weights(two, st)
        layer(two, t, out)
        layer(two, *big)
        s.synchronize()
        want = {k: (v.q if isinstance(v, pk.Mat8) else v).clone() for k, v in out.items()}
        want_big = big[1]["dw"].clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            layer(one, t, out)
            layer(one, *big)
        for _ in range(3):
            for v in out.values():
                (v.q if isinstance(v, pk.Mat8) else v).zero_()
            layer(one, *other)
            g.replay()
            s.synchronize()
            for k, v in out.items():
                assert torch.equal(v.q if isinstance(v, pk.Mat8) else v, want[k]), k
            assert torch.equal(big[1]["dw"], want_big)


def test_workspace_of_a_graph_outlives_a_larger_call():
    """A captured call keeps its workspace's address: a later call that needs a larger
    one must not free it."""
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        ctx = pk.Context(pk.config("tiny"), stream=s)
        big = layer_state(3000, 4000, 128)
        t, out = layer_state(70, 260, 128)
        for st in (t, big[0]):
            weights(ctx, st)
        layer(ctx, t, out)
        s.synchronize()
        want = out["dgain"].clone()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            layer(ctx, t, out)
        had = ctx._ws.data_ptr()
        layer(ctx, *big)
        assert ctx._ws.data_ptr() != had
        junk = torch.full((1 << 24,), float("nan"), device="cuda")  # takes what was freed
        for _ in range(3):
            out["dgain"].zero_()
            g.replay()
            s.synchronize()
            assert torch.equal(out["dgain"], want)
        assert bool(junk.isnan().all())


def test_two_contexts_on_two_streams_at_once():
    streams = [torch.cuda.Stream() for _ in range(2)]
    runs = []
    for s in streams:
        with torch.cuda.stream(s):
            ctx = pk.Context(pk.config("tiny"), stream=s)
            t, out = layer_state(520, 1024, 640)
            weights(ctx, t)
            layer(ctx, t, out)
            s.synchronize()
            runs.append((ctx, t, out, out["dw"].clone(), out["dgain"].clone()))
    for _ in range(3):
        for s, (ctx, t, out, _, _) in zip(streams, runs):
            with torch.cuda.stream(s):
                layer(ctx, t, out)
    torch.cuda.synchronize()
    for _, _, out, dw, dg in runs:
        assert torch.equal(out["dw"], dw) and torch.equal(out["dgain"], dg)


def test_binding_refuses_mismatched_tensors(ctx):
    a, b = pk.Mat8(8, 256), pk.Mat8(16, 256)
    out = torch.zeros(8, 16, device="cuda")
    x, g, y = torch.zeros(8, 256, device="cuda"), torch.ones(256, device="cuda"), pk.Mat8(8, 256)
    for bad in (lambda: ctx.matmul8(a, b, out.t()), lambda: ctx.matmul8(a, b, out[:, :15]), lambda: ctx.matmul8(a, b, out.double()),
                lambda: ctx.matmul8(a, pk.Mat8(16, 255), out), lambda: ctx.matmul8(a, b, out, bias=torch.zeros(15, device="cuda")),
                lambda: ctx.matmul8(a, b, out, bias=torch.zeros(16, dtype=BF, device="cuda")), lambda: ctx.matmul8(a, b, out.cpu()),
                lambda: ctx.matmul8(a, b, out, beta=0.5),
                lambda: ctx.quantize8(x, pk.Mat8(8, 255)), lambda: ctx.quantize8(x), lambda: ctx.quantize8(x.cpu(), y),
                lambda: ctx.quantize8(x, y, row_mul=g), lambda: ctx.quantize8(x.half(), y), lambda: ctx.quantize8(x[0], y),
                lambda: ctx.rmsnorm8(x, g.to(BF), y), lambda: ctx.rmsnorm8(x, g, y, residual=x.to(BF)),
                lambda: ctx.rmsnorm8(x, g, pk.Mat8(8, 256, pk.E5M2)), lambda: ctx.rmsnorm8(x, g, y, rstd=g),
                lambda: ctx.rmsnorm8_grad(x, x, g, g, x, g), lambda: ctx.rmsnorm8_grad(x, x, x[:, 0].contiguous(), g, x, g.double()),
                lambda: pk.Mat8(8, 256, q=torch.zeros(8, 128, dtype=torch.uint8, device="cuda")),
                lambda: pk.Mat8(8, 256, q=torch.zeros(8, 256, device="cuda")),
                lambda: pk.Mat8(8, 256, scale=torch.zeros(8, 4, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(pk.JaggError):
            bad()
