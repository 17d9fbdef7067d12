"""4-bit floating point on the GPU against the float64 oracle: quantisation bit for
bit in both directions, the values back, products, the single-token form, refusals.

Products: the operands are exact, so only the sum rounds.  Its error is at most
(cols / 16 + 8) 2^-23 sum_k |a_k b_k| (one rounding or truncation of the running sum,
which never exceeds that sum, for every 16 products at worst); rounding is monotone, so
a bf16 result lies between the roundings of the two ends."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2609_36662_amd as al
from oracle import mxfp4 as omx

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx():
    with al.autoloco_create(0) as c:
        yield c


def _codes_equal(got, want):
    """Equal codes, but for the sign of a zero."""
    z = lambda c: np.where(c & 7, c, 0)  # noqa: E731
    lo, hi = z(got & 15), z(got >> 4)
    assert np.array_equal(lo, z(want & 15)) and np.array_equal(hi, z(want >> 4))


def _edge_values(rows, cols, seed):
    """Values of all magnitudes: ties, neighbours of ties, subnormals, zeros, huge ones, blocks of one kind."""
    rng = np.random.default_rng(seed)
    x = rng.normal(0, 1, (rows, cols)) * np.exp2(rng.integers(-20, 20, (rows, 1)))
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0, 6.0, 4.0, 0.0, 7.75])
    pick = rng.random((rows, cols)) < 0.4
    x = np.where(pick, rng.choice(ties, (rows, cols)) * np.exp2(rng.integers(-3, 3, (rows, 1))) * rng.choice([-1, 1], (rows, cols)), x)
    x = np.where(rng.random((rows, cols)) < 0.05, np.nextafter(x.astype(np.float32), np.float32(9e9)), x)
    for r, s in ((0, 0.0), (1, 2.0 ** -140), (2, 2.0 ** -126), (3, 2.0 ** 125), (4, 2.0 ** -122), (5, 2.0 ** -96)):
        if r < rows:
            x[r] *= s
    return x.astype(np.float32)


SHAPES = [(1, 1), (1, 32), (2, 31), (3, 33), (7, 128), (5, 129), (33, 255), (64, 64), (129, 127), (130, 300), (257, 65)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("forms", ["rows", "cols", "both"])
def test_quantize(ctx, rows, cols, dtype, forms):
    x = torch.from_numpy(_edge_values(rows, cols, rows * 1000 + cols)).to(DT[dtype])
    q = al.Mxfp4.empty(rows, cols) if forms != "cols" else None
    qt = al.Mxfp4.empty(cols, rows) if forms != "rows" else None
    for m in (q, qt):
        if m is not None:
            m.codes.fill_(0xA5)
            m.scales.fill_(0xA5)
    al.autoloco_mxfp4_quantize(ctx, x.cuda(), q, qt)
    ref = x.double().numpy()
    for m, r in ((q, ref), (qt, ref.T)):
        if m is None:
            continue
        codes, scales = omx.pack(*omx.quantize(r))
        assert np.array_equal(m.scales.cpu().numpy(), scales)
        _codes_equal(m.codes.cpu().numpy(), codes)
        for out in (torch.float32, torch.bfloat16):
            back = torch.empty((m.rows, m.cols), dtype=out, device="cuda")
            al.autoloco_mxfp4_dequantize(ctx, m, back)
            assert np.array_equal(back.double().cpu().numpy(), omx.rounded(r), equal_nan=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_quantize_every_bf16_pattern(ctx, dtype):
    """Every bf16 number as the only value of its block, and beside a larger one."""
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    x = torch.zeros((1 << 16, 32), dtype=torch.bfloat16)
    x[:, 5] = bits
    x[:, 9] = bits * 0.3
    x[1::2, 20] = bits[1::2] * 3.0
    x = x.to(DT[dtype])
    q = al.Mxfp4.empty(*x.shape)
    al.autoloco_mxfp4_quantize(ctx, x.cuda(), q)
    codes, scales = omx.pack(*omx.quantize(x.double().numpy()))
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    _codes_equal(q.codes.cpu().numpy(), codes)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_non_finite_blocks_become_nan(ctx, dtype, bad):
    x = torch.randn(40, 200)
    x[3, 40] = bad
    x[39, 199] = bad
    x = x.to(DT[dtype])
    q, qt = al.Mxfp4.empty(40, 200), al.Mxfp4.empty(200, 40)
    al.autoloco_mxfp4_quantize(ctx, x.cuda(), q, qt)
    for m, r in ((q, x), (qt, x.t())):
        back = torch.empty((m.rows, m.cols), device="cuda")
        al.autoloco_mxfp4_dequantize(ctx, m, back)
        assert np.array_equal(back.cpu().numpy(), omx.rounded(r.double().numpy()), equal_nan=True)
    w = al.Mxfp4.empty(9, 200)
    al.autoloco_mxfp4_quantize(ctx, torch.randn(9, 200).cuda(), w)
    y = torch.empty((40, 9), device="cuda")
    al.autoloco_mxfp4_matmul(ctx, q, w, y)
    nan = torch.isnan(y.cpu()).all(1)
    assert nan[3] and nan[39] and int(torch.isnan(y).sum()) == 18
    few = torch.empty((6, 9), dtype=DT[dtype], device="cuda")
    al.autoloco_mxfp4_linear(ctx, x[1:7].contiguous().cuda(), w, few)
    assert torch.isnan(few).all(1).tolist() == [False, False, True, False, False, False] and int(torch.isnan(few).sum()) == 9


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_odd_addresses(ctx, dtype):
    """A window of a larger matrix that begins at an odd element, rows at odd strides; a broadcast row; outputs alike."""
    big = torch.randn(70, 301).to(DT[dtype]).cuda()
    for x in (big[3:60, 1:276], big[5:6].expand(40, 301), big[:, 7:8], big[2:66:2, 3:163]):
        q, qt = al.Mxfp4.empty(*x.shape), al.Mxfp4.empty(x.shape[1], x.shape[0])
        al.autoloco_mxfp4_quantize(ctx, x, q, qt)
        r = x.double().cpu().numpy()
        for m, v in ((q, r), (qt, r.T)):
            codes, scales = omx.pack(*omx.quantize(v))
            assert np.array_equal(m.scales.cpu().numpy(), scales)
            _codes_equal(m.codes.cpu().numpy(), codes)
    out = torch.full((61, 400), 7.0, dtype=DT[dtype], device="cuda")
    x = big[3:60, 1:276]
    q = al.Mxfp4.empty(*x.shape)
    al.autoloco_mxfp4_quantize(ctx, x, q)
    al.autoloco_mxfp4_dequantize(ctx, q, out[2:59, 3:278])
    want = torch.full((61, 400), 7.0)
    want[2:59, 3:278] = torch.from_numpy(omx.rounded(x.double().cpu().numpy())).float()
    assert torch.equal(out.float().cpu(), want)


def _check_product(got, a, b, dtype, cols):
    """a [m, k], b [n, k]: the float64 values of the operands."""
    ref, mag = a @ b.T, np.abs(a) @ np.abs(b).T
    bound = (cols / 16 + 8) * 2.0 ** -23 * mag
    ends = [torch.from_numpy(ref + s * bound).to(DT[dtype]).double().numpy() for s in (-1, 1)]
    g = got.double().cpu().numpy()
    bad = ~((ends[0] <= g) & (g <= ends[1]))
    assert not bad.any(), (np.argwhere(bad)[:4], g[bad][:4], ref[bad][:4])


PRODUCTS = [(1, 1, 1), (17, 1, 33), (1, 17, 200), (32, 32, 64), (64, 64, 128), (65, 63, 129), (128, 128, 256), (100, 300, 700),
            (257, 129, 515), (300, 511, 96), (256, 256, 1024), (513, 260, 384), (40, 1000, 2100), (1025, 40, 130)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", PRODUCTS)
def test_matmul(ctx, m, n, k, dtype):
    rng = np.random.default_rng(m + n + k)
    x = (rng.normal(0, 1, (m, k)) * np.exp2(rng.integers(-6, 6, (m, 1)))).astype(np.float32)
    w = rng.normal(0, 0.02, (n, k)).astype(np.float32)
    xq, wq = al.Mxfp4.empty(m, k), al.Mxfp4.empty(n, k)
    al.autoloco_mxfp4_quantize(ctx, torch.from_numpy(x).cuda(), xq)
    al.autoloco_mxfp4_quantize(ctx, torch.from_numpy(w).cuda(), wq)
    guard = torch.full((m + 2, n + 5), -77.0, dtype=DT[dtype], device="cuda")
    out = guard[1:m + 1, 3:n + 3]
    al.autoloco_mxfp4_matmul(ctx, xq, wq, out)
    _check_product(out, omx.rounded(x), omx.rounded(w), dtype, k)
    inside = torch.zeros_like(guard, dtype=torch.bool)
    inside[1:m + 1, 3:n + 3] = True
    assert torch.all(guard[~inside] == -77.0)
    first = out.clone()
    al.autoloco_mxfp4_matmul(ctx, xq, wq, out)
    assert torch.equal(first, out)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(2000, 2040, 3100), (1999, 1921, 4000), (2000, 1500, 300), (1999, 1501, 129), (2049, 1409, 640), (1700, 1931, 20), (3300, 3800, 1200),
                                   (3301, 3799, 1281), (3299, 3841, 2100)])
def test_matmul_large_tiles(ctx, m, n, k, dtype):
    """Sizes that take 128 x 128 and 256 x 256 tiles, ragged in every direction; the float64 product on the GPU."""
    rng = np.random.default_rng(m + n + k)
    x = (rng.normal(0, 1, (m, k)) * np.exp2(rng.integers(-6, 6, (m, 1)))).astype(np.float32)
    w = rng.normal(0, 0.02, (n, k)).astype(np.float32)
    xq, wq = al.Mxfp4.empty(m, k), al.Mxfp4.empty(n, k)
    al.autoloco_mxfp4_quantize(ctx, torch.from_numpy(x).cuda(), xq)
    al.autoloco_mxfp4_quantize(ctx, torch.from_numpy(w).cuda(), wq)
    guard = torch.full((m + 2, n + 5), -77.0, dtype=DT[dtype], device="cuda")
    out = guard[1:m + 1, 3:n + 3]
    al.autoloco_mxfp4_matmul(ctx, xq, wq, out)
    a, b = (torch.from_numpy(omx.rounded(v)).cuda() for v in (x, w))
    ref, bound = a @ b.t().contiguous(), (k / 16 + 8) * 2.0 ** -23 * (a.abs() @ b.abs().t().contiguous())
    assert torch.all((ref - bound).to(DT[dtype]) <= out) and torch.all(out <= (ref + bound).to(DT[dtype]))
    inside = torch.zeros_like(guard, dtype=torch.bool)
    inside[1:m + 1, 3:n + 3] = True
    assert torch.all(guard[~inside] == -77.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 16, 128), (1, 1000, 2048), (2, 33, 31), (3, 100, 4100), (8, 257, 515), (13, 4099, 640),
                                   (15, 48, 127), (16, 64, 1024), (16, 5000, 260), (17, 300, 515), (33, 70, 1000)])
def test_linear(ctx, m, n, k, dtype):
    rng = np.random.default_rng(m * n + k)
    x = torch.from_numpy((rng.normal(0, 1, (m, k)) * np.exp2(rng.integers(-6, 6, (m, 1)))).astype(np.float32)).to(DT[dtype])
    w = rng.normal(0, 0.02, (n, k)).astype(np.float32)
    wq = al.Mxfp4.empty(n, k)
    al.autoloco_mxfp4_quantize(ctx, torch.from_numpy(w).cuda(), wq)
    guard = torch.full((m + 2, n + 5), -77.0, dtype=DT[dtype], device="cuda")
    y = guard[1:m + 1, 3:n + 3]
    xq = al.Mxfp4.empty(m, k) if m > 16 else None
    padded = torch.randn(m, k + 3, device="cuda").to(DT[dtype])
    padded[:, 1:k + 1] = x.cuda()
    al.autoloco_mxfp4_linear(ctx, padded[:, 1:k + 1], wq, y, xq)
    _check_product(y, omx.rounded(x.double().numpy()), omx.rounded(w), dtype, k)
    inside = torch.zeros_like(guard, dtype=torch.bool)
    inside[1:m + 1, 3:n + 3] = True
    assert torch.all(guard[~inside] == -77.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_gradients_of_a_layer(ctx, dtype):
    """dx and dW against the formulas on the rounded operands, and against difference quotients of the layer's
    output: it is linear in either operand, so they are exact up to rounding."""
    m, n, k = 70, 90, 150
    rng = np.random.default_rng(5)
    dy = torch.from_numpy(rng.normal(0, 1e-2, (m, n)).astype(np.float32)).to(DT[dtype]).cuda()
    x = torch.from_numpy(rng.normal(0, 1, (m, k)).astype(np.float32)).to(DT[dtype]).cuda()
    w = torch.from_numpy(rng.normal(0, 0.05, (n, k)).astype(np.float32)).cuda()
    dyq, dyt, xt, wt = al.Mxfp4.empty(m, n), al.Mxfp4.empty(n, m), al.Mxfp4.empty(k, m), al.Mxfp4.empty(k, n)
    al.autoloco_mxfp4_quantize(ctx, dy, dyq, dyt)
    al.autoloco_mxfp4_quantize(ctx, x, None, xt)
    al.autoloco_mxfp4_quantize(ctx, w, None, wt)
    dx, dw = torch.empty((m, k), device="cuda"), torch.empty((n, k), device="cuda")
    al.autoloco_mxfp4_matmul(ctx, dyq, wt, dx)
    al.autoloco_mxfp4_matmul(ctx, dyt, xt, dw)
    d, xd, wd = dy.double().cpu().numpy(), x.double().cpu().numpy(), w.double().cpu().numpy()
    _check_product(dx, omx.rounded(d), omx.rounded(wd.T), "f32", n)
    _check_product(dw, omx.rounded(d.T), omx.rounded(xd.T), "f32", m)
    # sum(dy * y) with the rounded operands, moved by 1 in one weight, changes by that weight's gradient
    xr, dr = omx.rounded(xd.T).T, omx.rounded(d.T).T
    for i, j in ((0, 0), (n - 1, k - 1), (13, 77)):
        w2 = wd.copy()
        w2[i, j] += 1.0
        diff = np.sum(dr * (xr @ w2.T)) - np.sum(dr * (xr @ wd.T))
        assert abs(diff - float(dw[i, j])) <= 1e-9 + (m / 16 + 8) * 2.0 ** -23 * np.sum(np.abs(dr[:, i] * xr[:, j])) * 2


def test_codes_past_32_bits(ctx):
    """More than 2^32 bytes of codes, from one row broadcast: every row of the form is the first one's, and a product
    with it has equal columns."""
    rows, cols = 70001, 131072
    row = torch.randn(1, cols, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    q = al.Mxfp4.empty(rows, cols)
    q.codes[-1].fill_(0xA5)
    al.autoloco_mxfp4_quantize(ctx, row.expand(rows, cols), q)
    codes, scales = omx.pack(*omx.quantize(row.double().cpu().numpy()))
    want, wants = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).cuda()
    for a in range(0, rows, 10000):
        assert torch.equal(q.codes[a:a + 10000], q.codes[:1].expand(min(10000, rows - a), -1))
    _codes_equal(q.codes[-1:].cpu().numpy(), want.cpu().numpy())
    assert torch.equal(q.scales, wants.expand(-1, rows, -1))
    for m in (5, 40):
        x = torch.randn(m, cols, device="cuda")
        y, xq = torch.empty((m, rows), device="cuda"), al.Mxfp4.empty(m, cols)
        al.autoloco_mxfp4_linear(ctx, x, q, y, xq)
        assert torch.equal(y, y[:, :1].expand(m, rows))
        _check_product(y[:, -1:], omx.rounded(x.double().cpu().numpy()), omx.rounded(row.double().cpu().numpy()), "f32", cols)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_past_32_bits(ctx, dtype):
    """Rows of x and of the results that begin beyond 2^32 bytes."""
    rows, cols, stride = 21, 150, (1 << 28) + 3
    store = torch.empty(stride * (rows - 1) + cols, dtype=DT[dtype], device="cuda")
    x = torch.as_strided(store, (rows, cols), (stride, 1))
    x.copy_(torch.randn(rows, cols))
    q, qt = al.Mxfp4.empty(rows, cols), al.Mxfp4.empty(cols, rows)
    al.autoloco_mxfp4_quantize(ctx, x, q, qt)
    ref = x.double().cpu().numpy()
    for m, r in ((q, ref), (qt, ref.T)):
        codes, scales = omx.pack(*omx.quantize(r))
        assert np.array_equal(m.scales.cpu().numpy(), scales)
        _codes_equal(m.codes.cpu().numpy(), codes)
    w = al.Mxfp4.empty(cols, cols)
    wv = np.random.default_rng(2).normal(0, 1, (cols, cols)).astype(np.float32)
    al.autoloco_mxfp4_quantize(ctx, torch.from_numpy(wv).cuda(), w)
    for m in (rows, 9):
        y = torch.empty((m, cols), dtype=DT[dtype], device="cuda")
        al.autoloco_mxfp4_linear(ctx, x[:m], w, y, al.Mxfp4.empty(m, cols))
        _check_product(y, omx.rounded(ref[:m]), omx.rounded(wv), dtype, cols)
    y = x[:9].clone()
    al.autoloco_mxfp4_linear(ctx, y, w, x[9:18])
    _check_product(x[9:18], omx.rounded(ref[:9]), omx.rounded(wv), dtype, cols)
    al.autoloco_mxfp4_matmul(ctx, q, w, x)
    _check_product(x, omx.rounded(ref), omx.rounded(wv), dtype, cols)
    al.autoloco_mxfp4_dequantize(ctx, q, x)
    assert np.array_equal(x.double().cpu().numpy(), omx.rounded(ref))


def test_empty_matrices(ctx):
    e = al.Mxfp4.empty
    for rows, cols in ((0, 5), (5, 0), (0, 0)):
        x = torch.empty((rows, cols), device="cuda")
        al.autoloco_mxfp4_quantize(ctx, x, e(rows, cols), e(cols, rows))
        al.autoloco_mxfp4_dequantize(ctx, e(rows, cols), x)
    for m, n in ((3, 40), (40, 3)):   # nothing to add up: zeros
        for dt in DT.values():
            y = torch.full((m, n + 2), 7.0, dtype=dt, device="cuda")
            al.autoloco_mxfp4_matmul(ctx, e(m, 0), e(n, 0), y[:, 1:n + 1])
            assert torch.all(y[:, 1:n + 1] == 0) and torch.all(y[:, 0] == 7) and torch.all(y[:, n + 1] == 7)
            y.fill_(7.0)
            al.autoloco_mxfp4_linear(ctx, torch.empty((m, 0), dtype=dt, device="cuda"), e(n, 0), y[:, 1:n + 1], e(m, 0))
            assert torch.all(y[:, 1:n + 1] == 0) and torch.all(y[:, 0] == 7) and torch.all(y[:, n + 1] == 7)
    al.autoloco_mxfp4_matmul(ctx, e(0, 64), e(9, 64), torch.empty((0, 9), device="cuda"))
    al.autoloco_mxfp4_linear(ctx, torch.empty((0, 64), device="cuda"), e(9, 64), torch.empty((0, 9), device="cuda"))


def test_refusals(ctx):
    f = lambda *s, dt=torch.float32: torch.zeros(s, dtype=dt, device="cuda")  # noqa: E731
    e = al.Mxfp4.empty
    err = al.AutolocoError

    def refused(status, call, *args):
        with pytest.raises(err) as ex:
            call(ctx, *args)
        assert ex.value.status == status, ex.value

    quant, deq, mm, lin = (al.autoloco_mxfp4_quantize, al.autoloco_mxfp4_dequantize, al.autoloco_mxfp4_matmul,
                           al.autoloco_mxfp4_linear)
    refused(-1, quant, f(4, 64))                                   # neither form
    refused(-1, quant, f(4, 64), e(5, 64))
    refused(-1, quant, f(4, 64), None, e(4, 64))                   # not transposed
    refused(-1, deq, e(4, 64), f(4, 65))
    refused(-1, mm, e(4, 64), e(5, 65), f(4, 5))
    refused(-1, mm, e(4, 64), e(5, 64), f(5, 4))
    refused(-1, lin, f(20, 64), e(5, 64), f(20, 5))                # xq missing beyond 16 rows
    refused(-1, lin, f(20, 64), e(5, 64), f(20, 5), e(20, 65))
    refused(-1, lin, f(4, 64), e(5, 64), f(4, 5, dt=torch.bfloat16))
    refused(-1, deq, e(4, 64), torch.as_strided(f(400), (4, 64), (10, 1)))   # the output's rows overlap
    room = f(64 * 70, dt=torch.uint8)
    mis = al.Mxfp4(4, 64, room[1:257], f(16, dt=torch.uint8))
    refused(-2, quant, f(4, 64), mis)
    shared = f(8, 64)
    refused(-3, quant, shared.view(torch.uint8).view(torch.float32), al.Mxfp4(8, 64, shared.view(torch.uint8).reshape(-1)[:512], f(32, dt=torch.uint8)))
    q = e(4, 64)
    refused(-3, quant, f(4, 64), q, al.Mxfp4(64, 4, _same_codes(q), f(256, dt=torch.uint8)))
    q = e(4, 64)
    host = al._lib.Matrix(torch.zeros(4, 64).pin_memory().data_ptr(), 4, 64, 64, 0)
    assert al.lib().autoloco_mxfp4_quantize(ctx.handle, C.byref(host), C.byref(q.buffers), None) == -1
    assert "not device memory" in al.autoloco_last_error(ctx)
    bad = al.make_matrix(f(4, 64))
    for field, value in (("dtype", 7), ("rows", -1), ("cols", 1 << 31), ("stride", -4), ("data", None)):
        m = al._lib.Matrix(bad.data, bad.rows, bad.cols, bad.stride, bad.dtype)
        setattr(m, field, value)
        assert al.lib().autoloco_mxfp4_quantize(ctx.handle, C.byref(m), C.byref(q.buffers), None) == -1, field
    assert al.lib().autoloco_mxfp4_quantize(None, C.byref(bad), C.byref(q.buffers), None) == -1
    for args in ((f(4),), (torch.zeros(4, 64),), (f(4, 64, dt=torch.float64),), (f(64, 4).t(),)):
        with pytest.raises((TypeError, ValueError)):
            quant(ctx, *args, e(4, 64))
    with pytest.raises(ValueError):
        al.Mxfp4(4, 64, f(255, dt=torch.uint8), f(16, dt=torch.uint8))


def _same_codes(q):
    """A 64 x 4 matrix's codes that begin where q's do."""
    big = torch.zeros(64 * 64, dtype=torch.uint8, device="cuda")
    q.buffers.codes = big.data_ptr()
    return big


def test_graph_replays(ctx):
    """Captured into a graph and replayed, with eager work between, every replay gives the eager result."""
    stream = torch.cuda.Stream()
    with al.autoloco_create(0, stream) as c, torch.cuda.stream(stream):
        x, w = torch.randn(200, 300, device="cuda"), torch.randn(150, 300, device="cuda")
        wq, xq, y = al.Mxfp4.empty(150, 300), al.Mxfp4.empty(200, 300), torch.empty((200, 150), device="cuda")
        y1 = torch.empty((3, 150), device="cuda")
        def work():
            al.autoloco_mxfp4_quantize(c, w, wq)
            al.autoloco_mxfp4_linear(c, x, wq, y, xq)
            al.autoloco_mxfp4_linear(c, x[:3], wq, y1)
        work()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            work()
        for i in range(4):
            x.normal_()
            w.normal_()
            graph.replay()
            got = y.clone(), y1.clone()
            work()
            stream.synchronize()
            assert torch.equal(got[0], y) and torch.equal(got[1], y1)


@pytest.mark.parametrize("rows,stride", [(1 << 30, 1 << 40), ((1 << 24) + 1, 1 << 40), (1 << 30, 1 << 19)])
def test_a_matrix_longer_than_any_memory_is_refused(ctx, rows, stride):
    """Rows and strides in range whose product is not: the span must not wrap round 64 bits."""
    x = torch.zeros((4, 64), device="cuda")
    q = al.Mxfp4.empty(4, 64)
    m = al._lib.Matrix(x.data_ptr(), rows, 4, stride, 0)
    lib, handle = al.lib(), ctx.handle
    assert lib.autoloco_mxfp4_quantize(handle, C.byref(m), C.byref(q.buffers), None) == -1
    assert "shape of x out of range" in al.autoloco_last_error(ctx)
    assert lib.autoloco_mxfp4_dequantize(handle, C.byref(q.buffers), C.byref(m)) == -1
    assert "shape of out out of range" in al.autoloco_last_error(ctx)
