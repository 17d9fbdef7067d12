"""Products of 4-bit matrices whose blocks have the smallest scales times ones whose blocks have the largest: every
scale byte below 32 and from 230 to 252, each way round, in every tile and in the single-token form, which also
quantises x's values of that size.  The products are ordinary fp32 numbers; the bound is that of the other products
((cols / 16 + 8) 2^-23 sum_k |a_k b_k|, which no factor by a power of two changes)."""
import numpy as np
import pytest
import torch

import paper_2609_36662_amd as al
from oracle import mxfp4 as omx

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
SMALL, LARGE = (0, 32), (230, 253)


@pytest.fixture(scope="module")
def ctx():
    with al.autoloco_create(0) as c:
        yield c


def _matrix(rows, cols, scales, seed):
    """A random 4-bit matrix with scale bytes of a range: its stored form on the device and its float64 values."""
    rng = np.random.default_rng(seed)
    codes = rng.integers(0, 16, (rows, cols)).astype(np.uint8)
    s = rng.integers(*scales, (rows, -(-cols // 32))).astype(np.uint8)
    q = al.Mxfp4(rows, cols, *(torch.from_numpy(p).cuda() for p in omx.pack(codes, s)))
    return q, torch.from_numpy(omx.values(codes, s)).cuda()


def _check(out, a, b):
    k = a.shape[1]
    ref, bound = a @ b.t().contiguous(), (k / 16 + 8) * 2.0 ** -23 * (a.abs() @ b.abs().t().contiguous())
    assert torch.all((ref - bound).to(out.dtype) <= out) and torch.all(out <= (ref + bound).to(out.dtype))


@pytest.mark.parametrize("first,second", [(SMALL, LARGE), (LARGE, SMALL)], ids=["small by large", "large by small"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(1, 1, 32), (65, 63, 129), (300, 511, 700), (2000, 1500, 300), (2000, 2040, 3100), (3300, 3800, 1200)])
def test_matmul(ctx, m, n, k, dtype, first, second):
    (aq, a), (bq, b) = _matrix(m, k, first, m + k), _matrix(n, k, second, n)
    out = torch.full((m, n), 7.0, dtype=DT[dtype], device="cuda")
    al.autoloco_mxfp4_matmul(ctx, aq, bq, out)
    _check(out, a, b)


@pytest.mark.parametrize("first,second", [(SMALL, LARGE), (LARGE, SMALL)], ids=["small by large", "large by small"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", [(1, 100, 64), (3, 4099, 300), (13, 9000, 515), (16, 64, 2100), (17, 300, 515)])
def test_linear(ctx, m, n, k, dtype, first, second):
    (_, x), (wq, w) = _matrix(m, k, first, m + k), _matrix(n, k, second, n)
    x = x.to(DT[dtype])
    xr = torch.from_numpy(omx.rounded(x.double().cpu().numpy())).cuda()
    y = torch.full((m, n), 7.0, dtype=DT[dtype], device="cuda")
    al.autoloco_mxfp4_linear(ctx, x, wq, y, al.Mxfp4.empty(m, k) if m > 16 else None)
    _check(y, xr, w)
