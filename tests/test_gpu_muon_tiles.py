"""The orthogonalised step's products in tiles of each size, against the float64 oracle.  A batch's tile goes by all of its
matrices: lists of many, and one matrix of its own, reach each size for each of the products (by the rule, in the order
X X^T, the polynomial, the update: 64 in all three; 128 with four stages; 128; 256; 256 x 128 for the update of the last)."""
import math

import numpy as np
import pytest
import torch

import paper_2609_36662_amd as al
from oracle import block as ob
from tests.block_common import f64
from tests.test_gpu_muon import U16, U32, _keep

pytestmark = pytest.mark.gpu
LISTS = [(1, (90, 93)), (62, (204, 201)), (62, (201, 204)), (45, (272, 257)), (57, (388, 484)), (57, (484, 388)), (1, (1505, 2711)),
         (1, (2711, 1505))]


@pytest.fixture(scope="module")
def ctx():
    with al.autoloco_create(0) as c:
        yield c


def _bound(x, scale):
    """Of one iteration, value by value: u = 2^-11 for what is rounded to fp16, 2^-25 / scale below its normal range,
    2^-36 of A and B, and fp32 sums, one rounding or truncation (2^-23) for every four products at worst."""
    a, b, c = (abs(v) for v in ob.NS)
    sums = lambda k: (k / 4 + 8) * 2.0 ** -23  # noqa: E731
    x = np.abs(x)
    A = x @ x.T
    rows = np.sum(x, 1)[:, None]
    ea = (3.01 * U16 + sums(x.shape[1])) * A + 2.0 ** -36 + 1.01 * 2.0 ** -25 / scale * (rows + rows.T)
    bb = b * A + c * A @ A
    eb = b * ea + c * (ea @ A + A @ ea + ea @ ea + sums(A.shape[0]) * A @ A) + U16 * bb + 2.0 ** -36
    return eb @ x + (bb + eb) @ (U16 * x + 2.0 ** -25 / scale) + sums(A.shape[0]) * (bb @ x) + 2.0 ** -20 * a * x + 2.0 ** -24


@pytest.mark.parametrize("count,shape", LISTS)
@pytest.mark.parametrize("iterations", [1, 3])
def test_against_the_oracle(ctx, count, shape, iterations):
    gen = torch.Generator().manual_seed(shape[0] + count)
    grads = [torch.randn(shape, generator=gen) for _ in range(count)]
    params = [torch.zeros(shape, device="cuda") for _ in grads]
    ml = al.autoloco_muon_create(ctx, params, [torch.zeros(shape, device="cuda") for _ in grads], [g.cuda() for g in grads])
    al.autoloco_inner_muon(ctx, ml, al.make_muon_coeffs(lr=1.0, weight_decay=0.0, momentum=0.0, iterations=iterations))
    torch.cuda.synchronize()
    ml.close()
    for i in sorted({0, count // 2, count - 1}):
        g = f64(grads[i])
        got, ref = -f64(params[i]) / (0.2 * math.sqrt(max(shape))), ob.orthogonalise(g, iterations)
        if iterations == 1:
            x = g if shape[0] <= shape[1] else g.T
            err = _bound(x / (np.linalg.norm(x) + 1e-7), 2.0 ** round(math.log2(math.sqrt(max(shape)))))
            err = err if shape[0] <= shape[1] else err.T
            assert np.all(np.abs(got - ref) <= err + 8 * U32 * np.abs(ref)), i
        else:
            model, norm = ob.orthogonalise(g, iterations, keep=_keep(max(shape))), np.linalg.norm(ref)
            assert np.linalg.norm(got - ref) <= 2 * np.linalg.norm(model - ref) + 2 * U16 * norm, i
