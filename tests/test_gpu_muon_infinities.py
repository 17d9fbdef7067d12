"""A gradient that is not finite makes its whole matrix NaN in the orthogonalised step, after any number of iterations, and
no other."""
import pytest
import torch

import paper_2609_36662_amd as al

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    with al.autoloco_create(0) as c:
        yield c


@pytest.mark.parametrize("iterations", [0, 1, 5])
@pytest.mark.parametrize("bad", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_whole_matrix(ctx, bad, iterations, dtype):
    gen = torch.Generator().manual_seed(2)
    shapes = [(40, 130), (130, 40), (1, 1), (1, 9), (64, 64)]
    grads = [torch.randn(s, generator=gen).to(dtype).cuda() for s in shapes for _ in range(2)]
    params = [torch.ones(g.shape, device="cuda") for g in grads]
    for g in grads[::2]:
        g[-1, -1] = bad
    ml = al.autoloco_muon_create(ctx, params, [torch.zeros(g.shape, device="cuda") for g in grads], grads)
    al.autoloco_inner_muon(ctx, ml, al.make_muon_coeffs(lr=0.1, iterations=iterations))
    for i, p in enumerate(params):
        assert torch.isnan(p).all() if i % 2 == 0 else torch.isfinite(p).all(), (i, p.shape)
    ml.close()
