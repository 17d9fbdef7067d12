"""Scalars of the block's calls that a double holds and the kernels' fp32 does not are refused."""
import pytest
import torch

import paper_2609_36662_amd as al

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    with al.autoloco_create(0) as c:
        yield c


@pytest.mark.parametrize("word,bad", [("scale", {"scale": 1e39}), ("scale", {"scale": -3.5e38}), ("eps", {"eps": 1e39}),
                                      ("eps", {"eps": 1e-46}), ("eps", {"eps": 5e-324}), ("eps", {"eps": 2.0 ** -126 * 0.99})])
def test_residual(ctx, word, bad):
    x, z = torch.ones((3, 40), device="cuda"), torch.zeros((3, 40), device="cuda")
    out, y, dx = (torch.full((3, 40), 7.0, device="cuda") for _ in range(3))
    with pytest.raises(al.AutolocoError, match=word):
        al.autoloco_residual_norm(ctx, x, None, y, z=z, out=out, **bad)
    with pytest.raises(al.AutolocoError, match=word):
        al.autoloco_residual_norm_grad(ctx, x, None, y, dx, z=z, **bad)
    torch.cuda.synchronize()
    assert all(torch.all(t == 7) for t in (out, y, dx))


def test_residual_at_the_ends(ctx):
    """The largest scales and the least eps that are taken: no row of zeros becomes NaN, nothing of its own accord infinite."""
    x, z = torch.ones((3, 40), device="cuda"), torch.zeros((3, 40), device="cuda")
    for k in ({"scale": 3.4e38}, {"scale": -3.4e38}, {"scale": 1e-300}, {"eps": 2.0 ** -126}, {"eps": 0.0}, {"eps": 3e38}):
        out, y = torch.full_like(x, 7.0), torch.full_like(x, 7.0)
        al.autoloco_residual_norm(ctx, x, None, y, z=z, out=out, **k)
        assert torch.equal(out, x) and torch.isfinite(y).all(), k
    for eps in (2.0 ** -126, 1e-6):
        y, dx = torch.full_like(z, 7.0), torch.full_like(z, 7.0)
        al.autoloco_residual_norm(ctx, z, None, y, eps=eps)
        al.autoloco_residual_norm_grad(ctx, z, None, x, dx, eps=eps)
        # t / sqrt(eps), the root and the division each half a step off
        assert not y.any() and torch.all((dx.double() * eps ** 0.5 - 1).abs() <= 4 * 2.0 ** -24)


@pytest.mark.parametrize("bad", [{"lr": 1e39}, {"lr": 2e36}, {"lr": 1e30, "weight_decay": 1e10}])
def test_orthogonalised_step(ctx, bad):
    w, m, g = torch.ones((8, 9), device="cuda"), torch.zeros((8, 9), device="cuda"), torch.ones((8, 9), device="cuda")
    ml = al.autoloco_muon_create(ctx, [w], [m], [g])
    with pytest.raises(al.AutolocoError, match="lr"):
        al.autoloco_inner_muon(ctx, ml, al.make_muon_coeffs(**bad))
    torch.cuda.synchronize()
    assert torch.all(w == 1) and not m.any()
    al.autoloco_inner_muon(ctx, ml, al.make_muon_coeffs(lr=1e35, weight_decay=1.0))
    assert torch.isfinite(w).all() and not torch.all(w == 1)
    ml.close()
