"""The local step's operators together, as the example runs them: rounds of preference tuning with 4-bit layers."""
import numpy as np
import pytest
import torch

import paper_2609_36662_amd as al
from oracle import mxfp4 as omx
from oracle import preference as opref
from workloads import preference_step as ps

pytestmark = pytest.mark.gpu


def test_rounds_of_local_steps_learn_the_preferences():
    h = ps.run(workers=3, rounds=3, steps=6)
    # the policy starts as its reference: every pair's loss is log 2
    assert h[0]["first_loss"] == pytest.approx(np.log(2), abs=1e-6)
    assert all(r["last_loss"] < r["first_loss"] for r in h) and h[-1]["last_loss"] < 0.6 * np.log(2)
    assert all(r["finite"] and np.isfinite(r["grad_norm"]) and r["D"] > 0 and 0 <= r["C"] < 3 for r in h)
    assert h == ps.run(workers=3, rounds=3, steps=6)      # the same bits every time


def test_one_step_against_the_formulas():
    """Every stage of one worker's step against the float64 oracle on that stage's own inputs."""
    shape = ps.Shape(features=70, hidden=45, vocab=133, pairs=2, longest=12)
    n = 45 * 70 + 133 * 45
    with al.autoloco_create(0) as ctx:
        w = ps.Worker(ctx, shape, torch.randn(n, generator=torch.Generator().manual_seed(3)).cuda() * 0.3, 4)
        w.w[1].add_(0.05 * torch.randn(133, 45, device="cuda"))     # away from the reference
        w.gradients(0.5)
        torch.cuda.synchronize()
        f = lambda t: t.double().cpu().numpy()  # noqa: E731
        x, h, w1, w2, g = f(w.x), f(w.h), f(w.w[0]), f(w.w[1]), f(w.logits)
        h_ref = np.maximum(omx.rounded(x) @ omx.rounded(w1).T, 0)
        np.testing.assert_allclose(h, h_ref, rtol=2.0 ** -8, atol=1e-5)
        logits = torch.from_numpy(omx.rounded(h) @ omx.rounded(w2).T).to(torch.bfloat16).double().numpy()
        losses, logps, grads, _, _ = opref.preference(logits, w.labels.cpu().numpy(), w.offsets.cpu().numpy(), f(w.ref), 0.5, 0.0, 0.5)
        np.testing.assert_allclose(f(w.losses), losses, rtol=2e-3)   # a logit's bf16 rounding may fall the other way
        np.testing.assert_allclose(g, grads, rtol=0.05, atol=2e-4)
        np.testing.assert_allclose(f(w.grads[1]), omx.rounded(g.T) @ omx.rounded(h.T).T, rtol=1e-4, atol=1e-6)
        dh = (omx.rounded(g) @ omx.rounded(w2.T).T) * (h > 0)
        np.testing.assert_allclose(f(w.dh), dh, rtol=2.0 ** -8, atol=1e-6)
        np.testing.assert_allclose(f(w.grads[0]), omx.rounded(f(w.dh).T) @ omx.rounded(x.T).T, rtol=1e-4, atol=1e-6)
