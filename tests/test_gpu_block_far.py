"""The block's operators where offsets pass 32 bits and a product has more tiles than one launch takes, against the float64
oracle (of some rows and columns, where the whole would be too much)."""
import math

import numpy as np
import pytest
import torch

import paper_2609_36662_amd as al
from oracle import block as ob
from tests.block_common import f64, product_error, within
from tests.test_gpu_gated_ff import BF, _check_backward, _check_forward, _inputs
from tests.test_gpu_muon import U32
from tests.test_gpu_muon_tiles import _bound
from tests.test_gpu_residual_norm import _check_backward as check_norm_grad, _check_forward as check_norm, _inputs as norm_inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    with al.autoloco_create(0) as c:
        yield c


class Far:
    """Matrices side by side in rows of a stride that takes the last of them beyond 2^32 bytes."""

    def __init__(self, rows, stride, dtype):
        self.buffer, self.rows, self.stride, self.at = torch.zeros(rows * stride, dtype=dtype, device="cuda"), rows, stride, 0

    def __call__(self, cols, values=None):
        t = self.buffer.as_strided((self.rows, cols), (self.stride, 1), self.at)
        self.at += -(-cols // 8) * 8 + 8
        return t if values is None else t.copy_(values)


@pytest.mark.parametrize("stride", [2_000_000, (1 << 22) - 8, (1 << 22), 2_000_003])
def test_gated_ff(ctx, stride):
    """Rows at strides up to and beyond the most that loads straight into LDS take, and an odd one."""
    rows, d, ffn, out = 1100, 136, 328, 200
    p = _inputs(rows, d, ffn, out)
    far = Far(rows, stride, BF)
    x, dy = far(d, p["x"]), far(out, p["dy"])
    y, h, gate, up, dgate, dup, dx = far(out), far(ffn), far(ffn), far(ffn), far(ffn), far(ffn), far(d)
    wg, wu, wd = (p[k].cuda() for k in ("wg", "wu", "wd"))
    dwg, dwu, dwd = torch.empty_like(wg), torch.empty_like(wu), torch.empty_like(wd)
    al.autoloco_gated_ff(ctx, x, wg, wu, wd, y, h, gate=gate, up=up)
    _check_forward(p, y, h, gate, up, "silu")
    al.autoloco_gated_ff_grad(ctx, x, wg, wu, wd, h, gate, up, dy, dgate, dup, dx=dx, dw_gate=dwg, dw_up=dwu, dw_down=dwd)
    _check_backward(p, h, gate, up, dgate, dup, dx, dwg, dwu, dwd, "silu", f64(gate), f64(up))


def test_gated_ff_more_tiles_than_a_launch(ctx):
    """h of 2^34 elements: 2^21 tiles of both projections and 2^20 of dh, in launches of 2^20 at most."""
    rows, d, ffn, out = (1 << 17) + 5, 8, (1 << 17) + 8, 8
    gen = torch.Generator(device="cuda").manual_seed(6)
    r = lambda rows, cols, std: torch.randn((rows, cols), generator=gen, device="cuda").mul_(std).to(BF)  # noqa: E731
    x, wg, wu, wd, dy = r(rows, d, 1), r(ffn, d, 0.5), r(ffn, d, 0.4), r(out, ffn, ffn ** -0.5), r(rows, out, 1)
    y, dx = torch.empty((rows, out), dtype=BF, device="cuda"), torch.empty((rows, d), dtype=BF, device="cuda")
    h, gate, up = (torch.empty((rows, ffn), dtype=BF, device="cuda") for _ in range(3))
    al.autoloco_gated_ff(ctx, x, wg, wu, wd, y, h, gate=gate, up=up)
    some = torch.tensor([0, 1, 127, 128, 255, 8191, 65535, 65536, 65537, 100_003, rows - 262, rows - 133, rows - 6, rows - 5, rows - 1],
                        device="cuda")
    part = {"x": x[some], "wg": wg, "wu": wu, "wd": wd, "dy": dy[some]}
    kept = {k: t[some] for k, t in (("h", h), ("gate", gate), ("up", up))}
    _check_forward(part, y[some], kept["h"], kept["gate"], kept["up"], "silu")
    dwg, dwu, dwd = (torch.empty(s, device="cuda") for s in ((ffn, d), (ffn, d), (out, ffn)))
    columns = torch.tensor([0, 1, 65_537, ffn - 9, ffn - 1], device="cuda")
    h_columns = h[:, columns]
    al.autoloco_gated_ff_grad(ctx, x, wg, wu, wd, h, gate, up, dy, gate, up, dx=dx, dw_gate=dwg, dw_up=dwu, dw_down=dwd)
    _check_backward(part, kept["h"], kept["gate"], kept["up"], gate[some], up[some], dx[some], None, None, None, "silu",
                    f64(kept["gate"]), f64(kept["up"]))
    for got, left, right in ((dwg[columns], gate[:, columns], x), (dwu[columns], up[:, columns], x), (dwd[:, columns].t(), h_columns, dy)):
        a, b = f64(left).T.copy(), f64(right).T.copy()
        within(got, a @ b.T, product_error(a, b), "dw")


@pytest.mark.parametrize("post,gate", [(True, "token"), (False, "channel")])
def test_norms(ctx, post, gate):
    rows, cols = 1100, 40
    p = norm_inputs(rows, cols, torch.float32, gate, post)
    far = Far(rows, 1_000_003, torch.float32)
    x, z, dy, dout = (far(cols, p[k]) for k in ("x", "z", "dy", "dout"))
    g = p["gate"].cuda().expand(rows, cols) if gate == "channel" else far(cols, p["gate"])
    out, y, dx, dz = far(cols), far(cols), far(cols), far(cols)
    dgate = torch.empty((1, cols), device="cuda") if gate == "channel" else far(cols)
    w, wz = p["weight"].cuda(), p["z_weight"].cuda() if post else None
    dw, dwz = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda") if post else None
    al.autoloco_residual_norm(ctx, x, w, y, z=z, out=out, gate=g, z_weight=wz)
    check_norm(p, out, y, 1.0, 1e-6)
    al.autoloco_residual_norm_grad(ctx, out, w, dy, dx, dw, torch.empty(al.residual_norm_work(rows, cols), device="cuda"), dout=dout, z=z,
                                   dz=dz, gate=g, dgate=dgate, z_weight=wz, dz_weight=dwz)
    check_norm_grad(p, out, {"dx": dx, "dz": dz, "dgate": dgate, "dweight": dw, "dz_weight": dwz}, 1.0, 1e-6, rows / 64 + 1)


@pytest.mark.parametrize("rows,cols,stride", [(1100, 300, 1_000_003), (1100, 300, 4_000_000), (300, 70, 8_000_001)])
def test_orthogonalised_step(ctx, rows, cols, stride):
    """Tensors whose rows lie far apart: the values of the same ones side by side, bit by bit."""
    gen = torch.Generator().manual_seed(8)
    w, m, g = (torch.randn((rows, cols), generator=gen) for _ in range(3))
    near = [t.cuda() for t in (w, m, g)]
    far = Far(rows, stride, torch.float32)
    apart = [far(cols, t) for t in (w, m, g)]
    k = al.make_muon_coeffs(lr=0.1, momentum=0.9)
    for t in (near, apart):
        ml = al.autoloco_muon_create(ctx, [t[0]], [t[1]], [t[2]])
        for _ in range(2):
            al.autoloco_inner_muon(ctx, ml, k)
        torch.cuda.synchronize()
        ml.close()
    assert torch.equal(near[0], apart[0]) and torch.equal(near[1], apart[1])


def test_orthogonalised_step_of_a_large_matrix(ctx):
    """A tensor and scratch memory of more than 2^32 bytes each."""
    rows, cols = 33_003, 33_100
    gen = torch.Generator(device="cuda").manual_seed(9)
    g = torch.randn((rows, cols), generator=gen, device="cuda")
    norm = math.sqrt(sum(torch.dot(r.double().view(-1), r.double().view(-1)).item() for r in g.split(2048)))
    scale = 0.2 * math.sqrt(cols)
    w, m = torch.zeros_like(g), torch.zeros_like(g)
    ml = al.autoloco_muon_create(ctx, [w], [m], [g])
    k = dict(lr=1.0, momentum=0.0, weight_decay=0.0)
    al.autoloco_inner_muon(ctx, ml, al.make_muon_coeffs(iterations=0, **k))
    for at in range(0, rows, 4096):
        x = g[at:at + 4096].double() / norm
        got = -w[at:at + 4096].double() / scale
        # two parts of 11 bits each, the second of at most half a step of the first (or 2^-25 over X's scale of 2^8)
        assert torch.all((got - x).abs() <= 2.0 ** -21 * x.abs() + 2.0 ** -33), at
    # two blocks in opposite corners, and nothing between: the step of both alone
    small = (torch.randn((200, 300), generator=gen, device="cuda"), torch.randn((303, 310), generator=gen, device="cuda"))
    for t in (w, m, g):
        t.zero_()
    g[:200, :300], g[-303:, -310:] = small
    al.autoloco_inner_muon(ctx, ml, al.make_muon_coeffs(iterations=1, **k))
    torch.cuda.synchronize()
    ml.close()
    both = np.zeros((503, 610))
    both[:200, :300], both[200:, 300:] = (f64(t) for t in small)
    ref = ob.orthogonalise(both, 1)
    err = _bound(both / (np.linalg.norm(both) + 1e-7), 2.0 ** 8)
    for got, at in ((w[:200, :300], np.s_[:200, :300]), (w[-303:, -310:], np.s_[200:, 300:])):
        assert np.all(np.abs(-f64(got) / scale - ref[at]) <= err[at] + 8 * U32 * np.abs(ref[at]))
    w[:200, :300] = 0
    w[-303:, -310:] = 0
    assert not any(t.any() for t in w.split(2048))
