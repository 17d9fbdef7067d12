"""The gated feed-forward block in every tile and loop that its products take, against the float64 oracle: the shapes of
tests/block_shapes.py, whose tests say which path each is there for.  Outputs are windows of wider rows, so that a store
beyond a ragged tile's end shows; both directions are computed twice and give the same bits."""
import pytest
import torch

import paper_2609_36662_amd as al
from tests.block_common import f64, window
from tests.block_shapes import REGISTERS, TILES, TOKENS, TWO_TERMS
from tests.test_gpu_gated_ff import ACT, BF, _check_backward, _check_forward, _inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    with al.autoloco_create(0) as c:
        yield c


def _out(rows, cols, around, dtype=BF):
    return window(torch.full((rows, cols), float("nan"), dtype=dtype), around, around)


def _untouched(outs, around):
    for k, (win, whole) in outs.items():
        assert torch.all(whole[:, :around] == 7) and torch.all(whole[:, around + win.shape[1]:] == 7), k


def _forward(ctx, shape, name, around):
    rows, d, ffn, out = shape
    p = _inputs(rows, d, ffn, out)
    g = {k: v.cuda() for k, v in p.items()}
    runs = []
    for _ in range(2):
        o = {"y": _out(rows, out, around), "h": _out(rows, ffn, around), "gate": _out(rows, ffn, around), "up": _out(rows, ffn, around)}
        al.autoloco_gated_ff(ctx, g["x"], g["wg"], g["wu"], g["wd"], o["y"][0], o["h"][0], gate=o["gate"][0], up=o["up"][0],
                             activation=ACT[name])
        _untouched(o, around)
        runs.append({k: v[0] for k, v in o.items()})
    assert all(torch.equal(runs[0][k], runs[1][k]) for k in runs[0])
    o = runs[0]
    _check_forward(p, o["y"], o["h"], o["gate"], o["up"], name)
    # without gate and up: the same values
    y, h = _out(rows, out, around)[0], _out(rows, ffn, around)[0]
    al.autoloco_gated_ff(ctx, g["x"], g["wg"], g["wu"], g["wd"], y, h, activation=ACT[name])
    assert torch.equal(y, o["y"]) and torch.equal(h, o["h"])
    return p, g, o


def _backward(ctx, shape, name, around, p, g, o):
    rows, d, ffn, out = shape
    runs = []
    for dw in (BF, BF, torch.float32):
        q = {"dgate": _out(rows, ffn, around), "dup": _out(rows, ffn, around), "dx": _out(rows, d, around),
             "dw_gate": _out(ffn, d, around, dw), "dw_up": _out(ffn, d, around, dw), "dw_down": _out(out, ffn, around, dw)}
        w = {k: v[0] for k, v in q.items()}
        al.autoloco_gated_ff_grad(ctx, g["x"], g["wg"], g["wu"], g["wd"], o["h"], o["gate"], o["up"], g["dy"], w["dgate"], w["dup"],
                                  dx=w["dx"], dw_gate=w["dw_gate"], dw_up=w["dw_up"], dw_down=w["dw_down"], activation=ACT[name])
        _untouched(q, around)
        runs.append(w)
    assert all(torch.equal(runs[0][k], runs[1][k]) for k in runs[0])
    assert all(torch.equal(runs[0][k], runs[2][k].to(BF)) for k in runs[0])
    for w in (runs[0], runs[2]):
        _check_backward(p, o["h"], o["gate"], o["up"], w["dgate"], w["dup"], w["dx"], w["dw_gate"], w["dw_up"], w["dw_down"], name,
                        f64(o["gate"]), f64(o["up"]))


@pytest.mark.parametrize("shape", TILES + TWO_TERMS, ids=str)
def test_straight_into_lds(ctx, shape):
    """Aligned operands in both directions, windows whose rows are whole pieces too."""
    name = "gelu" if shape[0] * shape[2] < 200_000 else "silu"
    _backward(ctx, shape, name, 8, *_forward(ctx, shape, name, 8))


@pytest.mark.parametrize("shape", REGISTERS, ids=str)
def test_through_registers(ctx, shape):
    name = "gelu" if shape[0] * shape[2] < 200_000 else "silu"
    _backward(ctx, shape, name, 3, *_forward(ctx, shape, name, 3))


@pytest.mark.parametrize("shape", TOKENS, ids=str)
@pytest.mark.parametrize("name", ["silu", "gelu"])
def test_tokens(ctx, shape, name):
    _forward(ctx, shape, name, 3)
