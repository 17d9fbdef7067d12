"""The norms' gradients where a team of waves goes from row to row, for every number of waves and runs a row can take,
against the float64 oracle: the sums over rows are kept in registers over a team's rows, joined over the teams' and the
workgroups' parts, and the next row is fetched while one is worked on."""
import pytest
import torch

import paper_2609_36662_amd as al
from tests.block_common import DT
from tests.test_gpu_residual_norm import _backward, _check_backward, _check_forward, _gpu, _inputs

pytestmark = pytest.mark.gpu

# rows, cols, workgroups at most and teams of a workgroup: 1, 2, 4, 8 and 16 waves a row with one run a lane, 8 and 16 with
# four.  Rows that leave some teams one more than others, and rows that do not.
SHAPES = [(5003, 500, 512, 4), (4096, 512, 512, 4), (2500, 1001, 1024, 1), (3001, 1024, 1024, 1), (1301, 2047, 512, 1),
          (1024, 2048, 512, 1), (700, 4095, 256, 1), (768, 4096, 256, 1), (601, 8191, 256, 1), (515, 8200, 256, 1), (513, 16384, 256, 1),
          (300, 16401, 256, 1), (517, 20001, 256, 1)]


@pytest.fixture(scope="module")
def ctx():
    with al.autoloco_create(0) as c:
        yield c


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,cols,most,teams", SHAPES)
@pytest.mark.parametrize("gate,post", [("channel", True), ("token", True), ("none", False)])
def test_rows_of_a_team(ctx, rows, cols, most, teams, dtype, gate, post):
    dt, scale, eps = DT[dtype], 0.5, 1e-6
    p = _inputs(rows, cols, dt, gate, post)
    g = _gpu(p)
    out, y = torch.full_like(g["x"], float("nan")), torch.full_like(g["x"], float("nan"))
    al.autoloco_residual_norm(ctx, g["x"], g["weight"], y, z=g["z"], out=out, gate=g["gate"], z_weight=g["z_weight"], scale=scale, eps=eps)
    _check_forward(p, out, y, scale, eps)
    got = _backward(ctx, g, out, dt, scale, eps)
    # a team's rows one after another, then the teams of a workgroup in fp32 (the workgroups' parts are added in fp64)
    _check_backward(p, out, got, scale, eps, -(-rows // (min(most, max(256, rows // teams // 2)) * teams)) + teams)
    again = _backward(ctx, g, out, dt, scale, eps)
    assert all(torch.equal(again[k], got[k]) for k in got)
