"""A weight of so many rows that the single-token form's workgroups are more threads than a grid may have (2^32): its
rows, all quantised from one, give equal outputs to the last."""
import pytest
import torch

import paper_2609_36662_amd as al

pytestmark = pytest.mark.gpu


def test_single_tokens_through_more_rows_than_a_grid_has_threads():
    rows, cols = (1 << 23) * 48 + 1000, 5          # 48 rows a workgroup of 512 threads
    one = torch.tensor([[1.0, -2.0, 0.5, 3.0, -6.0]], dtype=torch.bfloat16, device="cuda")
    x = torch.tensor([[4.0, 1.0, -0.5, 2.0, 1.0]], dtype=torch.bfloat16, device="cuda")     # both are 4-bit values
    with al.autoloco_create(0) as ctx:
        w = al.Mxfp4.empty(rows, cols)
        al.autoloco_mxfp4_quantize(ctx, one.expand(rows, cols), w)
        y = torch.full((1, rows), 7.0, dtype=torch.bfloat16, device="cuda")
        al.autoloco_mxfp4_linear(ctx, x, w, y)
        torch.cuda.synchronize()
    want = float((one.double() * x.double()).sum())
    assert want == 1.75
    assert all(bool(torch.all(part == want)) for part in y[0].split(1 << 26))
