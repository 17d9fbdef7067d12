"""One pair of long sequences with short rows, whose loss and weights a kernel of their own takes between the rows' two:
rows of 4 to 16 KB and above, in both types, with logits as they are and far from 0 (the rows that are summed again), the
gradient beside the logits and in their place."""
import numpy as np
import pytest
import torch

import paper_2609_36662_amd as al
from oracle import preference as opref
from tests.test_gpu_preference import _check, _check_shifted, _inputs, _run, ctx  # noqa: F401

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.mark.parametrize("dtype,vocab", [("f32", 1100), ("f32", 4211), ("bf16", 2179), ("bf16", 8209)])
@pytest.mark.parametrize("shift", [0.0, -1e9])
def test_one_long_pair(ctx, dtype, vocab, shift):  # noqa: F811
    lens = [1500, 700]
    x, labels, off, ref = _inputs(lens, vocab, dtype, vocab)
    assert sum(lens) > 2048 and sum(lens) > vocab * (4 if dtype == "f32" else 2) / 16
    if shift:
        x = (x.float() + shift).to(DT[dtype])
        lp = opref.row_logps(x.double().numpy(), labels.numpy())[0]
        ref = torch.from_numpy(np.add.reduceat(lp, off.numpy()[:-1]).astype(np.float32))
    got = _run(ctx, x, labels, off, ref)
    if shift:
        _check_shifted(x, labels, off, ref, got, 0.1, dtype)
    else:
        _check(x, labels, off, ref, got, 0.1, 0.0, 1.0, dtype)
    there = _run(ctx, x.cuda(), labels, off, ref, grads="in place")
    assert all(torch.equal(a, b) for a, b in zip(got, there))


def test_one_long_pair_among_short_ones():
    """All but a few of the rows in one of 256 pairs take not much longer than the same rows in pairs of one length: the
    work does not grow with the square of the longest pair (measured: 1.2 times as long; where each row adds its own
    pair's rows up, 4.3 times)."""
    rows, vocab, pairs = 100_000, 4096, 256
    x = torch.randn((rows, vocab), dtype=torch.bfloat16, device="cuda")
    labels = torch.randint(0, vocab, (rows,), device="cuda")
    g = torch.empty_like(x)
    f = lambda n: torch.zeros(n, device="cuda")  # noqa: E731
    ref, losses, logps, work = f(2 * pairs), f(pairs), f(2 * pairs), f(2 * rows + 2 * pairs)
    even = [rows // (2 * pairs)] * (2 * pairs)
    skewed = [2] * (2 * pairs)
    skewed[3] = skewed[pairs + 3] = rows // 2 - 2 * pairs
    ms = {}
    with al.autoloco_create(0) as c:
        al.autoloco_set_timing(c, True)
        for name, lens in (("even", even), ("skewed", skewed)):
            off = torch.tensor(np.concatenate([[0], np.cumsum(lens)])).cuda()
            times = []
            for _ in range(6):
                al.autoloco_preference_loss(c, x, labels, off, ref, losses, logps, work, grads=g, beta=1e-6)
                torch.cuda.synchronize()
                times.append(al.autoloco_last_kernel_ms(c))
            ms[name] = min(times[1:])
    assert ms["skewed"] < 2.5 * ms["even"], ms


def test_rows_but_no_pairs():
    """Rows of no sequence, long and short ones: their gradient is zero."""
    with al.autoloco_create(0) as c:
        for rows, vocab, dtype in ((3, 40000, "bf16"), (600, 40000, "bf16"), (5, 3000, "f32"), (7, 11, "f32")):
            got = _run(c, torch.full((rows, vocab), float("nan"), dtype=DT[dtype]), torch.zeros(rows, dtype=torch.int64),
                       torch.zeros(1, dtype=torch.int64), torch.empty(0))
            assert not got[3].any()
