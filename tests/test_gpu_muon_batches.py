"""Lists of the orthogonalised step whose matrices do not fit one pass: batches share the scratch memory, one after
another.  Matrices whose sizes differ lie on both sides of each border; every one is compared, bit by bit, with a list of
its own, and small ones in every batch with the oracle."""
import math

import numpy as np
import pytest
import torch

import paper_2609_36662_amd as al
from oracle import block as ob
from tests.block_common import f64
from tests.test_gpu_muon import U16, U32, _keep

pytestmark = pytest.mark.gpu
LIMIT = 4 << 30     # of the scratch memory of lists whose matrices each take less
LARGE = [(8100, 8190), (8190, 7001), (6003, 9100)]


def _need(shape):
    """X in three parts and two products, rows and columns in whole steps of 64, and the norm's partial sums."""
    m, n = (-(-s // 64) * 64 for s in sorted(shape))
    return 3 * m * n * 2 + 2 * m * m * 2 + 2048


def _batches(shapes):
    at, taken = [], LIMIT + 1
    for i, s in enumerate(shapes):
        if taken + _need(s) > LIMIT:
            at.append([])
            taken = 0
        taken += _need(s)
        at[-1].append(i)
    return at


def _shapes():
    small = [(97, 260), (130, 33), (64, 700), (513, 129), (1, 77), (300, 200), (65, 63), (200, 520)]
    shapes, k = [], 0
    for i in range(21):
        shapes.append(LARGE[i % len(LARGE)])
        if i % 3 == 2:
            shapes.append(small[k])
            k += 1
    return shapes


def test_more_than_one_batch():
    """(What the test below relies on.)"""
    at = _batches(_shapes())
    assert len(at) >= 3 and all(any(max(_shapes()[i]) < 1000 for i in b) for b in at), at


@pytest.mark.parametrize("steps", [2])
def test_each_as_it_is_alone(steps):
    shapes = _shapes()
    gen = torch.Generator(device="cuda").manual_seed(4)
    normal = lambda s, std: torch.randn(s, generator=gen, device="cuda").mul_(std)  # noqa: E731
    w, m, g = ([normal(s, std) for s in shapes] for std in (0.02, 1e-3, 1e-3))
    alone = [[t.clone() for t in ts] for ts in (w, m)]
    first = [[f64(w[i]), f64(m[i])] for i in range(len(shapes)) if max(shapes[i]) < 1000]
    k = al.make_muon_coeffs(lr=0.01, momentum=0.9, weight_decay=0.1, iterations=2)
    with al.autoloco_create(0) as ctx:
        torch.cuda.synchronize()
        free = torch.cuda.mem_get_info()[0]
        ml = al.autoloco_muon_create(ctx, w, m, g)
        taken = free - torch.cuda.mem_get_info()[0]
        total = sum(_need(s) for s in shapes)
        # scratch for the largest batch only, and the tables
        assert taken <= LIMIT + (64 << 20) < total, (taken, total)
        for _ in range(steps):
            al.autoloco_inner_muon(ctx, ml, k)
        torch.cuda.synchronize()
        ml.close()
        for i, s in enumerate(shapes):
            one = al.autoloco_muon_create(ctx, [alone[0][i]], [alone[1][i]], [g[i]])
            for _ in range(steps):
                al.autoloco_inner_muon(ctx, one, k)
            torch.cuda.synchronize()
            one.close()
            assert torch.equal(w[i], alone[0][i]) and torch.equal(m[i], alone[1][i]), (i, s)
    at = 0
    for i, s in enumerate(shapes):
        if max(s) >= 1000:
            continue
        rw, rm = first[at]
        at += 1
        off = 0.0
        for _ in range(steps):
            u = (rm * 0.9 + f64(g[i])) * 0.9 + f64(g[i])
            x, rounded = ob.orthogonalise(u, 2), ob.orthogonalise(u, 2, keep=_keep(max(s)))
            off += 0.01 * 0.2 * math.sqrt(max(s)) * (2 * np.linalg.norm(rounded - x) + 2 * U16 * np.linalg.norm(x))
            # U, rounded some six times, moves X's direction by twice that, and two iterations that by 3.45 each
            off += 0.01 * 0.2 * math.sqrt(max(s)) * 144 * U32 + 4 * U32 * np.linalg.norm(rw)
            rw, rm = ob.muon_step(rw, rm, f64(g[i]), 0.01, mu=0.9, weight_decay=0.1, iterations=2)
            off += 4 * U32 * np.linalg.norm(rw)
        assert np.linalg.norm(f64(w[i]) - rw) <= off, (i, s)
