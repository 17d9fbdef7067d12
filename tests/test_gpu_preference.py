"""The preference loss and the sequences' log-probabilities on the GPU against the
float64 oracle, their gradient also against difference quotients, and refusals.

Tolerances.  A row's log sum exp: its sum of up to V positive terms is added up in fp32
in chains of at most 8 ceil(V / 2048) per lane and a tree above, each term within a few
ulps, so its relative error is at most e = (8 ceil(V / 2048) + 16) 2^-24, and the stored
value is rounded (2^-24 |lse|).  A log-probability adds the label's logit: 2^-24 of it.
Their sum over a sequence is in fp64, rounded once.  The loss has slope at most |beta| in
either sequence's log-probability; the weight at most |scale| beta^2 / 4.  A
probability's relative error: the exponent's rounding, 2^-22 (|x| + |lse|), and e."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2609_36662_amd as al
from oracle import preference as opref

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def ctx():
    with al.autoloco_create(0) as c:
        yield c


def _inputs(lens, vocab, dtype, seed, mask=0.3):
    rng = np.random.default_rng(seed)
    rows = sum(lens)
    x = rng.normal(0, 2, (rows, vocab))
    labels = rng.integers(0, vocab, rows)
    x[np.arange(rows), labels] += np.log(vocab)
    labels[rng.random(rows) < mask] = -100
    off = np.concatenate([[0], np.cumsum(lens)])
    x = torch.from_numpy(x.astype(np.float32)).to(DT[dtype])
    lp, _ = opref.row_logps(x.double().numpy(), labels)
    ref = np.array([lp[a:b].sum() for a, b in zip(off, off[1:])]) + rng.normal(0, 4, len(lens))
    return x, torch.from_numpy(labels), torch.from_numpy(off), torch.from_numpy(ref.astype(np.float32))


def _run(ctx, x, labels, off, ref, grads="new", beta=0.1, smoothing=0.0, scale=1.0):
    rows, vocab = x.shape
    seqs = off.numel() - 1
    d = x if x.is_cuda else x.cuda()
    losses, logps = torch.full((seqs // 2,), 9.0, device="cuda"), torch.full((seqs,), 9.0, device="cuda")
    work = torch.full((2 * rows + seqs,), 9.0, device="cuda")
    g = None if grads is None else d if grads == "in place" else torch.full((rows, vocab), 9.0, dtype=x.dtype, device="cuda") \
        if isinstance(grads, str) else grads
    al.autoloco_preference_loss(ctx, d, labels.cuda(), off.cuda(), ref.cuda(), losses, logps, work, grads=g, beta=beta,
                                label_smoothing=smoothing, grad_scale=scale)
    torch.cuda.synchronize()
    return losses, logps, work, g


def _row_tol(x, lse, labels):
    vocab = x.shape[1]
    e = (8 * -(-vocab // 2048) + 16) * 2.0 ** -24
    lab = np.abs(x[np.arange(len(labels)), np.clip(labels, 0, vocab - 1)])
    return np.where((labels >= 0) & (labels < vocab), e + 2.0 ** -23 * (np.abs(lse) + lab), 0.0)


def _check(x, labels, off, ref, got, beta, smoothing, scale, dtype):
    x, labels, off = x.double().cpu().numpy(), labels.numpy(), off.numpy()
    losses, logps, g, w, lse = opref.preference(x, labels, off, ref.numpy(), beta, smoothing, scale)
    row_tol = _row_tol(x, lse, labels)
    seq_tol = np.array([row_tol[a:b].sum() for a, b in zip(off, off[1:])])
    seqs, p = len(logps), len(losses)
    np.testing.assert_array_less(np.abs(got[1].double().cpu().numpy() - logps), seq_tol + 2.0 ** -24 * np.abs(logps) + 1e-30)
    z_tol = abs(beta) * (seq_tol[:p] + seq_tol[p:])
    np.testing.assert_array_less(np.abs(got[0].double().cpu().numpy() - losses), z_tol + 2.0 ** -23 * np.abs(losses) + 1e-30)
    work = got[2].double().cpu().numpy()
    rows = len(labels)
    assert np.all(np.abs(work[:rows] - lse) <= row_tol) and work.shape[0] == 2 * rows + seqs
    w_tol = np.concatenate([abs(scale * beta) * z_tol / 4] * 2) + 2.0 ** -23 * np.abs(w)
    if got[3] is None:
        return
    e = (8 * -(-x.shape[1] // 2048) + 16) * 2.0 ** -24
    out = 2.0 ** -23 if dtype == "f32" else 2.0 ** -8
    gg = got[3].double().cpu().numpy()
    for s in range(seqs):
        for r in range(off[s], off[s + 1]):
            if not 0 <= labels[r] < x.shape[1]:
                assert not gg[r].any()
                continue
            prob = np.exp(x[r] - lse[r])
            tol = abs(w[s]) * (prob * (2.0 ** -22 * (np.abs(x[r]) + abs(lse[r])) + 2 * e) + 2.0 ** -23 * (prob + (np.arange(len(prob)) == labels[r]))) \
                + w_tol[s] + out * np.abs(g[r]) + 1e-38
            assert np.all(np.abs(gg[r] - g[r]) <= tol), (r, np.abs(gg[r] - g[r]).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,vocab", [([1, 1], 1), ([1, 1], 2), ([3, 2], 7), ([1, 4], 8), ([2, 3, 4, 1], 64), ([5, 0, 0, 3], 65),
                                        ([0, 0], 9), ([7, 9], 1023), ([4, 4], 2048), ([3, 5], 2049), ([2, 2], 32000),
                                        ([1, 2], 50257), ([40, 1, 33, 12, 0, 25], 515), ([300, 280], 130)])
def test_loss_and_gradient(ctx, lens, vocab, dtype):
    t = _inputs(lens, vocab, dtype, vocab + len(lens))
    for smoothing, scale in ((0.0, 1.0), (0.1, 0.25)):
        got = _run(ctx, *t, smoothing=smoothing, scale=scale)
        _check(*t, got, 0.1, smoothing, scale, dtype)
    again = _run(ctx, *t, smoothing=0.1, scale=0.25)
    assert all(torch.equal(a, b) for a, b in zip(got, again))
    there = t[0].cuda()
    inplace = _run(ctx, there, *t[1:], grads="in place", smoothing=0.1, scale=0.25)
    assert torch.equal(inplace[3], got[3]) and torch.equal(there, got[3]) and torch.equal(inplace[0], got[0])
    plain = _run(ctx, *t, grads=None, smoothing=0.1, scale=0.25)
    assert torch.equal(plain[0], got[0]) and torch.equal(plain[1], got[1])
    logps, work = torch.empty(len(lens), device="cuda"), torch.empty(2 * sum(lens) + len(lens), device="cuda")
    al.autoloco_sequence_logps(ctx, t[0].cuda(), t[1].cuda(), t[2].cuda(), logps, work)
    assert torch.equal(logps, got[1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_many_rows(ctx, dtype):
    """More rows and pairs than a launch has workgroups in flight; lengths of all kinds."""
    rng = np.random.default_rng(8)
    lens = [int(n) for n in rng.integers(0, 160, 64)]
    t = _inputs(lens, 61, dtype, 4)
    _check(*t, _run(ctx, *t, smoothing=0.05, scale=1 / 32), 0.1, 0.05, 1 / 32, dtype)


@pytest.mark.parametrize("smoothing", [0.0, 0.3, 1.0])
def test_gradient_against_differences(ctx, smoothing):
    """Difference quotients of the oracle's loss at the same logits; the quotient's own error is about 1e-9."""
    x, labels, off, ref = _inputs([3, 4, 2, 5], 33, "f32", 12, mask=0.2)
    g = _run(ctx, x, labels, off, ref, beta=0.5, smoothing=smoothing, scale=0.5)[3].cpu().numpy()
    h, base = 1e-4, x.double().numpy()
    rng = np.random.default_rng(1)
    for r, v in [(int(a), int(b)) for a, b in zip(rng.integers(0, 14, 40), rng.integers(0, 33, 40))] + [(r, max(0, int(labels[r]))) for r in range(14)]:
        d = []
        for s in (h, -h):
            y = base.copy()
            y[r, v] += s
            d.append(opref.preference(y, labels.numpy(), off.numpy(), ref.numpy(), 0.5, smoothing, 0.5)[0].sum())
        assert abs(0.5 * (d[0] - d[1]) / (2 * h) - g[r, v]) <= 1e-8 + 1e-5 * abs(g[r, v])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_strides_and_odd_addresses(ctx, dtype):
    lens, vocab = [6, 5], 301
    x, labels, off, ref = _inputs(lens, vocab, dtype, 2)
    big = torch.zeros((11, 330), dtype=DT[dtype], device="cuda")
    big[:, 3:304] = x.cuda()
    out = torch.full((13, 311), 7.0, dtype=DT[dtype], device="cuda")
    got = _run(ctx, big[:, 3:304], labels, off, ref, grads=out[1:12, 5:306])
    _check(x, labels, off, ref, got, 0.1, 0.0, 1.0, dtype)
    inside = torch.zeros_like(out, dtype=torch.bool)
    inside[1:12, 5:306] = True
    assert torch.all(out[~inside] == 7.0)
    got2 = _run(ctx, big[:, 3:304], labels, off, ref, grads="in place")
    assert torch.equal(got2[3], got[3]) and not big[:, :3].any() and not big[:, 304:].any()


def test_masked_rows_are_not_read(ctx):
    """Rows masked by their label (any outside the vocabulary) or of no sequence may hold anything."""
    x, labels, off, ref = _inputs([4, 5], 40, "f32", 6, mask=0.0)
    labels[1], labels[5], labels[6], labels[7] = -1, 40, -(1 << 40), 1 << 40
    clean = _run(ctx, x, labels, off, ref)
    dirty = x.clone()
    for r, v in ((1, float("nan")), (5, float("inf")), (6, float("-inf")), (7, torch.finfo(torch.float32).min)):
        dirty[r] = v
    got = _run(ctx, dirty, labels, off, ref)
    assert all(torch.equal(a, b) for a, b in zip(clean, got))
    _check(x, labels, off, ref, got, 0.1, 0.0, 1.0, "f32")
    part = torch.tensor([2, 4, 8])     # rows 0, 1 and 8 are of no sequence
    dirty = x.clone()
    dirty[0] = float("nan")
    dirty[8] = float("nan")
    labels = torch.arange(9)
    got = _run(ctx, dirty, labels, part, ref)
    x[0], x[8] = 0.0, 0.0
    only = labels.clone()
    only[:2], only[8] = -1, -1
    want = opref.preference(x.double().numpy(), only.numpy(), part.numpy(), ref.numpy(), 0.1, 0.0, 1.0)
    np.testing.assert_allclose(got[1].cpu().numpy(), want[1], rtol=1e-5)
    np.testing.assert_allclose(got[3].cpu().numpy(), want[2], rtol=1e-4, atol=1e-7)
    assert not got[3][[0, 1, 8]].any()


def test_offsets_beyond_the_rows_count_as_their_ends(ctx):
    x, labels, _, ref = _inputs([4, 5], 40, "f32", 6, mask=0.0)
    got = _run(ctx, x, labels, torch.tensor([-5, 4, 1 << 50]), ref)
    want = _run(ctx, x, labels, torch.tensor([0, 4, 9]), ref)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_infinite_and_nan_logits(ctx, dtype):
    """-inf has probability 0 (also the type's lowest value beside others); a label at -inf makes the loss infinite or
    zero's limit; NaN, +inf or nothing but -inf make their pair NaN and no other."""
    x, labels, off, ref = _inputs([2, 2, 2, 2, 2, 2, 2, 2], 50, dtype, 3, mask=0.0)
    for r in range(16):   # pair p: rows 2p, 2p+1 and 2(p+4), 2(p+4)+1
        x[r, int(labels[r]) - 3] = float("-inf")
        x[r, int(labels[r]) - 4] = torch.finfo(DT[dtype]).min
    x[2, 7 if int(labels[2]) != 7 else 8] = float("nan")      # pair 1
    x[13, :] = float("-inf")                                   # pair 2, its rejected side
    x[6, 9] = float("inf")                                     # pair 3
    losses, logps, work, g = _run(ctx, x, labels, off, ref)
    assert torch.isnan(losses).tolist() == [False, True, True, True]
    assert torch.isnan(g).any(1).tolist() == [r // 2 % 4 != 0 for r in range(16)]
    keep = [0, 1, 8, 9]
    sub = _run(ctx, x[keep], labels[keep], torch.tensor([0, 2, 4]), ref[[0, 4]])
    assert torch.equal(sub[3], g[keep]) and torch.equal(sub[0], losses[:1])
    assert all(float(g[r, int(labels[r]) - 3]) == 0 for r in keep)
    want = opref.preference(x[keep].double().numpy(), labels[keep].numpy(), [0, 2, 4], ref[[0, 4]].numpy(), 0.1, 0.0, 1.0)
    np.testing.assert_allclose(g[keep].double().cpu().numpy(), want[2], rtol=2.0 ** -7, atol=1e-7)
    # a chosen label of probability 0: loss +inf and the full weight; a rejected one: loss 0 and no weight
    x, labels, off, ref = _inputs([1, 1, 1, 1], 50, dtype, 5, mask=0.0)
    x[0, labels[0]] = float("-inf")
    x[3, labels[3]] = float("-inf")
    losses, logps, work, g = _run(ctx, x, labels, off, ref)
    assert losses.tolist() == [float("inf"), 0.0] and torch.isinf(logps).tolist() == [True, False, False, True]
    assert work[-4:].tolist() == pytest.approx([-0.1, 0.0, 0.1, 0.0]) and torch.isfinite(g).all()


def test_large_logits(ctx):
    """No overflow: logits of +-3e4 and equal maxima."""
    x, labels, off, ref = _inputs([2, 3], 60, "f32", 9, mask=0.0)
    x = x * 1000
    x[:, :2] = 3e4
    got = _run(ctx, x, labels, off, ref, beta=1e-4)
    _check(x, labels, off, ref, got, 1e-4, 0.0, 1.0, "f32")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [7, 50, 3001])
def test_logits_at_the_ends_of_the_type(ctx, vocab, dtype):
    """Rows of the type's lowest value are uniform; its highest value has all the probability; one finite logit among
    -inf has probability 1; the lowest value beside ordinary ones has none, wherever it stands."""
    lo, hi, inf = torch.finfo(DT[dtype]).min, torch.finfo(DT[dtype]).max, float("inf")
    x, labels, off, ref = _inputs([3, 3], vocab, dtype, 11, mask=0.0)
    x[0] = lo
    x[1] = 0.0
    x[1, 3] = hi
    x[2] = -inf
    x[2, 4] = 1.5
    labels[1], labels[2] = 3, 4
    x[4] = lo
    x[4, 5] = 2.0
    labels[4] = 5
    x[5, ::2] = lo
    labels[5] = 1
    losses, logps, work, g = _run(ctx, x, labels, off, torch.zeros(2))
    assert work[6].item() == pytest.approx(-np.log(vocab), rel=1e-6)
    assert work[[7, 8, 10]].tolist() == [0.0, 0.0, 0.0]
    w = work[-2:].tolist()
    assert torch.isfinite(losses).all() and torch.isfinite(g).all()
    flat = torch.full((vocab,), -w[0] / vocab)
    flat[int(labels[0])] += w[0]
    assert torch.allclose(g[0].float().cpu(), flat, rtol=2.0 ** -7, atol=1e-9)
    assert not g[[1, 2, 4]].any() and not g[5, ::2].any()
    want = opref.row_logps(x[5:6].double().numpy(), labels[5:6].numpy())[0]
    assert work[11].item() == pytest.approx(float(want[0]), rel=1e-5)


def test_offsets_past_32_bits(ctx):
    """Rows that begin beyond 2^32 elements of the matrix."""
    vocab, stride, rows = 40, (1 << 32) // 5 + 1, 8
    store = torch.empty(stride * (rows - 1) + vocab, dtype=torch.bfloat16, device="cuda")
    x, labels, off, ref = _inputs([3, 5], vocab, "bf16", 7, mask=0.1)
    view = torch.as_strided(store, (rows, vocab), (stride, 1))
    view.copy_(x)
    got = _run(ctx, view, labels, off, ref, grads="in place")
    _check(x, labels, off, ref, got, 0.1, 0.0, 1.0, "bf16")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens,vocab", [([400, 250], 8209), ([300, 0, 220, 170], 3001)])
def test_many_long_rows(ctx, lens, vocab, dtype):
    """More than 512 rows of more than 16 KB, and of 4 to 16 KB."""
    t = _inputs(lens, vocab, dtype, 21)
    _check(*t, _run(ctx, *t, smoothing=0.1), 0.1, 0.1, 1.0, dtype)


def test_more_rows_than_one_launch(ctx):
    """A million and a half rows, one row of logits broadcast."""
    n, vocab = 1_500_000, 3
    x = torch.tensor([[0.5, -1.0, 2.0]], device="cuda").expand(n, vocab)
    labels = torch.zeros(n, dtype=torch.int64)
    off, ref = torch.tensor([0, 700_000, n]), torch.tensor([0.0, 0.0])
    g = torch.full((n, vocab), 9.0, device="cuda")
    losses, logps, work, _ = _run(ctx, x, labels, off, ref, grads=g, beta=1e-7)
    v = np.array([0.5, -1.0, 2.0])
    lse = np.log(np.exp(v).sum())
    z = 1e-7 * (0.5 - lse) * (700_000 - 800_000)
    assert logps.tolist() == pytest.approx([(0.5 - lse) * 700_000, (0.5 - lse) * 800_000], rel=1e-6)
    assert float(losses[0]) == pytest.approx(np.log1p(np.exp(-z)), rel=1e-6)
    w = 1e-7 * (1 / (1 + np.exp(-z)) - 1)
    want = w * ((np.arange(3) == 0) - np.exp(v - lse))
    for a, b, s in ((0, 700_000, 1), (700_000, n, -1)):
        assert torch.equal(g[a:b], g[a:a + 1].expand(b - a, vocab))
        np.testing.assert_allclose(g[a].cpu().numpy(), s * want, rtol=1e-5)


def test_no_rows_and_no_pairs(ctx):
    e = torch.empty
    got = _run(ctx, e(0, 10), e(0, dtype=torch.int64), torch.zeros(3, dtype=torch.int64), torch.tensor([1.0, 2.0]), beta=0.5)
    assert got[0].item() == pytest.approx(np.log1p(np.exp(-0.5)), rel=1e-6) and got[1].tolist() == [0, 0]
    g = _run(ctx, torch.ones(3, 10), torch.zeros(3, dtype=torch.int64), torch.zeros(1, dtype=torch.int64), e(0))[3]
    assert not g.any()


def test_refusals(ctx):
    x, labels, off, ref = _inputs([3, 4], 30, "f32", 1)
    x, labels, off, ref = x.cuda(), labels.cuda(), off.cuda(), ref.cuda()
    f = lambda n: torch.zeros(n, device="cuda")  # noqa: E731

    def refused(status, **kw):
        a = dict(logits=x, labels=labels, offsets=off, ref_logps=ref, losses=f(1), logps=f(2), work=f(16), grads=None)
        a.update(kw)
        with pytest.raises(al.AutolocoError) as ex:
            al.autoloco_preference_loss(ctx, **a)
        assert ex.value.status == status, ex.value

    refused(-1, offsets=off[:2])                       # one sequence
    refused(-1, beta=float("nan"))
    refused(-1, grad_scale=float("inf"))
    refused(-1, label_smoothing=1.5)
    refused(-1, label_smoothing=float("nan"))
    refused(-1, grads=torch.empty((7, 31), device="cuda"))
    refused(-1, grads=torch.empty((7, 30), dtype=torch.bfloat16, device="cuda"))
    refused(-1, grads=torch.as_strided(f(400), (7, 30), (20, 1)))
    room = f(7 * 30 + 16)
    refused(-3, logits=torch.as_strided(room, (7, 30), (30, 1)), grads=torch.as_strided(room, (7, 30), (30, 1), 4))
    refused(-3, logits=torch.as_strided(room, (7, 30), (30, 1)), grads=torch.as_strided(room, (7, 30), (31, 1)))
    both = f(20)
    refused(-3, losses=both[1:2], logps=both[:2])
    refused(-3, work=both[:16], logps=both[15:17])
    host = torch.zeros(2).pin_memory()
    s = al.make_sequences(x, labels, off, f(16))
    lib = al.lib()
    assert lib.autoloco_sequence_logps(ctx.handle, C.byref(s), host.data_ptr()) == -1
    assert lib.autoloco_sequence_logps(ctx.handle, C.byref(s), None) == -1
    assert lib.autoloco_sequence_logps(ctx.handle, None, ref.data_ptr()) == -1
    assert lib.autoloco_sequence_logps(None, C.byref(s), ref.data_ptr()) == -1
    assert lib.autoloco_preference_loss(ctx.handle, C.byref(s), None) == -1
    s.sequences = -1
    assert lib.autoloco_sequence_logps(ctx.handle, C.byref(s), ref.data_ptr()) == -1
    s = al.make_sequences(x, labels, off, f(16))
    s.labels += 4
    assert lib.autoloco_sequence_logps(ctx.handle, C.byref(s), ref.data_ptr()) == -2
    with pytest.raises(TypeError):
        al.make_sequences(x, labels.int(), off, f(16))
    with pytest.raises(ValueError):
        al.make_sequences(x, labels[:5], off, f(16))
    with pytest.raises(ValueError):
        al.make_sequences(x, labels, off, f(15))



def _check_shifted(x, labels, off, ref, got, beta, dtype):
    """As _check, with tolerances that do not grow with what a row's logits have in common.

    An exponential's exponent is rounded by 2^-24 of its own size, which, weighted by the
    probabilities, is at most 2^-24 (ln V + 1) for the whole sum, and the instruction by 2^-23.  The gradient
    takes the normaliser from numbers of at most 64 rounded to fp32, or adds it up again."""
    x, labels, off = x.double().cpu().numpy(), labels.numpy(), off.numpy()
    losses, logps, g, w, lse = opref.preference(x, labels, off, ref.numpy(), beta, 0.0, 1.0)
    lp, _ = opref.row_logps(x, labels)
    vocab, p = x.shape[1], len(losses)
    e = (8 * -(-vocab // 2048) + 16) * 2.0 ** -24 + 2.0 ** -22 * (np.log(vocab) + 2)
    row_tol = np.where((labels >= 0) & (labels < vocab), e + 2.0 ** -22 * np.abs(lp), 0.0)
    seq_tol = np.array([row_tol[a:b].sum() for a, b in zip(off, off[1:])])
    work = got[2].double().cpu().numpy()
    rows = len(labels)
    assert np.all(np.abs(work[rows:2 * rows] - lp) <= row_tol), np.abs(work[rows:2 * rows] - lp).max()
    assert np.all(work[rows:2 * rows] <= 0)
    np.testing.assert_array_less(np.abs(got[1].double().cpu().numpy() - logps), seq_tol + 2.0 ** -24 * np.abs(logps) + 1e-30)
    z_tol = abs(beta) * (seq_tol[:p] + seq_tol[p:])
    np.testing.assert_array_less(np.abs(got[0].double().cpu().numpy() - losses), z_tol + 2.0 ** -23 * np.abs(losses) + 1e-30)
    w_tol = np.concatenate([abs(beta) * z_tol / 4] * 2) + 2.0 ** -23 * np.abs(w)
    out = 2.0 ** -23 if dtype == "f32" else 2.0 ** -8
    gg = got[3].double().cpu().numpy()
    for s in range(len(logps)):
        for r in range(off[s], off[s + 1]):
            if not 0 <= labels[r] < vocab:
                assert not gg[r].any()
                continue
            d = (x[r] - x[r, labels[r]]) + lp[r]
            prob = np.exp(d)
            rel = 2 * e + 2.0 ** -22 * (np.abs(d) + min(abs(lse[r]), abs(lp[r]), 64.0) + 2)
            tol = abs(w[s]) * (prob * rel + 2.0 ** -23 * (np.arange(vocab) == labels[r])) + w_tol[s] + out * np.abs(g[r]) + 1e-38
            assert np.all(np.abs(gg[r] - g[r]) <= tol), (r, np.abs(gg[r] - g[r]).max())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [5, 301, 2051, 8209])
@pytest.mark.parametrize("shift", [100.0, -3000.0, 5e4, -1.1e7, 1.3e7, -1e9, 3e10, -1e20, 2e37])
def test_what_all_logits_of_a_row_have_in_common(ctx, shift, vocab, dtype):
    """A shift of all of a row's logits changes neither probabilities nor gradients, however large (also a whole row
    of an additive mask's -1e9); a label far below the rest of such a row has its log-probability."""
    x, labels, off, ref = _inputs([3, 4, 5, 2], vocab, dtype, 31, mask=0.0)
    x = (x.float() + shift).to(DT[dtype])
    x[0] = shift                                       # nothing but the shift
    x[4, int(labels[4])] = shift - 1000.0              # an improbable label
    x[9, int(labels[9])] = shift + 30.0                # a nearly certain one
    labels[6] = -1
    ref = torch.from_numpy(np.add.reduceat(opref.row_logps(x.double().numpy(), labels.numpy())[0], off.numpy()[:-1]).astype(np.float32))
    got = _run(ctx, x, labels, off, ref)
    _check_shifted(x, labels, off, ref, got, 0.1, dtype)
    there = _run(ctx, x.cuda(), labels, off, ref, grads="in place")
    assert torch.equal(there[3], got[3])


@pytest.mark.parametrize("lens", [[5, 3, 0, 7], [700, 600, 650, 630]], ids=["pairs in the gradient's kernel", "pairs apart"])
def test_graph_replays(lens):
    """Captured into a graph and replayed on new logits, with eager work between, every replay gives the eager result."""
    x, labels, off, ref = _inputs(lens, 200, "f32", 17)
    stream = torch.cuda.Stream()
    with al.autoloco_create(0, stream) as c, torch.cuda.stream(stream):
        d = [t.cuda() for t in (x, labels, off, ref)]
        losses, logps = torch.zeros(2, device="cuda"), torch.zeros(4, device="cuda")
        work, g = torch.zeros(2 * sum(lens) + 4, device="cuda"), torch.zeros_like(d[0])

        def call():
            al.autoloco_preference_loss(c, *d, losses, logps, work, grads=g, label_smoothing=0.1)

        call()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            call()
        for turn in range(3):
            d[0].copy_(x * (turn + 1))
            call()
            want = [t.clone() for t in (losses, logps, g)]
            for t in (losses, logps, work, g):
                t.fill_(9.0)
            graph.replay()
            stream.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, (losses, logps, g)))
