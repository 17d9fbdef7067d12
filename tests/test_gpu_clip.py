"""Global norms over many tensors, clipping and packing on the GPU against the float64 oracle, and refusals.

Tolerances.  Squares are added in fp32 within 8 values (relative error at most 8 2^-24) and in fp64 beyond, so a norm's is
at most 4 2^-24, and 2^-24 more as a stored fp32; the coefficient's the same; a clipped value is rounded to fp32 (the
coefficient and the product: 2 2^-24) and, in place, to its type (2^-8 bf16)."""
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


def _views(sizes, dtype, norm, seed, gap=0):
    """Tensors of these sizes, back to back (gap elements between) in one buffer, so that they begin at any element."""
    g = torch.Generator().manual_seed(seed)
    n = sum(sizes) + gap * len(sizes)
    flat = torch.randn(n, generator=g) * (norm / max(1, n) ** 0.5)
    flat = flat.to(DT[dtype]).cuda()
    out, at = [], 0
    for s in sizes:
        out.append(flat[at:at + s])
        at += s + gap
    return flat, out


SIZES = [[1], [7], [8, 8], [1, 2, 3, 5, 7, 9, 0, 11], [4096], [16384, 16384], [16385, 1, 16383, 3], [100003, 0, 1, 64, 17, 50000],
         [0], [33] * 300, [300001]]


@pytest.mark.parametrize("mode", ["packed", "in place"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "-".join(map(str, s[:4])))
def test_clip(ctx, sizes, dtype, mode):
    norms_in = (4.0, 0.5, 1.5)
    made = [_views(sizes if k != 1 else sizes[::-1], dtype, norms_in[k], k, gap=k) for k in range(3)]
    want = opref.clip([[t.double().cpu().numpy() for t in ts] for _, ts in made], 1.0)
    n = sum(sizes)
    guard = [torch.full((n + 16,), 7.0, device="cuda") for _ in range(3)]
    packed = [g[5 + k:5 + k + n] for k, g in enumerate(guard)] if mode == "packed" else None
    before = [f.clone() for f, _ in made]
    lst = al.autoloco_grads_create(ctx, [ts for _, ts in made], packed)
    norms = torch.full((3,), -1.0, device="cuda")
    st = al.autoloco_clip_grad_norm(ctx, lst, 1.0, norms=norms)
    for k in range(3):
        norm, c, ts = want[k]
        assert abs(st.grad_norm[k] - norm) <= 4 * 2.0 ** -24 * norm and abs(float(norms[k]) - norm) <= 5 * 2.0 ** -24 * norm
        assert abs(st.clip_coef[k] - c) <= 5 * 2.0 ** -24 * c and st.finite
        if mode == "packed":
            got = packed[k].double().cpu().numpy()
            ref = np.concatenate([t.reshape(-1) for t in ts]) if n else np.zeros(0)
            assert np.all(np.abs(got - ref) <= 8 * 2.0 ** -24 * np.abs(ref) + 1e-42)
            assert torch.equal(before[k], made[k][0])
            assert torch.all(guard[k][:5 + k] == 7) and torch.all(guard[k][5 + k + n:] == 7)
        else:
            mask = torch.ones_like(made[k][0], dtype=torch.bool)
            at = 0
            for s, ref, t in zip([len(x) for x in made[k][1]], ts, made[k][1]):
                got = t.double().cpu().numpy()
                assert np.all(np.abs(got - ref) <= (8 * 2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 0)) * np.abs(ref) + 1e-40)
                mask[at:at + s] = False
                at += s + k
            assert torch.equal(before[k][mask], made[k][0][mask])       # the gaps are left alone
            if c == 1.0:
                assert torch.equal(before[k], made[k][0])
    lst.close()


def test_mixed_types_shapes_and_reuse(ctx):
    """One list over fp32 and bf16 tensors of several shapes, used again after the gradients changed; bit-stable."""
    ts = [torch.randn(37, 19, device="cuda"), torch.randn(5, 3, 7, device="cuda").bfloat16(), torch.randn((), device="cuda"),
          torch.empty(0, 4, device="cuda"), torch.randn(20000, device="cuda").bfloat16()]
    n = sum(t.numel() for t in ts)
    packed = torch.empty(n, device="cuda")
    lst = al.autoloco_grads_create(ctx, [ts], [packed])
    for step in range(3):
        for t in ts:
            t.normal_()
        (norm, c, ref), = opref.clip([[t.double().cpu().numpy() for t in ts]], 2.5)
        st = al.autoloco_clip_grad_norm(ctx, lst, 2.5)
        assert abs(st.grad_norm[0] - norm) <= 4 * 2.0 ** -24 * norm
        got, flat = packed.double().cpu().numpy(), np.concatenate([r.reshape(-1) for r in ref])
        assert np.all(np.abs(got - flat) <= 8 * 2.0 ** -24 * np.abs(flat))
        first = packed.clone()
        st2 = al.autoloco_clip_grad_norm(ctx, lst, 2.5)
        assert st2.grad_norm[0] == st.grad_norm[0] and torch.equal(first, packed)
    assert al.autoloco_clip_grad_norm(ctx, lst, 0.0).clip_coef[0] == 1.0     # no clipping: packed as they are
    assert torch.equal(packed, torch.cat([t.float().reshape(-1) for t in ts]))


def test_same_norm_as_the_optimiser(ctx):
    """Packed and unclipped, then clipped by the AdamW step, or clipped here and then stepped: the same parameters but
    for the rounding of the clipped gradient (2^-24 relative), which moves a step of size lr by at most about 1e-6 lr."""
    n = 50003
    flat, ts = _views([20000, 3, 30000], "f32", 5.0, 2)
    a, b = torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    al.autoloco_clip_grad_norm(ctx, al.autoloco_grads_create(ctx, [ts], [a]), 0.0)
    sb = al.autoloco_clip_grad_norm(ctx, al.autoloco_grads_create(ctx, [ts], [b]), 1.0)
    new = lambda: [torch.zeros(n, device="cuda") for _ in range(3)]  # noqa: E731
    pa, pb = new(), new()
    sa = al.autoloco_inner_adamw(ctx, [pa[0]], [pa[1]], [pa[2]], [a], al.make_adamw_coeffs(1e-3, 1, max_grad_norm=1.0))
    al.autoloco_inner_adamw(ctx, [pb[0]], [pb[1]], [pb[2]], [b], al.make_adamw_coeffs(1e-3, 1, max_grad_norm=0.0))
    assert sa.grad_norm[0] == pytest.approx(sb.grad_norm[0], rel=1e-6) and sa.clip_coef[0] == pytest.approx(sb.clip_coef[0], rel=1e-6)
    assert torch.allclose(pa[0], pb[0], rtol=1e-5, atol=1e-8)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_non_finite_gradients(ctx, dtype):
    """NaN and infinities propagate to their worker only, as in the AdamW step."""
    made = [_views([5000, 13], dtype, 2.0, k)[1] for k in range(3)]
    made[0][1][3] = float("nan")
    made[1][0][7] = float("inf")
    packed = [torch.empty(5013, device="cuda") for _ in range(3)]
    st = al.autoloco_clip_grad_norm(ctx, al.autoloco_grads_create(ctx, made, packed), 1.0)
    assert not st.finite and np.isnan(st.grad_norm[0]) and np.isinf(st.grad_norm[1]) and np.isfinite(st.grad_norm[2])
    assert torch.isnan(packed[0]).all()
    assert int(torch.isnan(packed[1]).sum()) == 1 and not packed[1][packed[1] == packed[1]].any()
    assert torch.isfinite(packed[2]).all()


def test_small_and_large_magnitudes(ctx):
    """Squares of values from 2^-60 up to 2^60 in one worker neither vanish nor overflow in the sums."""
    t = torch.cat([torch.full((9,), 2.0 ** -60), torch.full((3,), 2.0 ** 60)]).cuda()
    st = al.autoloco_clip_grad_norm(ctx, al.autoloco_grads_create(ctx, [[t]], [torch.empty(12, device="cuda")]), 1.0)
    assert st.grad_norm[0] == pytest.approx(3 ** 0.5 * 2.0 ** 60, rel=1e-6)
    t = torch.full((9,), 2.0 ** -70, device="cuda")
    st = al.autoloco_clip_grad_norm(ctx, al.autoloco_grads_create(ctx, [[t]], None), 1.0)
    assert st.grad_norm[0] == pytest.approx(3 * 2.0 ** -70, rel=1e-6)


def test_no_tensors_and_sixteen_workers(ctx):
    lst = al.autoloco_grads_create(ctx, [[]])
    st = al.autoloco_clip_grad_norm(ctx, lst, 1.0)
    assert st.grad_norm[0] == 0 and st.clip_coef[0] == 1 and st.finite
    made = [[torch.full((k * 100 + 1,), 0.5, device="cuda")] for k in range(16)]
    norms = torch.empty(16, device="cuda")
    assert al.autoloco_clip_grad_norm(ctx, al.autoloco_grads_create(ctx, made), 0.0, norms=norms, stats=False) is None
    assert norms.tolist() == pytest.approx([0.5 * (k * 100 + 1) ** 0.5 for k in range(16)], rel=1e-6)


def test_tensor_past_32_bits(ctx):
    """A tensor of more than 2^32 elements: its end is read, clipped and left."""
    n = (1 << 32) + 100
    t = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    t[-1], t[5], t[1 << 32] = 3.0, 4.0, 12.0
    st = al.autoloco_clip_grad_norm(ctx, al.autoloco_grads_create(ctx, [[t]]), 6.5)
    assert st.grad_norm[0] == 13.0
    assert [float(t[i]) for i in (-1, 5, 1 << 32)] == [1.5, 2.0, 6.0]


def test_graph_replays():
    stream = torch.cuda.Stream()
    with al.autoloco_create(0, stream) as c, torch.cuda.stream(stream):
        ts = [torch.randn(3000, device="cuda"), torch.randn(71, device="cuda").bfloat16()]
        packed, norms = torch.empty(3071, device="cuda"), torch.empty(1, device="cuda")
        lst = al.autoloco_grads_create(c, [ts], [packed])
        run = lambda: al.autoloco_clip_grad_norm(c, lst, 1.0, norms=norms, stats=False)  # noqa: E731
        run()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            run()
        for _ in range(4):
            for t in ts:
                t.normal_()
            graph.replay()
            got = packed.clone(), norms.clone()
            run()
            stream.synchronize()
            assert torch.equal(got[0], packed) and torch.equal(got[1], norms)
        stream.synchronize()
        lst.close()


def test_refusals(ctx):
    f = lambda n: torch.zeros(n, device="cuda")  # noqa: E731
    err = al.AutolocoError
    room = f(100)
    for grads, packed, status in (([[room[:50], room[40:]]], None, -3), ([[room]], [room], -3), ([[f(10)], [f(10)]], [room[:10], room[5:15]], -3)):
        with pytest.raises(err) as ex:
            al.autoloco_grads_create(ctx, grads, packed)
        assert ex.value.status == status
    for bad in ([[torch.zeros(4)]], [[f(8)[::2]]], [[f(8).double()]]):
        with pytest.raises(TypeError):
            al.autoloco_grads_create(ctx, bad)
    for call in (lambda: al.autoloco_grads_create(ctx, []), lambda: al.autoloco_grads_create(ctx, [[]] * 17),
                 lambda: al.autoloco_grads_create(ctx, [[f(9)]], [f(8)]), lambda: al.autoloco_grads_create(ctx, [[f(9)]], [])):
        with pytest.raises(ValueError):
            call()
    lst = al.autoloco_grads_create(ctx, [[f(9)]])
    for norm in (-1.0, float("nan"), float("inf")):
        with pytest.raises(err) as ex:
            al.autoloco_clip_grad_norm(ctx, lst, norm)
        assert ex.value.status == -1
    lib, h = al.lib(), C.c_void_p()
    Grad = al._lib.Grad
    t = f(16)
    for g, status in ((Grad(t.data_ptr(), None, 4, 7, 0), -1), (Grad(t.data_ptr(), None, -1, 0, 0), -1), (Grad(None, None, 4, 0, 0), -1),
                      (Grad(t.data_ptr(), None, 4, 0, 1), -1), (Grad(t.data_ptr() + 2, None, 4, 0, 0), -2),
                      (Grad(torch.zeros(4).pin_memory().data_ptr(), None, 4, 0, 0), -1)):
        assert lib.autoloco_grads_create(ctx.handle, C.byref(g), 1, 1, C.byref(h)) == status
    two = (Grad * 2)(Grad(t.data_ptr(), t.data_ptr() + 16, 2, 0, 0), Grad(t.data_ptr() + 40, None, 2, 0, 0))
    assert lib.autoloco_grads_create(ctx.handle, two, 2, 1, C.byref(h)) == -1
    assert lib.autoloco_grads_create(ctx.handle, None, 1, 1, C.byref(h)) == -1
    assert lib.autoloco_grads_create(ctx.handle, two, -1, 1, C.byref(h)) == -1
    assert lib.autoloco_grads_create(None, two, 1, 1, C.byref(h)) == -1
    assert lib.autoloco_clip_grad_norm(ctx.handle, None, 1.0, None, None) == -1
    lst.close()
    with pytest.raises(err):
        al.autoloco_clip_grad_norm(ctx, lst, 1.0)
    al.autoloco_grads_destroy(lst)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("size", [2.0 ** 100, 2.0 ** -100])
def test_squares_beyond_the_range_of_fp32(ctx, size, dtype):
    """Gradients whose squares neither overflow nor vanish: norms and clipped values as for any other."""
    g = torch.Generator().manual_seed(3)
    ts = [(torch.randn(n, generator=g) * size).to(DT[dtype]).cuda() for n in (5001, 3, 70001)]
    norm, c, want = opref.clip([[t.double().cpu().numpy() for t in ts]], size)[0]
    packed = torch.empty(sum(t.numel() for t in ts), device="cuda")
    norms = torch.empty(1, device="cuda")
    st = al.autoloco_clip_grad_norm(ctx, al.autoloco_grads_create(ctx, [ts], [packed]), size, norms=norms)
    assert abs(st.grad_norm[0] - norm) <= 4 * 2.0 ** -24 * norm and abs(float(norms[0]) - norm) <= 5 * 2.0 ** -24 * norm
    assert abs(st.clip_coef[0] - c) <= 5 * 2.0 ** -24 * c and st.finite
    ref = np.concatenate(want)
    assert np.all(np.abs(packed.double().cpu().numpy() - ref) <= 8 * 2.0 ** -24 * np.abs(ref) + 2.0 ** -149)
