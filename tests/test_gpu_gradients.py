"""The norm over many gradients and clipping, on the GPU."""
import numpy as np
import pytest
import torch

import block_math as bm
import ends_math as em
from paper_2509_25149_amd import binding as nv

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


def gradients(kind, seed=0):
    r = np.random.default_rng(seed)
    t = lambda shape, dtype=F32: torch.as_tensor((1e-3 * r.standard_normal(shape)).astype(np.float32)).to("cuda", dtype)
    if kind == "one":
        return [t((1,))]
    if kind == "block":
        return [t((272,)), t((272, 1040)), t((1040,)), t((1040, 272)), t((272,))]
    if kind == "mixed":      # odd sizes, views that start anywhere, rows that lie apart, more than two dimensions, nothing at all
        flat, wide = t((5000,), BF16), t((70, 300))
        return [t((0,)), t((3,), BF16), flat[1:1001], t((8193,)), wide[:, 4:105], t((70, 304), BF16)[:, 8:296], t((5, 7, 11)), t((64, 0)), t((33, 16384 + 24))[:, :16384 + 9], t((9, 1)),
                t((200, 20))[:, 3:4], t((1, 77), BF16)]
    if kind == "many":
        return [t((int(n),), (F32, BF16)[i % 2]) for i, n in enumerate(r.integers(1, 300, 3000))]
    return [t((1 << 22) + 3) for _ in range(3)]      # large: several units each


KINDS = ["one", "block", "mixed", "many", "large"]


def norm_of(grads):
    return np.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))


def check(outs, before, coef):
    """One rounding of the factor, one of the product, one to the type."""
    for o, b in zip(outs, before):
        ref = b * coef
        bm.within(o.reshape(-1), ref.reshape(-1), (2 * em.U * np.abs(ref) + bm.rounding(ref, o.dtype)).reshape(-1) + 1e-40)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("factor", [0.25, 4.0])
def test_in_place(kind, factor):
    grads = gradients(kind)
    before, bits = [bm.f64(g) for g in grads], [g.clone() for g in grads]
    n = nv.Gradients(grads)
    norm = norm_of(grads)
    sumsq = nv.nvfp4_grad_sumsq(n)
    assert abs(float(sumsq) - norm ** 2) <= 1e-12 * norm ** 2 and torch.equal(sumsq, nv.nvfp4_grad_sumsq(n))
    got = nv.nvfp4_grad_clip(n, sumsq, factor * norm)
    assert abs(float(got) - norm) <= 2 * em.U * norm
    if factor > 1:
        assert all(torch.equal(a, b) for a, b in zip(grads, bits))
    else:
        check(grads, before, factor)
        assert abs(norm_of(grads) - factor * norm) <= 2.0 ** -8 * factor * norm


def test_what_lies_between_rows_and_around_views_is_left_alone():
    wide = torch.full((70, 300), 7.0, device="cuda")
    flat = torch.full((1000,), 7.0, device="cuda", dtype=BF16)
    a, b = wide[:, 4:105], flat[1:900]
    a.fill_(1.0), b.fill_(1.0)
    n = nv.Gradients([a, b])
    nv.nvfp4_grad_clip(n, nv.nvfp4_grad_sumsq(n), 0.0)
    assert bool((a == 0).all()) and bool((b == 0).all())
    assert bool((wide[:, :4] == 7).all()) and bool((wide[:, 105:] == 7).all()) and float(flat[0]) == 7 and bool((flat[900:] == 7).all())


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("out_type", [F32, BF16])
@pytest.mark.parametrize("max_norm", [1e-4, 1e9, float("inf")])
def test_into_other_tensors(kind, out_type, max_norm):
    grads = gradients(kind, 1)
    before, bits = [bm.f64(g) for g in grads], [g.clone() for g in grads]
    outs = [torch.full(g.shape, 7.0, device="cuda", dtype=out_type) for g in grads]
    if kind == "mixed":
        outs[4] = torch.full((70, 128), 7.0, device="cuda", dtype=out_type)[:, :101]
    n = nv.Gradients(grads, outs)
    norm = norm_of(grads)
    assert abs(float(nv.nvfp4_grad_clip(n, nv.nvfp4_grad_sumsq(n), max_norm)) - norm) <= 2 * em.U * norm
    check(outs, before, min(1.0, float(np.float32(max_norm)) / norm))
    assert all(torch.equal(a, b) for a, b in zip(grads, bits))


def test_numbers_whose_squares_leave_fp32():
    g = [torch.full((1000,), 1e30, device="cuda"), torch.full((10,), 1e-30, device="cuda")]
    n = nv.Gradients(g)
    norm = nv.nvfp4_grad_clip(n, nv.nvfp4_grad_sumsq(n), 1.0)
    assert abs(float(norm) / (1e30 * np.sqrt(1000)) - 1) <= 1e-6 and abs(float(g[0][0]) * np.sqrt(1000) - 1) <= 1e-6 and bool((g[1] == 0).all())
    small = nv.Gradients([torch.full((100,), 1e-30, device="cuda")])
    assert abs(float(nv.nvfp4_grad_clip(small, nv.nvfp4_grad_sumsq(small), float("inf"))) / 1e-29 - 1) <= 1e-6
    top = [torch.full((2,), 3e38, device="cuda")]            # the norm itself is beyond FP32: it still clips
    n = nv.Gradients(top)
    assert float(nv.nvfp4_grad_clip(n, nv.nvfp4_grad_sumsq(n), 1.0)) == float("inf") and abs(float(top[0][0]) * np.sqrt(2) - 1) <= 1e-6


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_norm_that_is_not_finite_leaves_the_gradients(bad):
    g = [torch.ones(100, device="cuda"), torch.ones(9, 16, device="cuda", dtype=BF16)]
    g[0][17] = bad
    before = [t.clone() for t in g]
    n = nv.Gradients(g)
    norm = float(nv.nvfp4_grad_clip(n, nv.nvfp4_grad_sumsq(n), 0.5))
    assert (np.isnan(norm) if np.isnan(bad) else norm == float("inf"))
    assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(g, before))


def test_nothing_and_zeros():
    for tensors in ([], [torch.empty(0, device="cuda")], [torch.zeros(50, device="cuda")]):
        n = nv.Gradients(tensors)
        sumsq = nv.nvfp4_grad_sumsq(n, out=torch.full((1,), 3.0, device="cuda", dtype=torch.float64))
        assert float(sumsq) == 0 and float(nv.nvfp4_grad_clip(n, sumsq, 0.0)) == 0


def test_sums_of_several_lists():
    a, b = gradients("block", 3), gradients("many", 4)
    norm, before = norm_of(a + b), [bm.f64(g) for g in a + b]
    lists = [nv.Gradients(a), nv.Gradients(b)]
    total = nv.nvfp4_grad_sumsq(lists[0]) + nv.nvfp4_grad_sumsq(lists[1])
    for n in lists:
        assert abs(float(nv.nvfp4_grad_clip(n, total, norm / 2)) - norm) <= 2 * em.U * norm
    check(a + b, before, 0.5)


def test_more_than_2_to_the_31_elements():
    g = torch.full(((1 << 31) + 5000,), 0.5, device="cuda")
    n = nv.Gradients([g, torch.ones(3, device="cuda")])
    norm = float(nv.nvfp4_grad_clip(n, nv.nvfp4_grad_sumsq(n), 1.0))
    want = np.sqrt(0.25 * g.numel() + 3)
    assert abs(norm - want) <= 2 * em.U * want
    assert bool((g == g[0]).all()) and abs(float(g[0]) - 0.5 / want) <= 3 * em.U * 0.5 / want


def test_the_list_refuses():
    t = torch.ones(64, 64, device="cuda")
    for bad in (lambda: nv.Gradients([t, t]), lambda: nv.Gradients([t, t[3:5]]), lambda: nv.Gradients([t], [torch.ones(64, 63, device="cuda")]), lambda: nv.Gradients([t], []),
                lambda: nv.Gradients([t.half()]), lambda: nv.Gradients([t.t()[:3]]), lambda: nv.Gradients([t, torch.ones(3)]), lambda: nv.Gradients([t], [t.bfloat16().view(F32)])):
        with pytest.raises((ValueError, nv.NVFP4Error)):
            bad()
    nv.Gradients([t[:, :8], t[:, 8:]])            # columns of one tensor lie between each other's rows
    nv.Gradients([t, t], [torch.empty_like(t), torch.empty_like(t)])
