"""Log probabilities, entropy, best alternatives and the logits' gradient on the GPU."""
import numpy as np
import pytest
import torch

import block_math as bm
import ends_math as em
from paper_2509_25149_amd import binding as nv

pytestmark = pytest.mark.gpu
F32, BF16, I32, I64 = torch.float32, torch.bfloat16, torch.int32, torch.int64
OUT = {F32: nv.OUT_F32, BF16: nv.OUT_BF16}
# one column and fewer than eight; whole and broken groups of eight; a wavefront, 256 and 512 threads to a row; pieces of a row (one row of 65536 columns and more)
SHAPES = [(1, 1), (2, 7), (3, 8), (5, 9), (4, 100), (3, 513), (9, 4096), (2, 4100), (1, 5000), (3, 50257), (1, 131072), (300, 5001), (515, 4097), (513, 20003), (1, 262147)]


def pad_of(cols, extra=0):
    return -cols % 8 + extra


def logits(rows, cols, seed, dtype, extra=0, kind="plain"):
    r = np.random.default_rng(seed)
    z = 2 * r.standard_normal((rows, cols))
    if kind == "masked":
        z[:, r.random(cols) < 0.4] = -np.inf
        z[:, 0] = 1.0
    if kind == "far":
        z = 100 * z + r.choice([-1e4, 1e4], (rows, 1))
    return bm.tensor(z, dtype, pad_of(cols, extra))


def targets_of(rows, cols, seed):
    r = np.random.default_rng(seed)
    t = r.integers(0, cols, rows)
    if rows > 2:
        t[r.integers(0, rows, 1 + rows // 10)] = r.choice([-1, -100, cols, 2 ** 31 - 1])
    return t


def check_forward(out, z, scale, targets, top, entropy):
    z64, scale = bm.f64(z), float(np.float32(scale))
    m, logsum, p, logp, h = em.logits_statistics(z64, scale)
    rel = em.sum_error(z64, scale)[0]
    rows, cols = z64.shape
    if out.stats is not None:
        bm.within(out.stats[:, 0], m, np.zeros(rows))
        bm.within(out.stats[:, 1], logsum, rel + 2 * em.U * np.abs(logsum) + em.U)
    lse = scale * m + logsum
    bm.within(out.lse, lse, rel + em.U * (2 * np.abs(scale * m) + 3 * np.abs(logsum) + 2 * np.abs(lse)) + em.U)
    at = lambda col: (logp[np.arange(rows)[:, None], col], rel[:, None] + em.U * (4 * np.abs(logp + logsum[:, None]) + 4 * np.abs(logsum)[:, None] + 2 * np.abs(logp))[
        np.arange(rows)[:, None], col] + em.U)
    if targets is not None:
        counted = (targets >= 0) & (targets < cols)
        ref, tol = (v[:, 0] for v in at(np.clip(targets, 0, cols - 1)[:, None]))
        got, ref, tol = bm.f64(out.logprob), np.where(counted, ref, 0.0), np.where(counted, tol, 0.0)
        same = np.isneginf(ref)                                     # a masked target
        assert np.all(np.isneginf(got[same]))
        bm.within(got[~same], ref[~same], tol[~same])
    if entropy:
        bm.within(out.entropy, h, em.entropy_error(z64, scale))
    if top:
        want = em.best(z64, top)
        assert np.array_equal(out.top_index.cpu().numpy(), want)
        ref, tol = at(want)
        got, same = bm.f64(out.top_logprob), np.isneginf(ref)
        assert np.all(np.isneginf(got[same]))
        bm.within(got[~same], ref[~same], tol[~same])


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dt,it,scale,entropy,top,kind", [(BF16, I64, 1.0, True, 5, "plain"), (F32, I32, 0.7, False, 0, "plain"), (F32, I64, 1.25, True, 32, "masked"),
                                                          (BF16, I32, 1.0, False, 1, "far"), (F32, I32, 1.0, True, 0, "far"), (BF16, I64, 3.0, True, 0, "masked")])
def test_forward(rows, cols, dt, it, scale, entropy, top, kind):
    z = logits(rows, cols, rows + cols, dt, 8, kind)
    t, top = targets_of(rows, cols, 1), min(top, cols)
    out = nv.nvfp4_logprob_forward(z, em.index(t, it), scale=scale, entropy=entropy, top=top, for_backward=True)
    check_forward(out, z, scale, t, top, entropy)
    again = nv.nvfp4_logprob_forward(z, None, scale=scale, entropy=entropy, top=top)
    assert again.logprob is None and again.stats is None and all(torch.equal(getattr(out, f), getattr(again, f)) for f in ("lse", "entropy", "top_index", "top_logprob") if getattr(out, f) is not None)


def check_gradient(dz, z, scale, targets, g, g_lse, g_entropy, dtype):
    f = lambda v: None if v is None else bm.f64(v)
    ref, tol = em.logits_gradient(bm.f64(z), float(np.float32(scale)), targets, f(g), f(g_lse), f(g_entropy))
    bm.within(dz, ref, tol + bm.rounding(ref, dtype))


@pytest.mark.parametrize("rows,cols", [s for s in SHAPES if s[0] * s[1] < 1 << 22])
@pytest.mark.parametrize("dt,ot,it,scale,which,kind", [(BF16, BF16, I64, 1.0, "g", "plain"), (F32, F32, I32, 0.7, "gle", "plain"), (BF16, F32, I64, 1.25, "ge", "masked"),
                                                       (F32, BF16, I32, 1.0, "l", "far"), (BF16, BF16, I32, 1.0, "e", "plain"), (F32, F32, I64, 2.0, "gl", "masked")])
def test_backward(rows, cols, dt, ot, it, scale, which, kind):
    r = np.random.default_rng(cols)
    z = logits(rows, cols, rows * 7 + cols, dt, 8, kind)
    t = targets_of(rows, cols, 2)
    g, gl, ge = (torch.as_tensor(r.standard_normal(rows).astype(np.float32)).cuda() if c in which else None for c in "gle")
    fwd = nv.nvfp4_logprob_forward(z, em.index(t, it), scale=scale, entropy=True, for_backward=True)
    args = dict(g_logprob=g, g_lse=gl, g_entropy=ge, entropy=fwd.entropy if ge is not None else None, scale=scale)
    tt = em.index(t, it) if g is not None else None
    dz = nv.nvfp4_logprob_backward(z, tt, fwd.stats, out_dtype=OUT[ot], **args)
    assert dz.dtype == ot and dz.stride(0) % 8 == 0
    check_gradient(dz, z, scale, t if g is not None else None, g, gl, ge, ot)
    own = bm.tensor(np.zeros((rows, cols)), ot, pad_of(cols, 16))
    assert nv.nvfp4_logprob_backward(z, tt, fwd.stats, out=own, **args) is own and torch.equal(own, dz)
    behind = pad_of(cols, 16)
    assert torch.isnan(own.as_strided((rows, behind), (own.stride(0), 1), cols)).all()
    if dt == ot:      # over the logits
        assert nv.nvfp4_logprob_backward(z, tt, fwd.stats, out=z, **args) is z and torch.equal(z, dz)
        assert torch.isnan(z.as_strided((rows, pad_of(cols, 8)), (z.stride(0), 1), cols)).all()


@pytest.mark.parametrize("rows,cols", [s for s in SHAPES if s[0] * s[1] < 1 << 22] + [(1030, 4100), (1100, 60), (600, 9000)])
@pytest.mark.parametrize("dt,ot,it,scale,kind", [(BF16, BF16, I64, 1.0, "plain"), (F32, F32, I32, 0.7, "masked"), (BF16, F32, I64, 1.0, "far"), (F32, BF16, I32, 1.5, "plain")])
def test_loss_and_gradient_together(rows, cols, dt, ot, it, scale, kind):
    r = np.random.default_rng(cols)
    z = logits(rows, cols, rows * 5 + cols, dt, 0, kind)
    t, g = targets_of(rows, cols, 3), torch.as_tensor((-r.random(rows) / rows).astype(np.float32)).cuda()
    out = nv.nvfp4_logprob_with_gradient(z, em.index(t, it), g, scale=scale, out_dtype=OUT[ot])
    check_forward(out, z, scale, t, 0, False)
    check_gradient(out.dlogits, z, scale, t, g, None, None, ot)
    if dt == ot:
        over = nv.nvfp4_logprob_with_gradient(z, em.index(t, it), g, scale=scale, out=z)
        assert over.dlogits is z and torch.equal(z, out.dlogits) and torch.equal(over.logprob, out.logprob)
        behind = pad_of(cols)
        assert behind == 0 or torch.isnan(z.as_strided((rows, behind), (z.stride(0), 1), cols)).all()


@pytest.mark.parametrize("rows,cols", [(6, 40), (6, 4097), (6, 9000), (600, 20000)])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_rows_that_masks_leave_nothing_of(rows, cols, dt):
    z = bm.tensor(np.random.default_rng(1).standard_normal((rows, cols)), dt, pad_of(cols))
    lowest = torch.finfo(dt).min
    z[0] = -torch.inf                                       # nothing
    z[1] = lowest                                           # masked by the lowest value: uniform
    z[2] = -torch.inf
    z[2, cols - 1] = 3.0                                    # one value
    z[3] = lowest
    z[3, 5] = 1.0
    z[4, 1::2] = lowest
    t = np.full(rows, 5)
    t[2] = cols - 1
    out = nv.nvfp4_logprob_forward(z, em.index(t, I64), entropy=True, top=3, for_backward=True)
    lp, h, idx, tl = bm.f64(out.logprob), bm.f64(out.entropy), out.top_index.cpu().numpy(), bm.f64(out.top_logprob)
    assert np.isneginf(lp[0]) and np.isneginf(bm.f64(out.lse)[0]) and h[0] == 0 and list(idx[0]) == [0, 1, 2] and np.all(np.isneginf(tl[0]))
    assert abs(lp[1] + np.log(cols)) <= 1e-5 and abs(h[1] - np.log(cols)) <= 1e-5 and list(idx[1]) == [0, 1, 2] and np.all(np.abs(tl[1] + np.log(cols)) <= 1e-5)
    assert lp[2] == 0 and h[2] == 0 and list(idx[2]) == [cols - 1, 0, 1] and tl[2, 0] == 0 and np.all(np.isneginf(tl[2, 1:]))
    assert lp[3] == 0 and h[3] == 0 and idx[3, 0] == 5
    g = torch.ones(rows, device="cuda")
    dz = bm.f64(nv.nvfp4_logprob_backward(z, em.index(t, I64), out.stats, g_logprob=g, g_lse=g, g_entropy=g, entropy=out.entropy))
    assert np.all(np.isfinite(dz)) and np.all(dz[0] == 0)
    uniform = np.where(np.arange(cols) == 5, 1.0, 0.0)     # g_lse takes the other part away
    assert np.all(np.abs(dz[1] - uniform) <= 2.0 ** -8 * np.abs(uniform) + 1e-5)
    one = nv.nvfp4_logprob_with_gradient(z, em.index(t, I64), g)
    assert torch.equal(one.dlogits[0], torch.zeros_like(one.dlogits[0])) and bool(torch.isfinite(one.dlogits).all())
    assert np.all(np.abs(bm.f64(one.dlogits)[1] - uniform + 1 / cols) <= 2.0 ** -8 + 1e-5 / cols)
    assert np.isneginf(bm.f64(one.logprob)[0]) and float(one.logprob[2]) == 0


@pytest.mark.parametrize("rows,cols", [(4, 40), (4, 9000), (600, 4100)])
def test_trouble_shows_in_its_row_and_nowhere_else(rows, cols):
    z = bm.tensor(np.random.default_rng(2).standard_normal((rows, cols)), F32, pad_of(cols))
    clean = nv.nvfp4_logprob_forward(z, None, entropy=True, top=2)
    z[1, 7], z[2, cols - 1] = torch.nan, torch.inf
    t = torch.zeros(rows, dtype=I64, device="cuda")
    out = nv.nvfp4_logprob_forward(z, t, entropy=True, top=2, for_backward=True)
    for v in (out.logprob, out.lse, out.entropy):
        assert bool(torch.isnan(v[1:3]).all()) and bool(torch.isfinite(v[0]).all()) and bool(torch.isfinite(v[3:]).all())
    assert int(out.top_index[2, 0]) == cols - 1 and 7 not in out.top_index[1].tolist() and torch.equal(out.top_index[3:], clean.top_index[3:])
    assert torch.equal(out.lse[3:], clean.lse[3:])
    dz = nv.nvfp4_logprob_backward(z, t, out.stats, g_logprob=torch.ones(rows, device="cuda"))
    assert bool(torch.isnan(dz[1:3]).all()) and bool(torch.isfinite(dz[0]).all()) and bool(torch.isfinite(dz[3:]).all())


@pytest.mark.parametrize("top", [1, 2, 31, 32])
@pytest.mark.parametrize("rows,cols", [(2, 32), (3, 100), (2, 2000), (600, 3000), (3, 9001), (600, 33000), (1, 131072)])
def test_best_alternatives_where_many_are_equal(rows, cols, top):
    r = np.random.default_rng(rows + cols + top)
    kinds = [np.zeros(cols), np.sort(r.standard_normal(cols)), -np.sort(r.standard_normal(cols)), np.round(2 * r.standard_normal(cols)), np.where(np.arange(cols) % 2, 0.0, -0.0),
             np.where(np.arange(cols) > cols - 5, 1.0, -np.inf), np.where(np.arange(cols) % 7 == 3, r.standard_normal(cols), -np.inf)]
    for first in range(0, len(kinds), rows):
        z = np.stack([kinds[(first + i) % len(kinds)] for i in range(rows)])
        for dt in (F32, BF16):
            x = bm.tensor(z, dt, pad_of(cols))
            out = nv.nvfp4_logprob_forward(x, None, top=top)
            assert np.array_equal(out.top_index.cpu().numpy(), em.best(bm.f64(x), top))


def test_gradients_agree_with_differences():
    """Of a weighted sum of log probabilities, normalisers and entropies, against differences of the formula in 64 bits."""
    rows, cols, scale = 5, 300, 0.7
    r = np.random.default_rng(3)
    z, t = r.standard_normal((rows, cols)).astype(np.float32), r.integers(0, cols, rows)
    w = [r.standard_normal(rows).astype(np.float32) for _ in range(3)]

    def f(z):
        m, logsum, p, logp, h = em.logits_statistics(z, scale)
        return (w[0] * logp[np.arange(rows), t] + w[1] * (scale * m + logsum) + w[2] * h).sum()
    x = bm.tensor(z, F32, pad_of(cols))
    fwd = nv.nvfp4_logprob_forward(x, em.index(t, I64), scale=scale, entropy=True, for_backward=True)
    g = [torch.as_tensor(v).cuda() for v in w]
    dz = bm.f64(nv.nvfp4_logprob_backward(x, em.index(t, I64), fwd.stats, g_logprob=g[0], g_lse=g[1], g_entropy=g[2], entropy=fwd.entropy, scale=scale))
    for _ in range(4):
        v = r.standard_normal(z.shape)
        diff = (f(z + 1e-5 * v) - f(z - 1e-5 * v)) / 2e-5
        assert abs((dz * v).sum() - diff) <= 1e-5 * np.sqrt((dz ** 2).sum()) * np.sqrt(2)


def test_without_rows():
    z, t = torch.empty(0, 96, device="cuda", dtype=BF16), torch.empty(0, dtype=I32, device="cuda")
    out = nv.nvfp4_logprob_forward(z, t, entropy=True, top=4)
    assert out.logprob.shape == (0,) and out.top_index.shape == (0, 4)
    assert nv.nvfp4_logprob_with_gradient(z, t, torch.empty(0, device="cuda")).dlogits.shape == (0, 96)


def test_more_rows_than_a_launch_has_threads_for():
    rows, cols = (1 << 24) + 100_000, 8
    z = torch.zeros(rows, cols, device="cuda", dtype=BF16)
    z[-1, 3] = 5.0
    t = torch.full((rows,), 3, dtype=I32, device="cuda")
    g = torch.ones(rows, device="cuda")
    out = nv.nvfp4_logprob_with_gradient(z, t, g)
    want = em.logits_statistics(bm.f64(z[-2:]), 1.0)
    bm.within(out.logprob[-2:], want[3][:, 3], np.full(2, 1e-6))
    assert int((out.logprob[:-1] == out.logprob[0]).sum()) == rows - 1
    bm.within(out.dlogits[-2:], np.eye(8)[[3, 3]] - want[2], np.full((2, 8), 2.0 ** -8))
    assert bool((out.dlogits[:-1] == out.dlogits[0]).all())


def test_offsets_beyond_2_to_the_31():
    rows, cols = 17_000, 131072
    z = torch.zeros(rows, cols, device="cuda", dtype=BF16)
    z[-1, -1] = 20.0
    t = torch.full((rows,), cols - 1, dtype=I64, device="cuda")
    out = nv.nvfp4_logprob_forward(z, t, entropy=True, for_backward=True)
    s = np.exp(20.0) + cols - 1
    assert abs(float(out.logprob[-1]) - (20 - np.log(s))) <= 1e-5 and abs(float(out.logprob[0]) + np.log(cols)) <= 1e-5
    dz = nv.nvfp4_logprob_backward(z, t, out.stats, g_logprob=torch.ones(rows, device="cuda"), out=z)
    assert abs(float(dz[-1, -1]) - (1 - np.exp(20.0) / s)) <= 1e-6 and abs(float(dz[-1, 0]) + 1 / s) <= 2.0 ** -8 / s
    assert abs(float(dz[-2, -1]) - 1) <= 2.0 ** -8
