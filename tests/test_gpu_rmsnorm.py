"""Residual addition and root-mean-square norm with its 8-bit output, and the gradient, on the GPU."""
import numpy as np
import pytest
import torch

import block_math as bm
from paper_2509_25149_amd import binding as nv

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
OUT = {F32: nv.OUT_F32, BF16: nv.OUT_BF16}
EPS = 1e-5
# columns at and beside the limits of a wavefront (512, 1024), a workgroup with one, two and four chunks (2048, 16384, 32768); a few rows, which the
# backward pass gives to one workgroup, and as many as there are workgroups or (1025 x 2064) more
SHAPES = [(1, 16), (1, 5120), (5, 496), (3, 512), (9, 528), (6, 1024), (7, 1040), (2, 2048), (3, 2064), (5, 5120), (2, 16384), (3, 16400), (2, 32768),
          (1030, 256), (2100, 48), (517, 1040), (1025, 2064)]
FP32 = 64 * 2.0 ** -24     # relative error of a row's sum of squares (a tree of depth 64 at most) and of the operations behind it


def activations(rows, cols, seed, dtype):
    r = np.random.default_rng(seed)
    v = r.standard_normal((rows, cols)) * np.where(r.random((rows, cols)) < 0.01, 50, 1) * np.exp2(r.integers(-3, 4, (rows, 1)))
    return bm.f64(torch.as_tensor(v.astype(np.float32)).to(dtype))


def check_checkpoint(c, ref):
    """A value within half a step of E4M3 at its scale (and FP32's error); the scale that of an amax within FP32's error of the true one."""
    codes, scales = c.codes.cpu().numpy(), c.scales.cpu().numpy()
    lo, hi = bm.encode(ref * (1 - 2 * FP32))[1], bm.encode(ref * (1 + 2 * FP32))[1]
    assert np.all((scales == lo) | (scales == hi))
    step = np.repeat(np.exp2(scales.astype(np.float64) - 127), 16, 1) * 2.0 ** -10
    bm.within(bm.decode(codes, scales), ref, np.maximum(np.abs(ref) * 2.0 ** -4, step) * (1 + 2.0 ** -10) + 2 * FP32 * np.abs(ref))


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("xt,ht,yt,residual,gamma,pad", [(BF16, BF16, BF16, True, True, 0), (F32, F32, F32, True, True, 8), (BF16, F32, BF16, True, False, 0),
                                                         (BF16, BF16, F32, False, True, 8), (F32, BF16, BF16, True, True, 0), (F32, F32, BF16, False, False, 0)])
def test_forward(rows, cols, xt, ht, yt, residual, gamma, pad):
    r = np.random.default_rng(rows + cols)
    x, res = activations(rows, cols, 1, xt), activations(rows, cols, 2, ht) if residual else None
    g = (1 + 0.1 * r.standard_normal(cols)).astype(np.float32) if gamma else None
    h, rstd, xhat, y = bm.norm(x, res, None if g is None else g.astype(np.float64), EPS)
    gt = None if g is None else torch.as_tensor(g).cuda()
    xg, rg = bm.tensor(x, xt, pad), bm.tensor(res, ht, pad) if residual else None
    out = nv.nvfp4_rmsnorm_forward(xg, gt, residual=rg, eps=EPS, y_dtype=OUT[yt], checkpoint=True)
    bm.within(out.rstd, rstd, FP32 * rstd)
    bm.within(out.y, y, 2 * FP32 * np.abs(y) + bm.rounding(y, yt))
    if residual:
        assert out.h.dtype == ht
        bm.within(out.h, h, 2.0 ** -24 * np.abs(h) + bm.rounding(h, ht))
    else:
        assert out.h is xg
    check_checkpoint(out.checkpoint, xhat)
    out_y = nv.nvfp4_rmsnorm_forward(xg, gt, residual=rg, eps=EPS, y_dtype=None, checkpoint=True, keep_kind=nv.NORM_KEEP_OUTPUT)
    assert out_y.y is None
    check_checkpoint(out_y.checkpoint, y)
    # into the caller's own tensors, without the checkpoint: the same bits
    yo = bm.tensor(np.zeros((rows, cols)), yt, 24)
    again = nv.nvfp4_rmsnorm_forward(xg, gt, residual=rg, eps=EPS, y=yo)
    assert again.y is yo and again.checkpoint is None and torch.equal(yo, out.y) and torch.equal(again.rstd, out.rstd)
    assert torch.isnan(yo.as_strided((rows, 24), yo.stride(), cols)).all()


def test_sum_over_the_residual_and_norm_over_the_input():
    x, res = (bm.tensor(activations(37, 2064, s, BF16), BF16) for s in (3, 4))
    want = nv.nvfp4_rmsnorm_forward(x, None, residual=res, eps=EPS)
    got = nv.nvfp4_rmsnorm_forward(x, None, residual=res, eps=EPS, h=res, y=x)
    assert torch.equal(got.h, want.h) and torch.equal(got.y, want.y) and got.h is res and got.y is x


def test_rows_of_zeros_of_huge_numbers_and_of_infinities():
    x = np.ones((5, 2064), np.float32)
    x[0] = 0
    x[1] = 1e15
    x[2, 7] = np.inf
    x[3, 9] = np.nan
    out = nv.nvfp4_rmsnorm_forward(bm.tensor(x, F32), None, eps=EPS, y_dtype=nv.OUT_F32, checkpoint=True)
    y = bm.f64(out.y)
    assert np.all(y[0] == 0) and np.allclose(y[1], 1, atol=1e-5) and np.allclose(y[4], 1, atol=1e-4)
    assert np.isnan(y[2, 7]) and np.all(y[2, :7] == 0) and np.all(np.isnan(y[3]))
    s = out.checkpoint.scales.cpu().numpy()
    assert np.all(s[0] == 0) and s[2, 0] == 255 and np.all(s[2, 1:] == 0) and np.all(s[3] == 255)
    # the largest numbers whose squares still have a sum
    big = nv.nvfp4_rmsnorm_forward(torch.full((1, 64), 1e18, device="cuda"), None, eps=0.0, y_dtype=nv.OUT_F32)
    assert np.allclose(bm.f64(big.y), 1, atol=1e-5)


def backward_tolerance(dy, xhat, rstd, g, dres, ref):
    """c is a mean along a tree of depth 64 at most of products of three rounded factors; then four operations."""
    c = np.abs(g * xhat).mean(1, keepdims=True)
    return 2 * FP32 * (rstd[:, None] * (np.abs(g) + np.abs(xhat) * c) + (0 if dres is None else np.abs(dres)))


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dt,st,saved8,gamma,res,pad", [(BF16, BF16, True, True, True, 0), (BF16, BF16, False, True, True, 8), (F32, F32, False, False, True, 0),
                                                        (F32, F32, True, True, False, 8), (BF16, F32, False, True, True, 0), (BF16, F32, True, False, True, 0),
                                                        (F32, BF16, True, True, True, 0), (F32, BF16, False, True, False, 0)])
def test_backward(rows, cols, dt, st, saved8, gamma, res, pad):
    r = np.random.default_rng(rows * 3 + cols)
    h = bm.tensor(activations(rows, cols, 5, st), st, pad)
    gt = torch.as_tensor((1 + 0.1 * r.standard_normal(cols)).astype(np.float32)).cuda() if gamma else None
    fwd = nv.nvfp4_rmsnorm_forward(h, gt, eps=EPS, checkpoint=True)
    dy = bm.tensor(1e-3 * r.standard_t(3, (rows, cols)), dt, pad)
    dres = bm.tensor(1e-3 * r.standard_t(3, (rows, cols)), st, pad) if res else None
    saved = fwd.checkpoint if saved8 else h
    old = torch.as_tensor(r.standard_normal(cols).astype(np.float32)).cuda()
    dx, dgamma = nv.nvfp4_rmsnorm_backward(dy, saved, fwd.rstd, gt, dres=dres, dx_dtype=OUT[st])
    rstd = bm.f64(fwd.rstd)
    xhat = bm.decode(saved.codes.cpu().numpy(), saved.scales.cpu().numpy()) if saved8 else bm.f64(h) * rstd[:, None]
    d64, g64, r64 = bm.f64(dy), None if gt is None else bm.f64(gt), None if dres is None else bm.f64(dres)
    ref, ref_gamma = bm.norm_backward(d64, xhat, rstd, g64, r64)
    bm.within(dx, ref, backward_tolerance(d64, xhat, rstd, d64 if g64 is None else d64 * g64, r64, ref) + bm.rounding(ref, st))
    depth = -(-rows // 512) + 4 + 64
    tol = depth * 2.0 ** -24 * np.abs(d64 * xhat).sum(0) + 1e-37
    bm.within(dgamma, ref_gamma, tol)
    before = bm.f64(old)
    dx2, grown = nv.nvfp4_rmsnorm_backward(dy, saved, fwd.rstd, gt, dres=dres, dx=dy if dt == st else None, dx_dtype=OUT[st], dgamma=old, accumulate_dgamma=True)
    assert torch.equal(dx2, dx)
    bm.within(grown, ref_gamma + before, tol + 2.0 ** -23 * (np.abs(before) + np.abs(ref_gamma)))


def test_the_gradient_agrees_with_differences():
    """Along random directions in x and gamma, against differences of the formula in 64 bits."""
    rows, cols = 6, 1040
    r = np.random.default_rng(8)
    x, g, w = r.standard_normal((rows, cols)).astype(np.float32), (1 + 0.1 * r.standard_normal(cols)).astype(np.float32), r.standard_normal((rows, cols)).astype(np.float32)
    fwd = nv.nvfp4_rmsnorm_forward(bm.tensor(x, F32), torch.as_tensor(g).cuda(), eps=EPS, y_dtype=nv.OUT_F32)
    dx, dgamma = nv.nvfp4_rmsnorm_backward(bm.tensor(w, F32), bm.tensor(x, F32), fwd.rstd, torch.as_tensor(g).cuda())
    f = lambda x, g: (bm.norm(x, None, g, EPS)[3] * w).sum()
    x64, g64 = x.astype(np.float64), g.astype(np.float64)
    for _ in range(4):
        vx, vg, t = r.standard_normal(x.shape), r.standard_normal(g.shape), 1e-5
        diff = (f(x64 + t * vx, g64 + t * vg) - f(x64 - t * vx, g64 - t * vg)) / (2 * t)
        got = (bm.f64(dx) * vx).sum() + (bm.f64(dgamma) * vg).sum()
        # FP32's errors of dx and dgamma are independent over 6240 + 1040 terms; the differences are good to 1e-8 of the same sum
        size = np.sqrt((bm.f64(dx) ** 2).sum() + (bm.f64(dgamma) ** 2).sum())
        assert abs(got - diff) <= 1e-5 * size * np.sqrt(2)


def test_tensors_without_rows():
    x = torch.empty(0, 5120, device="cuda", dtype=BF16)
    out = nv.nvfp4_rmsnorm_forward(x, None, residual=x, checkpoint=True)
    assert out.y.shape == (0, 5120) and out.rstd.shape == (0,)
    dx, dgamma = nv.nvfp4_rmsnorm_backward(x, out.checkpoint, out.rstd)
    assert dx.shape == (0, 5120) and torch.equal(dgamma, torch.zeros(5120, device="cuda"))


def test_same_bits_every_time_and_on_another_stream():
    rows, cols = 1025, 2064
    h = bm.tensor(activations(rows, cols, 6, BF16), BF16)
    dy = bm.tensor(np.random.default_rng(1).standard_normal((rows, cols)), BF16)
    fwd = nv.nvfp4_rmsnorm_forward(h, checkpoint=True)
    want = nv.nvfp4_rmsnorm_backward(dy, fwd.checkpoint, fwd.rstd)
    need = nv.rowsum_workspace_bytes(rows, cols)
    buf = torch.full((need + 4096,), 0xAB, dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = nv.nvfp4_rmsnorm_backward(dy, fwd.checkpoint, fwd.rstd, workspace=buf[:need])
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.all(buf[need:] == 0xAB)


def test_more_rows_than_a_launch_has_threads_for():
    """67.2 million rows of 16 columns, a wavefront each: 2^32 threads are reached at 67.1 million."""
    rows, cols = (1 << 26) + 100_000, 16
    x = torch.ones(rows, cols, device="cuda", dtype=BF16)
    v = activations(3, cols, 11, BF16)
    x[-3:] = bm.tensor(v, BF16)
    x[(1 << 26) - 4] = 0
    out = nv.nvfp4_rmsnorm_forward(x, eps=EPS, checkpoint=True)
    ref = bm.norm(v, None, None, EPS)[3]
    bm.within(out.y[-3:], ref, 2 * FP32 * np.abs(ref) + bm.rounding(ref, BF16))
    rest = out.y[:-3]
    assert int((rest == 0).sum()) == cols and int((rest == 1).sum()) == rest.numel() - cols
    assert int((out.checkpoint.codes[:-3] == 0).sum()) == cols
    check_checkpoint(nv.Checkpoint8(out.checkpoint.codes[-3:], out.checkpoint.scales[-3:]), ref)
