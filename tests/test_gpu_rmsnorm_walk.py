"""The norm's gradient where a workgroup takes several rows, one after the other with the next one's loads ahead, in every form that the kernel has; and leaves partial sums behind."""
import numpy as np
import pytest
import torch

import block_math as bm
from paper_2509_25149_amd import binding as nv
from test_gpu_rmsnorm import BF16, EPS, F32, OUT, activations, backward_tolerance

pytestmark = pytest.mark.gpu
# rows, columns, workgroups, rows that a workgroup takes at a time: a wavefront per row with one chunk and two; a workgroup per row with one chunk, two with up to 512 threads and
# with more, four (sums in LDS).  Even and uneven shares, the last workgroups with a row less than the first.
WALKS = [(4500, 256, 1024, 4), (8200, 496, 768, 4), (2050, 528, 512, 4), (1027, 1024, 256, 4), (2100, 1008, 512, 4), (1300, 1040, 1024, 1), (1100, 2048, 512, 1), (1025, 2064, 512, 1),
         (600, 5120, 256, 1), (257, 8192, 256, 1), (300, 8208, 256, 1), (520, 12304, 256, 1), (300, 16384, 256, 1), (300, 16400, 256, 1), (260, 32768, 256, 1), (515, 20480, 256, 1)]


@pytest.mark.parametrize("rows,cols,parts,each", WALKS)
@pytest.mark.parametrize("dt,st,saved8,gamma,res,pad", [(BF16, BF16, True, True, True, 0), (BF16, F32, False, True, True, 8), (F32, F32, False, False, False, 0), (F32, BF16, True, True, False, 8),
                                                        (BF16, BF16, False, False, True, 0), (F32, F32, True, True, True, 0)])
def test_backward_over_several_rows(rows, cols, parts, each, dt, st, saved8, gamma, res, pad):
    assert nv.rowsum_workspace_bytes(rows, cols) == parts * cols * 4 and parts > 1 and parts * each < rows
    r = np.random.default_rng(rows * 3 + cols)
    h = bm.tensor(activations(rows, cols, 5, st), st, pad)
    gt = torch.as_tensor((1 + 0.1 * r.standard_normal(cols)).astype(np.float32)).cuda() if gamma else None
    fwd = nv.nvfp4_rmsnorm_forward(h, gt, eps=EPS, checkpoint=True)
    dy = bm.tensor(1e-3 * r.standard_t(3, (rows, cols)), dt, pad)
    dres = bm.tensor(1e-3 * r.standard_t(3, (rows, cols)), st, pad) if res else None
    saved = fwd.checkpoint if saved8 else h
    dx, dgamma = nv.nvfp4_rmsnorm_backward(dy, saved, fwd.rstd, gt, dres=dres, dx_dtype=OUT[st])
    rstd = bm.f64(fwd.rstd)
    xhat = bm.decode(saved.codes.cpu().numpy(), saved.scales.cpu().numpy()) if saved8 else bm.f64(h) * rstd[:, None]
    d64, g64, r64 = bm.f64(dy), None if gt is None else bm.f64(gt), None if dres is None else bm.f64(dres)
    ref, ref_gamma = bm.norm_backward(d64, xhat, rstd, g64, r64)
    bm.within(dx, ref, backward_tolerance(d64, xhat, rstd, d64 if g64 is None else d64 * g64, r64, ref) + bm.rounding(ref, st))
    # a lane's rows, the wavefronts of a workgroup, a sixteenth of the parts, sixteen of those; xhat's and the product's own rounding
    depth = -(-rows // (parts * each)) + 4 + -(-parts // 16) + 16 + 2
    tol = depth * 2.0 ** -24 * np.abs(d64 * xhat).sum(0) + 1e-37
    bm.within(dgamma, ref_gamma, tol)
    # the same bits again, added to what was there, and over an input
    old = torch.as_tensor(r.standard_normal(cols).astype(np.float32)).cuda()
    before, over = bm.f64(old), dres if res else dy if dt == st else None
    dx2, grown = nv.nvfp4_rmsnorm_backward(dy, saved, fwd.rstd, gt, dres=dres, dx=over, dx_dtype=OUT[st], dgamma=old, accumulate_dgamma=True)
    assert torch.equal(dx2, dx) and (over is None or dx2 is over)
    bm.within(grown, ref_gamma + before, tol + 2.0 ** -23 * (np.abs(before) + np.abs(ref_gamma)))


def test_rows_whose_squares_overflow():
    """FP32's largest number is 3.4e38: from 1.8e19 on a square is infinite, and what it is the norm of comes out as 0; the rows beside it are as ever."""
    x = torch.ones(3, 2064, device="cuda")
    x[1, 7] = 1.9e19
    out = nv.nvfp4_rmsnorm_forward(x, y_dtype=nv.OUT_F32, checkpoint=True)
    assert float(out.rstd[1]) == 0 and bool((out.y[1] == 0).all()) and bool((out.checkpoint.scales[1] == 0).all())
    assert torch.allclose(out.y[[0, 2]], x[[0, 2]], atol=1e-5)
