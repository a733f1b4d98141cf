"""Log probabilities where the launch takes another shape than for the sizes of test_gpu_logprob.py: rows cut into pieces (fewer than 96 rows of 65536 columns and more: 64 pieces
down to 10), and loss and gradient of long rows by 512 and 1024 threads, in every pair of types."""
import numpy as np
import pytest
import torch

import block_math as bm
import ends_math as em
import test_gpu_logprob as base
from paper_2509_25149_amd import binding as nv

pytestmark = pytest.mark.gpu
F32, BF16, I32, I64 = torch.float32, torch.bfloat16, torch.int32, torch.int64
CUT = [(2, 65536), (17, 70001), (33, 65537), (40, 90001), (95, 65544), (95, 131073)]      # 64, 60, 31, 25, 10 and 10 pieces


@pytest.mark.parametrize("rows,cols", CUT)
@pytest.mark.parametrize("dt,it,scale,entropy,top,kind", [(BF16, I64, 1.0, True, 32, "plain"), (F32, I32, 0.7, False, 31, "masked"), (F32, I64, 1.25, True, 1, "far"),
                                                          (BF16, I32, 1.0, False, 0, "masked")])
def test_rows_in_pieces(rows, cols, dt, it, scale, entropy, top, kind):
    z, t = base.logits(rows, cols, rows + cols, dt, 8, kind), base.targets_of(rows, cols, 1)
    base.check_forward(nv.nvfp4_logprob_forward(z, em.index(t, it), scale=scale, entropy=entropy, top=top, for_backward=True), z, scale, t, top, entropy)


@pytest.mark.parametrize("rows,cols", CUT[:4])
@pytest.mark.parametrize("dt,ot,it,scale,kind", [(BF16, BF16, I64, 1.0, "plain"), (F32, F32, I32, 0.7, "masked"), (BF16, F32, I64, 1.0, "far"), (F32, BF16, I32, 1.5, "plain")])
def test_loss_and_gradient_of_rows_in_pieces(rows, cols, dt, ot, it, scale, kind):
    base.test_loss_and_gradient_together(rows, cols, dt, ot, it, scale, kind)


@pytest.mark.parametrize("rows,cols", [(6, 70001), (40, 65537)])
@pytest.mark.parametrize("dt", [F32, BF16])
def test_pieces_that_masks_leave_nothing_of(rows, cols, dt):
    base.test_rows_that_masks_leave_nothing_of(rows, cols, dt)


@pytest.mark.parametrize("rows,cols", [(4, 65537), (40, 70001)])
def test_trouble_in_a_piece_shows_in_its_row_and_nowhere_else(rows, cols):
    base.test_trouble_shows_in_its_row_and_nowhere_else(rows, cols)


@pytest.mark.parametrize("top", [1, 2, 31, 32])
@pytest.mark.parametrize("rows,cols", [(40, 65600), (7, 70001)])
def test_best_alternatives_of_pieces_where_many_are_equal(rows, cols, top):
    base.test_best_alternatives_where_many_are_equal(rows, cols, top)


# 1024 threads: bf16 rows of more than 160 KB (with 2048 rows of more than 72 KB), FP32 rows half as long; 512: FP32 rows of 20003.  Whole groups of eight columns and broken ones.
@pytest.mark.parametrize("rows,cols", [(97, 90001), (96, 131072), (100, 20003), (2048, 36873)])
@pytest.mark.parametrize("dt,ot,scale,kind", [(BF16, BF16, 1.0, "plain"), (F32, F32, 0.7, "masked"), (BF16, F32, 1.25, "masked"), (F32, BF16, 1.0, "far")])
def test_loss_and_gradient_of_long_rows(rows, cols, dt, ot, scale, kind):
    """Row r is row r % 16 again, so that 16 are compared with 64 bits and the others have to be the same bits."""
    few = 16
    z = base.logits(few, cols, cols, dt, 8, kind)
    t, r = base.targets_of(few, cols, 3), np.random.default_rng(cols)
    g = torch.as_tensor((-r.random(few) / few).astype(np.float32)).cuda()
    again = torch.arange(rows, device="cuda") % few
    wide = z.as_strided((few, z.stride(0)), (z.stride(0), 1))[again]
    many, targets = wide[:, :cols], em.index(t, I64)[again]
    out = nv.nvfp4_logprob_with_gradient(many, targets, g[again], scale=scale, out_dtype=base.OUT[ot])
    for whole, row in ((out.logprob, out.logprob[:few]), (out.lse, out.lse[:few]), (out.dlogits, out.dlogits[:few])):
        assert torch.equal(whole, row[again])
    first = nv.LogProbs(out.logprob[:few], out.lse[:few])
    base.check_forward(first, z, scale, t, 0, False)
    base.check_gradient(out.dlogits[:few], z, scale, t, g, None, None, ot)
    if dt == ot:
        over = nv.nvfp4_logprob_with_gradient(many, targets, g[again], scale=scale, out=many)
        assert over.dlogits is many and torch.equal(many, out.dlogits) and torch.equal(over.logprob, out.logprob) and torch.equal(over.lse, out.lse)
        assert torch.isnan(wide[:, cols:]).all()
