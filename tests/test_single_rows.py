"""One row, cut from a wider tensor: how far apart rows would be says nothing then, and torch leaves it open."""
import pytest
import torch

from paper_2509_25149_amd import binding as nv


class OnGpu(torch.Tensor):
    is_cuda = property(lambda self: True)


@pytest.mark.parametrize("stride", [64, 100, 67, 65, 16, 1, 0])
def test_the_leading_dimension_of_a_single_row_is_its_length(stride):
    row = torch.zeros(256).as_strided((1, 64), (stride, 1)).as_subclass(OnGpu)
    assert nv._matrix(row, "x") == (nv.OUT_F32, row.data_ptr(), 64)
    rows = torch.zeros(256).as_strided((2, 64), (72, 1)).as_subclass(OnGpu)
    assert nv._matrix(rows, "x")[2] == 72


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_calls_on_a_row_of_a_wider_tensor(dtype):
    cols = 5120
    wide = torch.randn(1, cols + 37, device="cuda").to(dtype)
    x, y = wide[:, :cols], torch.zeros(1, cols + 37, device="cuda", dtype=dtype)[:, :cols]
    c, r = x.contiguous(), torch.randn(1, cols, device="cuda").to(dtype)
    assert x.stride(0) % 8 == 5
    out = nv.OUT_F32 if dtype == torch.float32 else nv.OUT_BF16
    want = nv.nvfp4_rmsnorm_forward(c, residual=r, y_dtype=out, checkpoint=True)
    got = nv.nvfp4_rmsnorm_forward(x, residual=r, y=y, checkpoint=True)
    assert got.y is y and torch.equal(y, want.y) and torch.equal(got.h, want.h) and torch.equal(got.checkpoint.codes, want.checkpoint.codes)
    for a, b in zip(nv.nvfp4_rmsnorm_backward(x, want.checkpoint, want.rstd, dres=x, dx=y), nv.nvfp4_rmsnorm_backward(c, want.checkpoint, want.rstd, dres=c)):
        assert torch.equal(a, b)
    assert torch.equal(nv.nvfp4_checkpoint_save(x).codes, nv.nvfp4_checkpoint_save(c).codes)
    assert torch.equal(nv.nvfp4_checkpoint_load(want.checkpoint, out=y), nv.nvfp4_checkpoint_load(want.checkpoint, out_dtype=out))
    for a, b in zip(nv.nvfp4_activation_backward(x, want.checkpoint, nv.ACT_GELU, dz=y), nv.nvfp4_activation_backward(c, want.checkpoint, nv.ACT_GELU)):
        assert torch.equal(a, b)
