"""nvfp4_gemm_epilogue on operands that nvfp4_predecode has decoded beforehand: one of them or both, with room for the rest, for the partial tiles, or for neither."""
import pytest
import torch

from paper_2509_25149_amd import binding as nv
from test_gpu_gemm_epilogue import BF16, F32, Product, act64, act_bound, check_kept, close, decode, slope64, ulp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k", [(64, 336, 256), (256, 256, 512), (7760, 1568, 512), (2048, 5120, 5120), (2064, 5136, 4096), (8192, 2576, 2048), (2944, 8192, 1024)])
@pytest.mark.parametrize("row_scales", [False, True])
@pytest.mark.parametrize("which", ["a", "b", "ab"])
def test_the_same_result_from_decoded_operands(m, n, k, which, row_scales):
    p = Product(m, n, k, row_scales=row_scales, seed=12)
    for name in which:
        nv.nvfp4_predecode(getattr(p, name), nv.COPY_ROW)
    bias, res = p.normal(n), p.normal(m, n).to(BF16)
    z = p.z + bias.double()
    tol = p.tol + 2.0 ** -23 * (p.z.abs() + z.abs())
    for workspace in (False, True):
        keep = nv.alloc_checkpoint(m, n)
        out = p.run(workspace, bias=bias, activation=nv.ACT_GELU, keep=keep, out_dtype=nv.OUT_F32)
        ref = act64(z, "gelu")
        close(out, ref, 1.2 * tol + act_bound(z, "gelu") + ulp(ref, F32))
        check_kept(keep, z, tol)
        out = p.run(workspace, bias=bias, residual=res, out_dtype=nv.OUT_BF16)
        ref = z + res.double()
        close(out, ref, tol + 2.0 ** -23 * ref.abs() + ulp(ref, BF16))
        out = p.run(workspace, activation=nv.ACT_RELU2, grad_of=keep, out_dtype=nv.OUT_F32)
        s = slope64(decode(keep), "relu2")
        close(out, p.z * s, (p.tol + 2.0 ** -22 * p.z.abs()) * s.abs() + 1e-37)
