"""CPU: nvfp4_gemm_epilogue refuses results whose rows or columns are not multiples of 16 -- its output stages work on whole 16 x 16 blocks -- before anything is enqueued."""
import ctypes

import pytest

from paper_2509_25149_amd import binding as nv

P = 0x10000      # fake, aligned, never dereferenced by the checks
BAD_SHAPE, MISMATCH = -2, -4


def operand(outer, k):
    d = nv.QTensorStruct()
    d.rows, d.cols, d.layout_mask, d.block_dim = outer, k, nv.LAYOUT_ROW, nv.BLOCK_1x16
    d.row_codes = d.row_scales = d.row_tensor_scale = P
    return d


def call(m, n, k=64, **fields):
    a, b, e = operand(m, k), operand(n, k), nv.EpilogueStruct(**fields)
    return nv.load_library().nvfp4_gemm_epilogue(ctypes.byref(a), ctypes.byref(b), nv.OP_DGRAD, ctypes.byref(e), P, nv.OUT_F32, -(-n // 8) * 8, None, 0, None)


@pytest.mark.parametrize("m,n", [(0, 48), (20, 48), (1, 48), (15, 48), (4100, 5120), (32, 40), (32, 8), (4100, 5128), (32, 0), (2064, 4104)])
def test_sizes_that_are_not_whole_blocks_are_refused(m, n):
    kept = ctypes.pointer(nv.CheckpointStruct(m, n, P, P))
    for fields in ({}, dict(bias=P, activation=nv.ACT_GELU), dict(residual=P, ldr=-(-n // 8) * 8), dict(keep=kept), dict(grad_of=kept, activation=nv.ACT_RELU2)):
        assert call(m, n, **fields) == BAD_SHAPE, fields


def test_whole_blocks_pass_this_check():
    assert call(32, 48, keep=ctypes.pointer(nv.CheckpointStruct(32, 64, P, P))) == MISMATCH      # what is refused here is looked at behind the sizes
