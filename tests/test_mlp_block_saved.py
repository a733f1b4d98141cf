"""What examples/mlp_block.py keeps for the backward pass: no descriptor points to memory that was given back."""
import ctypes
import importlib.util
import os

import pytest
import torch

from paper_2509_25149_amd import binding as nv

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
POINTERS = {"row_codes": "row_codes", "row_scales": "row_scales", "row_tensor_scale": "row_ts", "col_codes": "col_codes", "col_scales": "col_scales", "col_tensor_scale": "col_ts"}


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("mlp_block_saved", os.path.join(ROOT, "examples", "mlp_block.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def points_only_to_what_it_holds(q):
    for field, name in POINTERS.items():
        held = getattr(q, name)
        assert getattr(q.desc, field) == (None if held is None else held.data_ptr()), field


def test_a_copy_that_was_given_back_is_refused(example):
    q, w = (nv.alloc_qtensor(32, 32, nv.LAYOUT_ROW | nv.LAYOUT_COL, device="cpu") for _ in range(2))
    q.desc.layout_mask = w.desc.layout_mask = nv.LAYOUT_ROW | nv.LAYOUT_COL
    assert example.keep_col_copy(q) is q
    points_only_to_what_it_holds(q)
    assert q.col_codes is not None and q.desc.layout_mask == nv.LAYOUT_COL
    for op in (nv.OP_FPROP, nv.OP_DGRAD):
        assert nv.load_library().nvfp4_gemm(ctypes.byref(q.desc), ctypes.byref(w.desc), op, 0x10000, nv.OUT_F32, 32, None, 0, None) == -3      # no such copy


@pytest.mark.gpu
def test_what_the_forward_pass_keeps(example):
    block = example.MlpBlock(512, 1024)
    x, r = (torch.randn(256, 512, device="cuda").bfloat16() for _ in range(2))
    _, (_, _, qn, _, qa) = block.forward(x, r)
    for q in (qn, qa):
        points_only_to_what_it_holds(q)
        with pytest.raises(nv.NVFP4Error):
            nv.nvfp4_gemm(q, block.q1, nv.OP_FPROP)
