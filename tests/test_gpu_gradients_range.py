"""Clipping where the factor itself is below FP32's normal numbers."""
import numpy as np
import pytest
import torch

import block_math as bm
import ends_math as em
from paper_2509_25149_amd import binding as nv

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("max_norm", [1.0, 1e-3, 1e-7, 1e-30, 1e-37])
@pytest.mark.parametrize("dt,ot,in_place", [(F32, F32, True), (BF16, BF16, True), (F32, F32, False), (BF16, BF16, False), (F32, BF16, False), (BF16, F32, False)])
def test_a_large_norm_and_a_small_bound(max_norm, dt, ot, in_place):
    """data max_norm / norm is a normal number for the large values, whatever the factor is.  The factor is rounded once, the product once, and a result below FP32's normal numbers (2^-126) is off by
    up to two halves of 2^-149, in bf16 by a half of 2^-133."""
    r = np.random.default_rng(1)
    big = torch.as_tensor((2.9e38 * r.uniform(0.5, 1.0, 5003)).astype(np.float32)).cuda().to(dt)
    wide = torch.zeros(33, 300, device="cuda", dtype=dt)
    wide[:, :101] = torch.as_tensor((1e30 * r.standard_normal((33, 101))).astype(np.float32)).cuda().to(dt)
    grads = [big, wide[:, :101], torch.ones(3, device="cuda", dtype=dt)]
    before = [bm.f64(g) for g in grads]
    norm = np.sqrt(sum((b ** 2).sum() for b in before))
    outs = None if in_place else [torch.full(g.shape, 7.0, device="cuda", dtype=ot) for g in grads]
    n = nv.Gradients(grads, outs)
    nv.nvfp4_grad_clip(n, nv.nvfp4_grad_sumsq(n), max_norm)
    least = 2.0 ** -149 + (2.0 ** -134 if ot == BF16 else 0.0)
    for o, b in zip(grads if in_place else outs, before):
        ref = b * (float(np.float32(max_norm)) / norm)
        half = 2.0 ** -8 if ot == BF16 else 0.0
        bm.within(o.reshape(-1), ref.reshape(-1), ((2 * em.U + half) * 1.01 * np.abs(ref) + least).reshape(-1))
