"""Log probabilities at the ends of what a scale, the logits and the gradients may be."""
import numpy as np
import pytest
import torch

import block_math as bm
import ends_math as em
import test_gpu_logprob as base
from paper_2509_25149_amd import binding as nv

pytestmark = pytest.mark.gpu
F32, BF16, I32, I64 = torch.float32, torch.bfloat16, torch.int32, torch.int64
# 64 threads to a row; 256; 512 of the loss; rows cut into pieces
SHAPES = [(5, 24), (6, 9001), (40, 20000), (3, 70001)]


def vectors(rows, seed, size=1.0):
    r = np.random.default_rng(seed)
    return [torch.as_tensor((size * r.standard_normal(rows)).astype(np.float32)).cuda() for _ in range(3)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dt", [F32, BF16])
@pytest.mark.parametrize("scale", [0.5, 1e-37, 1e-38, 2.0 ** -127, 1e-40, 1e-45])
def test_differences_beyond_fp32_at_a_small_scale(rows, cols, dt, scale):
    """scale (z - max) may be small where z - max is beyond FP32's range.  (A scale below 2^-126 has fewer bits in its base-2 form: that moves an exponent by at most 2^129 2^-150 = 2^-21,
    4.8e-7, against the 160 U = 9.5e-6 that a row's sum is allowed.)  Gradients of size 1e30, so that the logits' are not lost in what is allowed for underflow."""
    scale = float(np.float32(scale))
    r = np.random.default_rng(cols)
    v = r.choice([3e38, 1e38, 0.0, -1e38, -3e38, -np.inf], (rows, cols))
    v[:, 1], v[:, 2] = 3e38, -3e38
    v[0, 3] = float(torch.finfo(dt).min)
    z, t = bm.tensor(v, dt, base.pad_of(cols, 8)), base.targets_of(rows, cols, 1)
    t[:2] = 2
    g, gl, ge = vectors(rows, cols, 1e30)
    out = nv.nvfp4_logprob_forward(z, em.index(t, I64), scale=scale, entropy=True, top=5, for_backward=True)
    base.check_forward(out, z, scale, t, 5, True)
    dz = nv.nvfp4_logprob_backward(z, em.index(t, I64), out.stats, g_logprob=g, g_lse=gl, g_entropy=ge, entropy=out.entropy, scale=scale)
    base.check_gradient(dz, z, scale, t, g, gl, ge, dt)
    one = nv.nvfp4_logprob_with_gradient(z, em.index(t, I64), g, scale=scale)
    base.check_forward(one, z, scale, t, 0, False)
    base.check_gradient(one.dlogits, z, scale, t, g, None, None, dt)


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dt,ot", [(F32, F32), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("scale,size", [(2.0 ** 122, 1.0), (2.0 ** 127, 1.0), (2.0 ** 64, 2.0 ** 63), (1.0, 2.0 ** 126), (2.0 ** -100, 2.0 ** 126)])
def test_gradients_near_the_end_of_fp32(rows, cols, dt, ot, scale, size):
    """scale times a gradient may be beyond FP32 where p makes it small again, and a probability of 0 makes a 0 of it: columns masked by -infinity or the type's lowest value, or
    far below the others.  The logits that count are k / scale apart, k up to 30."""
    r = np.random.default_rng(cols)
    v = np.full((rows, cols), -np.inf)
    v[:, 4:8] = float(torch.finfo(dt).min) if scale >= 1 else -3e38
    v[:, 8:12] = -256 / scale
    v[:, 12:20] = -r.integers(3, 30, (rows, 8)) / scale
    v[:, cols - 3] = -4 / scale
    v[:, 2] = 0.0
    z = bm.tensor(v, dt, base.pad_of(cols, 8))
    t = np.full(rows, 2)
    t[rows // 2] = -1
    t[0] = 0                                                  # masked
    g, gl, ge = (torch.full((rows,), a * size, device="cuda") for a in (3.0, 0.2, 0.25))
    g[0] = 0.5 * size
    out = nv.nvfp4_logprob_forward(z, em.index(t, I32), scale=scale, entropy=True, for_backward=True)
    base.check_forward(out, z, scale, t, 0, True)
    for use in ((g, None, None), (g, gl, ge), (None, None, ge)):
        dz = nv.nvfp4_logprob_backward(z, em.index(t, I32), out.stats, g_logprob=use[0], g_lse=use[1], g_entropy=use[2], entropy=out.entropy, scale=scale, out_dtype=base.OUT[ot])
        assert bool(torch.isfinite(dz).all())
        base.check_gradient(dz, z, scale, t, *use, ot)
    one = nv.nvfp4_logprob_with_gradient(z, em.index(t, I32), g, scale=scale, out_dtype=base.OUT[ot])
    assert bool(torch.isfinite(one.dlogits).all())
    base.check_gradient(one.dlogits, z, scale, t, g, None, None, ot)
