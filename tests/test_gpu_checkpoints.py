"""8-bit checkpoints on the GPU: save, load with activation and column factor, the activation's gradient with the bias gradient."""
import numpy as np
import pytest
import torch

import block_math as bm
from paper_2509_25149_amd import binding as nv

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
OUT = {F32: nv.OUT_F32, BF16: nv.OUT_BF16}
# one row; fewer and more rows than a workgroup takes; columns at and beside the width of a strip (512), one block
SHAPES = [(1, 16), (1, 5120), (3, 48), (4, 512), (5, 528), (17, 496), (130, 1040), (1027, 1296), (64, 20480)]


def values(rows, cols, seed, dtype=BF16):
    """Activations, with blocks of zeros, of tiny and of huge numbers, and of single values."""
    r = np.random.default_rng(seed)
    v = r.standard_normal((rows, cols)) * np.where(r.random((rows, cols)) < 0.01, 50, 1)
    scale = np.exp2(r.integers(-100, 100, (rows, cols // 16))) * (r.random((rows, cols // 16)) < 0.2)
    v = v * np.repeat(np.where(scale > 0, scale, 1), 16, 1)
    v[:, :16] = np.where(r.random((rows, 1)) < 0.3, 0, v[:, :16])
    return bm.f64(torch.as_tensor(v.astype(np.float32)).to(dtype))


def kept(rows, cols, seed):
    """A checkpoint of activations near 1, and its values."""
    r = np.random.default_rng(seed)
    v = r.standard_normal((rows, cols)) * np.where(r.random((rows, cols)) < 0.02, 20, 1)
    c = nv.nvfp4_checkpoint_save(bm.tensor(v, F32))
    return c, bm.decode(c.codes.cpu().numpy(), c.scales.cpu().numpy())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad", [0, 8])
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_save_is_the_definition_byte_for_byte(rows, cols, pad, dtype):
    v = values(rows, cols, rows + cols, dtype)
    c = nv.nvfp4_checkpoint_save(bm.tensor(v, dtype, pad))
    codes, scales = bm.encode(v)
    assert np.array_equal(c.scales.cpu().numpy(), scales)
    assert np.array_equal(c.codes.cpu().numpy(), codes)


def test_save_at_the_limits_of_a_scale():
    """Largest magnitudes at, just below and just above 448 * 2^e, over all exponents, and every code's neighbourhood."""
    rows = []
    for e in range(-149, 120):
        for m in (448.0, np.nextafter(np.float32(448.0), np.float32(0)), np.nextafter(np.float32(448.0), np.float32(500)), 449.0, 256.0, 255.0):
            row = np.zeros(16)
            row[3] = np.float64(m) * 2.0 ** e
            row[5] = -row[3] / 2
            row[6] = row[3] * 2.0 ** -9 * 1.5
            rows.append(row)
    ties = (bm.E4M3[1:] + bm.E4M3[:-1]) / 2
    for t in ties:
        for f in (1.0, 1 - 2.0 ** -20, 1 + 2.0 ** -20):
            rows.append(np.array([448.0, t * f, -t * f] + [0.0] * 13))
    v = np.array(rows, np.float32).astype(np.float64)
    c = nv.nvfp4_checkpoint_save(bm.tensor(v, F32))
    codes, scales = bm.encode(v)
    assert np.array_equal(c.scales.cpu().numpy(), scales)
    assert np.array_equal(c.codes.cpu().numpy(), codes)


def test_blocks_that_hold_infinities_or_nans_read_back_as_nan():
    v = np.ones((4, 64))
    v[0, 5], v[1, 20], v[2, 63] = np.inf, -np.inf, np.nan
    for dtype in (F32, BF16):
        c = nv.nvfp4_checkpoint_save(bm.tensor(v, dtype))
        bad = ~np.isfinite(v).reshape(4, 4, 16).all(-1)
        assert np.array_equal(c.scales.cpu().numpy() == 255, bad)
        out = bm.f64(nv.nvfp4_checkpoint_load(c, out_dtype=nv.OUT_F32))
        assert np.array_equal(np.isnan(out), np.repeat(bad, 16, 1)) and np.all(out[~np.repeat(bad, 16, 1)] == 1)
        for act in (nv.ACT_RELU2, nv.ACT_GELU, nv.ACT_SILU):      # no activation and no derivative hides them
            assert np.array_equal(np.isnan(bm.f64(nv.nvfp4_checkpoint_load(c, act))), np.repeat(bad, 16, 1))
            dz, _ = nv.nvfp4_activation_backward(torch.ones(4, 64, device="cuda"), c, act)
            assert np.array_equal(np.isnan(bm.f64(dz)), np.repeat(bad, 16, 1))


@pytest.mark.parametrize("name", list(bm.ACTS))
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols,pad,factor", [(1, 16, 0, False), (5, 528, 8, True), (130, 1040, 0, True), (64, 20480, 0, False)])
def test_load(rows, cols, pad, factor, dtype, name):
    c, z = kept(rows, cols, 7 * rows + cols)
    f = np.random.default_rng(1).standard_normal(cols).astype(np.float32) if factor else None
    out = bm.tensor(np.zeros((rows, cols)), dtype, pad)
    nv.nvfp4_checkpoint_load(c, bm.ACTS[name], None if f is None else torch.as_tensor(f).cuda(), out=out)
    ref = bm.act(z, name) * (1 if f is None else f.astype(np.float64))
    tol = bm.act_tolerance(z, name) * (1 if f is None else np.abs(f)) + bm.rounding(ref, F32) + bm.rounding(ref, dtype)
    bm.within(out, ref, tol)
    if pad:
        assert torch.isnan(out.as_strided((rows, pad), out.stride(), cols)).all()


@pytest.mark.parametrize("name", list(bm.ACTS))
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols,pad", [(1, 16, 0), (3, 48, 8), (5, 528, 0), (130, 1040, 8), (1027, 1296, 0), (4100, 512, 0)])
def test_activation_backward(rows, cols, pad, dtype, name):
    c, z = kept(rows, cols, 3 * rows + cols)
    r = np.random.default_rng(5)
    da = bm.tensor(1e-3 * r.standard_t(3, (rows, cols)), dtype, pad)
    old = r.standard_normal(cols).astype(np.float32)
    dz, dbias = nv.nvfp4_activation_backward(da, c if name != "none" else None, bm.ACTS[name])
    ref = bm.f64(da) * bm.slope(z, name)
    each = np.abs(bm.f64(da)) * bm.slope_tolerance(z, name) + bm.rounding(ref, F32)
    bm.within(dz, ref, each + bm.rounding(ref, dtype))
    # a sum of n numbers in FP32 along a tree of depth d is off by at most d 2^-24 of the sum of magnitudes: a lane's rows, its workgroup, the parts
    depth = -(-rows // 4) + 4 + 64
    tol = each.sum(0) + depth * 2.0 ** -24 * np.abs(ref).sum(0) + 1e-37
    bm.within(dbias, ref.sum(0), tol)
    grown = torch.as_tensor(old).cuda()
    again = nv.nvfp4_activation_backward(da, c if name != "none" else None, bm.ACTS[name], want_dz=False, dbias=grown, accumulate_dbias=True)
    assert again[0] is None and again[1] is grown
    bm.within(grown, ref.sum(0) + old, tol + 2.0 ** -23 * (np.abs(old) + np.abs(ref.sum(0))))
    # the same bits again, without the sum, and over its own input
    dz2, none = nv.nvfp4_activation_backward(da, c if name != "none" else None, bm.ACTS[name], bias_grad=False)
    assert none is None and torch.equal(dz, dz2)
    assert torch.equal(dbias, nv.nvfp4_activation_backward(da, c if name != "none" else None, bm.ACTS[name])[1])
    nv.nvfp4_activation_backward(da, c if name != "none" else None, bm.ACTS[name], dz=da)
    assert torch.equal(da, dz)


@pytest.mark.parametrize("name", ["relu2", "gelu", "silu"])
def test_the_derivative_agrees_with_differences(name):
    c, z = kept(64, 512, 11)
    dz, _ = nv.nvfp4_activation_backward(torch.ones(64, 512, device="cuda"), c, bm.ACTS[name])
    d = 1e-5 * np.maximum(1, np.abs(z))
    diff = (bm.act(z + d, name) - bm.act(z - d, name)) / (2 * d)
    # central differences: d^2 / 6 times a third derivative below 2, the rounding of both values over 2 d, half of relu2's kink at 0
    tol = d * d + 2.0 ** -51 * (np.abs(bm.act(z, name)) + 1) / d + (d if name == "relu2" else 0) + bm.slope_tolerance(z, name)
    bm.within(dz, diff, tol)


@pytest.mark.parametrize("name", ["gelu", "silu", "relu2"])
def test_far_from_zero(name):
    """Where exponentials and powers overflow the derivative is 0 or 1 (2 z), and the function 0 or z (z^2)."""
    z = np.zeros((1, 32), np.float32)
    z[0, :16], z[0, 16:] = -1e15, 1e15
    c = nv.nvfp4_checkpoint_save(bm.tensor(z, F32))
    kept_z = bm.decode(c.codes.cpu().numpy(), c.scales.cpu().numpy())
    out = bm.f64(nv.nvfp4_checkpoint_load(c, bm.ACTS[name], out_dtype=nv.OUT_F32))
    dz = bm.f64(nv.nvfp4_activation_backward(torch.ones(1, 32, device="cuda"), c, bm.ACTS[name])[0])
    assert np.all(out[0, :16] == 0) and np.all(dz[0, :16] == 0)
    if name == "relu2":
        assert np.allclose(out[0, 16:], kept_z[0, 16:] ** 2, rtol=1e-6) and np.allclose(dz[0, 16:], 2 * kept_z[0, 16:], rtol=1e-6)
    else:
        assert np.all(out[0, 16:] == kept_z[0, 16:]) and np.all(dz[0, 16:] == 1)


def test_tensors_without_rows():
    x = torch.empty(0, 64, device="cuda", dtype=BF16)
    c = nv.nvfp4_checkpoint_save(x)
    assert nv.nvfp4_checkpoint_load(c).shape == (0, 64)
    dz, dbias = nv.nvfp4_activation_backward(x, c, nv.ACT_GELU)
    assert dz.shape == (0, 64) and torch.equal(dbias, torch.zeros(64, device="cuda"))
    old = torch.ones(64, device="cuda")
    nv.nvfp4_activation_backward(x, c, nv.ACT_GELU, dbias=old, accumulate_dbias=True)
    assert torch.equal(old, torch.ones(64, device="cuda"))


def test_on_another_stream_and_within_the_workspace():
    rows, cols = 1027, 1296
    c, z = kept(rows, cols, 2)
    da = bm.tensor(np.random.default_rng(3).standard_normal((rows, cols)), BF16)
    want = nv.nvfp4_activation_backward(da, c, nv.ACT_SILU)
    need = nv.rowsum_workspace_bytes(rows, cols)
    buf = torch.full((need + 4096,), 0xAB, dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = nv.nvfp4_activation_backward(da, c, nv.ACT_SILU, workspace=buf[:need])
    s.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert torch.all(buf[need:] == 0xAB)


def test_offsets_beyond_32_bits():
    """40000 x 65536: 2.6e9 elements; the last rows are where they belong."""
    rows, cols = 40000, 65536
    x = torch.zeros(rows, cols, dtype=BF16, device="cuda")
    v = values(2, cols, 9)
    x[-2:] = bm.tensor(v, BF16)
    c = nv.nvfp4_checkpoint_save(x)
    codes, scales = bm.encode(v)
    assert np.array_equal(c.scales[-2:].cpu().numpy(), scales) and np.array_equal(c.codes[-2:].cpu().numpy(), codes)
    assert int(c.scales[:-2].max()) == 0
    nv.nvfp4_checkpoint_load(c, out=x)
    ref = bm.decode(codes, scales)
    bm.within(x[-2:], ref, bm.rounding(ref, BF16))
    dz, dbias = nv.nvfp4_activation_backward(x, dz=x)
    bm.within(dbias, bm.f64(x[-2:]).sum(0), 2.0 ** -22 * np.abs(bm.f64(x[-2:])).sum(0))
