"""nvfp4_gemm_epilogue on the GPU against binary64 products of the decoded operands: every kernel that a product can take, each kind of epilogue."""
import ctypes

import numpy as np
import pytest
import torch

import block_math as bm
from paper_2509_25149_amd import binding as nv

pytestmark = pytest.mark.gpu
F32, BF16 = torch.float32, torch.bfloat16
OUT = {F32: nv.OUT_F32, BF16: nv.OUT_BF16}
ROW = nv.LAYOUT_ROW


class Product:
    """Operands of an [m, n, k] Dgrad-shaped product (both row copies) and its exact value (on the GPU in float64)."""

    def __init__(self, m, n, k, mx=False, row_scales=False, seed=1):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        x = torch.randn(m, k, generator=g, device="cuda")
        x = torch.where(torch.rand(m, k, generator=g, device="cuda") < 1e-3, 20 * x, x).to(BF16)
        w = (torch.randn(n, k, generator=g, device="cuda") / k ** 0.5).to(BF16)
        block = nv.BLOCK_MX32 if mx else nv.BLOCK_1x16
        self.a = nv.nvfp4_quantize(x, ROW | (nv.LAYOUT_ROW_SCALES if row_scales else 0), block)
        self.b = nv.nvfp4_quantize(w, ROW, block if mx else nv.BLOCK_16x16)
        da, db = (nv.nvfp4_dequantize(q, nv.COPY_ROW, out_dtype=nv.OUT_F32).double() for q in (self.a, self.b))
        self.z = da @ db.t()
        # an FP32 sum of k products along a chain of k / 16 matrix instructions and the splits of K
        self.tol = (k / 16 + 16) * 2.0 ** -24 * (da.abs() @ db.abs().t())
        self.m, self.n, self.k = m, n, k
        self.g = g

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda")

    def run(self, workspace, op=nv.OP_DGRAD, **kw):
        ws = torch.empty(nv.gemm_workspace_bytes(self.m, self.n, self.k), dtype=torch.uint8, device="cuda") if workspace else None
        return nv.nvfp4_gemm_epilogue(self.a, self.b, op, workspace=ws, **kw)


def act64(z, name):
    if name == "relu2":
        return torch.where(z > 0, z * z, torch.zeros_like(z))
    if name == "none":
        return z
    return z / (1 + torch.exp(-arg64(z, name)))


def arg64(z, name):
    return z if name == "silu" else 2 * (2 / np.pi) ** 0.5 * (z + 0.044715 * z ** 3)


def slope64(z, name):
    if name == "relu2":
        return torch.where(z > 0, 2 * z, torch.zeros_like(z))
    if name == "none":
        return torch.ones_like(z)
    p = arg64(z, name)
    dp = 1.0 if name == "silu" else 2 * (2 / np.pi) ** 0.5 * (1 + 3 * 0.044715 * z * z)
    s = torch.sigmoid(p)
    return s + z * s * torch.sigmoid(-p) * dp


def act_bound(z, name):
    """How far act may be off by FP32's evaluation (see block_math)."""
    if name in ("none", "relu2"):
        return 2.0 ** -23 * act64(z, name).abs()
    return 2.0 ** -22 * (4 + arg64(z, name).abs()) * act64(z, name).abs() + 1e-37


def ulp(ref, dtype):
    return (2.0 ** -8 if dtype == BF16 else 2.0 ** -24) * ref.abs() * 1.01 + 1e-37


def close(got, ref, tol):
    off = (got.double() - ref).abs() - tol
    worst = int(off.argmax())
    assert off.flatten()[worst] <= 0, (divmod(worst, ref.shape[1]), got.flatten()[worst].item(), ref.flatten()[worst].item(), tol.flatten()[worst].item())


def decode(c):
    v = c.codes.view(torch.float8_e4m3fn).double().reshape(c.rows, -1, 16) * c.scales.view(torch.float8_e8m0fnu).double()[..., None]
    return v.reshape(c.rows, c.cols)


def check_kept(c, z, tol):
    """Each value within half a step at its scale; each scale that of an amax within the product's error."""
    lo, hi = (((z.abs() + s * tol).clamp_min(0)).reshape(c.rows, -1, 16).amax(-1) for s in (-1, 1))
    scale = c.scales.view(torch.float8_e8m0fnu).double()
    assert bool((448 * scale >= lo * (1 - 2.0 ** -23)).all()) and bool(((448 * scale / 2 < hi * (1 + 2.0 ** -23)) | (c.scales == 0)).all())
    step = scale.repeat_interleave(16, 1) * 2.0 ** -10
    close(decode(c), z, torch.maximum(z.abs() * 2.0 ** -4, step) * (1 + 2.0 ** -10) + 2 * tol)


# m, n, k, workspace, MXFP4: the direct kernel's tiles (K split or not, K not a multiple of 64 or of 128, fewer than a window), 128 x 128 tiles, the 256 x 256 kernel
# without a workspace, the two-pass kernel's widths with one and with several tiles to a workgroup and with a split last round, MXFP4 of both kernels; ragged edges
SIZES = [(16, 16, 16, False, False), (16, 256, 4096, False, False), (48, 336, 112, False, False), (64, 5120, 2080, False, False), (256, 256, 512, True, False),
         (1040, 1296, 2064, True, False), (2064, 4112, 48, False, False), (4112, 5136, 16, False, False), (528, 784, 8192, False, False),
         (4112, 4368, 1088, False, False), (7760, 1568, 512, False, False), (7760, 1568, 512, True, False), (2048, 5120, 5120, True, False), (2064, 5136, 4096, True, False), (2560, 8208, 1024, True, False),
         (8192, 2576, 2048, True, False), (4096, 1808, 4096, True, False), (2944, 8192, 1024, True, False), (8208, 4112, 4096, True, False),
         (64, 96, 128, False, True), (544, 672, 384, False, True), (2080, 2592, 1024, False, True), (4128, 5152, 512, False, True), (1056, 4704, 2560, False, True),
         (1088, 7072, 512, False, True), (1632, 8160, 512, False, True), (4096, 15360, 512, False, True)]


@pytest.mark.parametrize("m,n,k,workspace,mx", SIZES)
def test_bias_activation_checkpoint(m, n, k, workspace, mx):
    p = Product(m, n, k, mx)
    bias = 0.5 * p.normal(n)
    for i, (name, dtype) in enumerate([("relu2", BF16), ("gelu", F32), ("silu", BF16), ("none", F32)]):
        keep = nv.alloc_checkpoint(m, n) if i < 2 else None
        out = p.run(workspace, bias=bias, activation=bm.ACTS[name], keep=keep, out_dtype=OUT[dtype])
        z = p.z + bias.double()
        tol = p.tol + 2.0 ** -23 * (p.z.abs() + z.abs())
        # |act'| <= 1.2 but for relu2's 2 z
        steep = (2 * z.abs() + 2 * tol) if name == "relu2" else 1.2
        ref = act64(z, name)
        close(out, ref, steep * tol + act_bound(z, name) + ulp(ref, dtype))
        if keep is not None:
            check_kept(keep, z, tol)


@pytest.mark.parametrize("m,n,k,workspace,mx", SIZES)
def test_residual(m, n, k, workspace, mx):
    p = Product(m, n, k, mx, seed=2)
    for rt, dtype, name, pad, biased in [(BF16, BF16, "none", 0, True), (F32, F32, "silu", 8, False), (BF16, F32, "relu2", 16, True), (F32, BF16, "none", 0, False)]:
        res = bm.tensor(p.normal(m, n).cpu().numpy(), rt, pad)
        bias = p.normal(n) if biased else None
        keep = nv.alloc_checkpoint(m, n) if name == "silu" else None
        out = p.run(workspace, bias=bias, activation=bm.ACTS[name], residual=res, keep=keep, out_dtype=OUT[dtype])
        z = p.z + (bias.double() if biased else 0)
        tol = p.tol + 2.0 ** -23 * (p.z.abs() + z.abs())
        steep = (2 * z.abs() + 2 * tol) if name == "relu2" else 1.2
        ref = act64(z, name) + res.double()
        close(out, ref, steep * tol + act_bound(z, name) + 2.0 ** -24 * ref.abs() + ulp(ref, dtype))
        if keep is not None:
            check_kept(keep, z, tol)
        if rt == dtype:      # over the residual itself
            again = p.run(workspace, bias=bias, activation=bm.ACTS[name], residual=res, out_dtype=OUT[dtype], out=res)
            assert again is res and torch.equal(res, out)


@pytest.mark.parametrize("m,n,k,workspace,mx", SIZES)
def test_times_the_derivative(m, n, k, workspace, mx):
    p = Product(m, n, k, mx, seed=3)
    saved = nv.nvfp4_checkpoint_save(2 * p.normal(m, n) * torch.exp2(torch.randint(-3, 4, (m, n // 16), device="cuda").float()).repeat_interleave(16, 1))
    v = decode(saved)
    for name, dtype in [("relu2", BF16), ("gelu", F32), ("silu", BF16), ("none", F32)]:
        out = p.run(workspace, activation=bm.ACTS[name], grad_of=saved, out_dtype=OUT[dtype])
        s = slope64(v, name)
        ref = p.z * s
        if name in ("none", "relu2"):
            bound = 2.0 ** -23 * s.abs()
        else:
            x = arg64(v, name)
            bound = 2.0 ** -22 * (4 + 2 * x.abs()) * (torch.sigmoid(x) + v.abs() * torch.sigmoid(x) * torch.sigmoid(-x) * (1 + (0.7 * v * v if name == "gelu" else 0)) * 1.6) + 1e-37
        close(out, ref, (p.tol + 2.0 ** -23 * p.z.abs()) * (s.abs() + bound) + p.z.abs() * bound + ulp(ref, dtype))


@pytest.mark.parametrize("m,n,k,workspace", [(48, 336, 112, False), (7760, 1568, 512, False), (7760, 1568, 512, True), (7760, 2096, 512, True), (1040, 1296, 2064, False), (4112, 5136, 16, False), (2048, 5120, 5120, True), (8192, 2576, 2048, True),
                                             (2944, 8192, 1024, True)])
def test_scales_per_row(m, n, k, workspace):
    p = Product(m, n, k, row_scales=True, seed=4)
    bias, res = p.normal(n), p.normal(m, n)
    keep = nv.alloc_checkpoint(m, n)
    out = p.run(workspace, bias=bias, activation=nv.ACT_GELU, keep=keep, out_dtype=nv.OUT_F32)
    z = p.z + bias.double()
    tol = p.tol + 2.0 ** -23 * (p.z.abs() + z.abs())
    ref = act64(z, "gelu")
    close(out, ref, 1.2 * tol + act_bound(z, "gelu") + ulp(ref, F32))
    check_kept(keep, z, tol)
    out = p.run(workspace, residual=res, out_dtype=nv.OUT_BF16)
    ref = p.z + res.double()
    close(out, ref, p.tol + 2.0 ** -23 * (p.z.abs() + ref.abs()) + ulp(ref, BF16))
    out = p.run(workspace, activation=nv.ACT_RELU2, grad_of=keep, out_dtype=nv.OUT_F32)
    s = slope64(decode(keep), "relu2")
    close(out, p.z * s, (p.tol + 2.0 ** -22 * p.z.abs()) * s.abs() + 1e-37)


@pytest.mark.parametrize("m,n,k,workspace,mx", SIZES)
def test_with_nothing_to_do_it_is_the_product(m, n, k, workspace, mx):
    """Not bit for bit where the tiles differ (320 x 320 and a split last round sum in another order): within the product's own error of each other."""
    p = Product(m, n, k, mx, seed=5)
    ws = torch.empty(nv.gemm_workspace_bytes(m, n, k), dtype=torch.uint8, device="cuda") if workspace else None
    a, b = nv.nvfp4_gemm(p.a, p.b, nv.OP_DGRAD, nv.OUT_F32, workspace=ws), p.run(workspace, out_dtype=nv.OUT_F32)
    close(b, a.double(), 2 * p.tol + 2.0 ** -23 * p.z.abs())


def shapes():
    lib = nv.load_library()
    got, out = [], (ctypes.c_int * 4)()
    while lib.nvfp4_internal_direct_shape_at(len(got), out):
        got.append(tuple(out))
    return got


@pytest.mark.parametrize("shape", range(13))
def test_every_shape_of_the_direct_kernel(shape):
    lib = nv.load_library()
    assert len(shapes()) == 13
    lib.nvfp4_internal_gemm_epilogue_direct.argtypes = lib.nvfp4_gemm_epilogue.argtypes[:7] + [ctypes.c_int, ctypes.c_void_p]
    for m, n, k in ((16, 16, 256), (176, 336, 656), (272, 240, 2560)):
        p = Product(m, n, k, seed=6)
        bias, keep = p.normal(n), nv.alloc_checkpoint(m, n)
        out = torch.empty(m, n, device="cuda")
        e = nv.EpilogueStruct(bias=bias.data_ptr(), activation=nv.ACT_GELU, keep=ctypes.pointer(keep.desc))
        assert lib.nvfp4_internal_gemm_epilogue_direct(ctypes.byref(p.a.desc), ctypes.byref(p.b.desc), nv.OP_DGRAD, ctypes.byref(e), out.data_ptr(), nv.OUT_F32, n, shape, None) == 0
        z = p.z + bias.double()
        tol = p.tol + 2.0 ** -23 * (p.z.abs() + z.abs())
        close(out, act64(z, "gelu"), 1.2 * tol + act_bound(z, "gelu") + ulp(z, F32))
        check_kept(keep, z, tol)
        e = nv.EpilogueStruct(activation=nv.ACT_RELU2, grad_of=ctypes.pointer(keep.desc))
        assert lib.nvfp4_internal_gemm_epilogue_direct(ctypes.byref(p.a.desc), ctypes.byref(p.b.desc), nv.OP_DGRAD, ctypes.byref(e), out.data_ptr(), nv.OUT_F32, n, shape, None) == 0
        s = slope64(decode(keep), "relu2")
        close(out, p.z * s, (p.tol + 2.0 ** -22 * p.z.abs()) * s.abs() + 1e-37)


def test_fprop_and_wgrad_read_the_copies_that_nvfp4_gemm_reads():
    tokens, d_in, d_out = 272, 528, 336
    g = torch.Generator(device="cuda")
    g.manual_seed(7)
    x, w, dy = (torch.randn(*s, generator=g, device="cuda").to(BF16) for s in ((tokens, d_in), (d_in, d_out), (tokens, d_out)))
    qx, qw = nv.nvfp4_quantize(x, 3, rht_on_col=True, rht_seed=3), nv.nvfp4_quantize(w, 3, nv.BLOCK_16x16)
    qdy = nv.nvfp4_quantize(dy, 3, rounding=nv.ROUND_SR, rht_on_col=True, rht_seed=3, sr_seed=9)
    for a, b, op in ((qx, qw, nv.OP_FPROP), (qdy, qw, nv.OP_DGRAD), (qx, qdy, nv.OP_WGRAD)):
        d = nv.nvfp4_gemm(a, b, op, nv.OUT_F32)
        res = torch.randn(*d.shape, generator=g, device="cuda")
        assert torch.equal(nv.nvfp4_gemm_epilogue(a, b, op, residual=res, out_dtype=nv.OUT_F32), d + res)
        keep = nv.alloc_checkpoint(*d.shape)
        nv.nvfp4_gemm_epilogue(a, b, op, activation=nv.ACT_RELU2, keep=keep)
        assert torch.equal(keep.codes, nv.nvfp4_checkpoint_save(d).codes) and torch.equal(keep.scales, nv.nvfp4_checkpoint_save(d).scales)


def test_infinities_and_nans_reach_the_result():
    m, n, k = 64, 96, 256
    p = Product(m, n, k, seed=8)
    bias = torch.zeros(n, device="cuda")
    bias[5], bias[40] = float("nan"), float("inf")
    for name in bm.ACTS:
        keep = nv.alloc_checkpoint(m, n)
        out = p.run(False, bias=bias, activation=bm.ACTS[name], keep=keep, out_dtype=nv.OUT_F32)
        assert bool(torch.isnan(out[:, 5]).all()) and not bool(torch.isfinite(out[:, 40]).any())
        assert bool((keep.scales[:, [0, 2]] == 255).all()) and not bool((keep.scales[:, [1, 3, 4, 5]] == 255).any())
        assert torch.isfinite(out[:, 48:]).all()


def test_in_a_graph_and_on_another_stream():
    """Replayed several times, with other work in between, against the call by itself."""
    m, n, k = 2048, 5120, 5120
    p = Product(m, n, k, seed=9)
    ws = torch.empty(nv.gemm_workspace_bytes(m, n, k), dtype=torch.uint8, device="cuda")
    bias, keep, out = p.normal(n), nv.alloc_checkpoint(m, n), torch.empty(m, n, dtype=BF16, device="cuda")
    want = nv.nvfp4_gemm_epilogue(p.a, p.b, nv.OP_DGRAD, bias=bias, activation=nv.ACT_SILU, keep=keep, workspace=ws)
    codes = keep.codes.clone()
    call = lambda: nv.nvfp4_gemm_epilogue(p.a, p.b, nv.OP_DGRAD, bias=bias, activation=nv.ACT_SILU, keep=keep, out=out, workspace=ws)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    s.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(4):
        out.zero_()
        keep.codes.zero_()
        torch.mm(torch.ones(64, 64, device="cuda"), torch.ones(64, 64, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(keep.codes, codes)


def test_nothing_outside_the_result_is_written():
    for m, n, k, workspace in ((48, 336, 112, False), (4112, 4368, 1088, False), (2064, 5136, 4096, True)):
        p = Product(m, n, k, seed=10)
        wide = torch.full((m + 2, n + 32), 7.0, dtype=BF16, device="cuda")
        codes, scales = torch.full((m + 2, n), 0xAB, dtype=torch.uint8, device="cuda"), torch.full((m + 2, n // 16), 0xAB, dtype=torch.uint8, device="cuda")
        keep = nv.Checkpoint8(codes[1:-1], scales[1:-1])
        p.run(workspace, keep=keep, activation=nv.ACT_GELU, out=wide[1:-1, 16:-16])
        assert bool((wide[[0, -1]] == 7).all()) and bool((wide[:, :16] == 7).all()) and bool((wide[:, -16:] == 7).all())
        assert bool((codes[[0, -1]] == 0xAB).all()) and bool((scales[[0, -1]] == 0xAB).all())
