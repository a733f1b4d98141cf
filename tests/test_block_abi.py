"""CPU: the calls around the linear layers refuse bad arguments before anything is enqueued; the binding refuses what it can see."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2509_25149_amd import binding as nv

P = 0x10000      # fake, aligned, never dereferenced by the checks


@pytest.fixture(scope="module")
def lib():
    return nv.load_library()


def ckpt(rows=32, cols=64, codes=P, scales=P):
    return ctypes.byref(nv.CheckpointStruct(rows, cols, codes, scales))


def test_struct_layouts_match_the_header(tmp_path):
    structs = {"nvfp4_checkpoint": nv.CheckpointStruct, "nvfp4_epilogue": nv.EpilogueStruct}
    lines = []
    for name, mirror in structs.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f[0]}));' for f in mirror._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "nvfp4.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0;\n}\n")
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    want = [v for m in structs.values() for v in [ctypes.sizeof(m)] + [getattr(m, f[0]).offset for f in m._fields_]]
    assert got == want


def test_struct_layout():
    assert ctypes.sizeof(nv.CheckpointStruct) == 32 and nv.CheckpointStruct.codes.offset == 16 and nv.CheckpointStruct.scales.offset == 24


def test_sizes(lib):
    c, s = ctypes.c_size_t(), ctypes.c_size_t()
    assert lib.nvfp4_checkpoint_sizes(3, 48, ctypes.addressof(c), ctypes.addressof(s)) == 0 and (c.value, s.value) == (144, 9)
    assert lib.nvfp4_checkpoint_sizes(0, 48, ctypes.addressof(c), None) == 0 and c.value == 0
    for rows, cols in ((-1, 16), (1, 0), (1, 24), (1, -16), (1 << 31, 16), (1, 1 << 31)):
        assert lib.nvfp4_checkpoint_sizes(rows, cols, None, None) == -2
        assert lib.nvfp4_rowsum_workspace_bytes(rows, cols, ctypes.addressof(c)) == -2
    assert lib.nvfp4_rowsum_workspace_bytes(16, 16, None) == -1
    assert nv.rowsum_workspace_bytes(0, 64) == 0 and nv.rowsum_workspace_bytes(1, 5120) == 0
    assert nv.rowsum_workspace_bytes(8192, 5120) >= 2 * 5120 * 4


def test_save_and_load_refuse(lib):
    save = lambda x=P, dt=1, ld=64, c=None: lib.nvfp4_checkpoint_save(x, dt, ld, c or ckpt(), None)
    assert lib.nvfp4_checkpoint_save(P, 1, 64, None, None) == -1
    assert save(x=None) == -1 and save(x=P + 8) == -1 and save(dt=2) == -1 and save(dt=-1) == -1
    assert save(ld=48) == -2 and save(ld=68) == -2
    assert save(c=ckpt(cols=40), ld=40) == -2 and save(c=ckpt(rows=-1)) == -2
    assert save(c=ckpt(codes=None)) == -1 and save(c=ckpt(scales=None)) == -1 and save(c=ckpt(codes=P + 8)) == -1
    load = lambda c=None, act=0, f=None, out=P, dt=1, ld=64: lib.nvfp4_checkpoint_load(c or ckpt(), act, f, out, dt, ld, None)
    assert lib.nvfp4_checkpoint_load(None, 0, None, P, 1, 64, None) == -1
    assert load(act=4) == -1 and load(act=-1) == -1 and load(dt=2) == -1 and load(out=None) == -1 and load(out=P + 4) == -1 and load(f=P + 4) == -1
    assert load(ld=56) == -2 and load(ld=65) == -2


def test_norm_refuses(lib):
    def fwd(x=P, xt=1, ldx=64, r=None, ldr=64, g=None, eps=1e-5, rows=32, cols=64, h=None, ht=1, ldh=64, y=P, yt=1, ldy=64, rstd=P, keep=None, kind=0):
        return lib.nvfp4_rmsnorm_forward(x, xt, ldx, r, ldr, g, eps, rows, cols, h, ht, ldh, y, yt, ldy, rstd, keep, kind, None)
    assert fwd(x=None) == -1 and fwd(x=P + 2) == -1 and fwd(xt=2) == -1 and fwd(ht=3) == -1 and fwd(yt=-1) == -1
    assert fwd(eps=-1.0) == -1 and fwd(eps=float("nan")) == -1 and fwd(kind=2) == -1
    assert fwd(rows=-1) == -2 and fwd(cols=0) == -2 and fwd(cols=24) == -2 and fwd(cols=32784, ldx=32784, ldy=32784) == -2
    assert fwd(ldx=48) == -2 and fwd(ldx=68) == -2 and fwd(r=P, ldr=48) == -2 and fwd(h=P, ldh=63) == -2 and fwd(ldy=60) == -2
    assert fwd(r=P + 4) == -1 and fwd(h=P + 8) == -1 and fwd(y=P + 8) == -1 and fwd(g=P + 4) == -1 and fwd(rstd=P + 2) == -1
    assert fwd(keep=ckpt(rows=16)) == -4 and fwd(keep=ckpt(cols=48)) == -4 and fwd(keep=ckpt(codes=None)) == -1

    def bwd(dy=P, dt=1, lddy=64, h=P, ldh=64, saved=None, rstd=P, g=None, dres=None, lddr=64, rows=32, cols=64, dx=P, st=1, lddx=64, dg=P, acc=0, ws=P, n=1 << 20):
        return lib.nvfp4_rmsnorm_backward(dy, dt, lddy, h, ldh, saved, rstd, g, dres, lddr, rows, cols, dx, st, lddx, dg, acc, ws, n, None)
    assert bwd(dy=None) == -1 and bwd(dt=2) == -1 and bwd(st=2) == -1 and bwd(rstd=None) == -1 and bwd(rstd=P + 2) == -1
    assert bwd(h=None) == -1 and bwd(saved=ckpt()) == -1                    # exactly one of the two
    assert bwd(h=None, saved=ckpt(rows=31)) == -4 and bwd(h=None, saved=ckpt(scales=None)) == -1
    assert bwd(cols=72) == -2 and bwd(rows=-1) == -2 and bwd(lddy=56) == -2 and bwd(ldh=8) == -2 and bwd(dres=P, lddr=56) == -2 and bwd(lddx=60) == -2
    assert bwd(dres=P + 8) == -1 and bwd(dx=P + 8) == -1 and bwd(dg=P + 4) == -1 and bwd(g=P + 8) == -1
    assert bwd(ws=None) == -6 and bwd(n=16) == -6 and bwd(ws=P + 8) == -6


def test_activation_backward_refuses(lib):
    def bwd(da=P, dt=1, ldda=64, rows=32, cols=64, saved=ckpt(), act=1, dz=P, lddz=64, db=P, acc=0, ws=P, n=1 << 20):
        return lib.nvfp4_activation_backward(da, dt, ldda, rows, cols, saved, act, dz, lddz, db, acc, ws, n, None)
    assert bwd(da=None) == -1 and bwd(da=P + 8) == -1 and bwd(dt=2) == -1 and bwd(act=4) == -1 and bwd(saved=None) == -1
    assert bwd(rows=31) == -4 and bwd(cols=48) == -4 and bwd(cols=56) == -2 and bwd(rows=-2) == -2
    assert bwd(ldda=56) == -2 and bwd(lddz=60) == -2 and bwd(dz=P + 8) == -1 and bwd(db=P + 4) == -1
    assert bwd(ws=None) == -6 and bwd(n=8) == -6


def test_the_binding_refuses():
    x = torch.zeros(4, 32)
    for call in (lambda: nv.nvfp4_checkpoint_save(x), lambda: nv.nvfp4_rmsnorm_forward(x), lambda: nv.nvfp4_activation_backward(x),
                 lambda: nv.nvfp4_rmsnorm_backward(x, x, torch.zeros(4)), lambda: nv.Checkpoint8(x.byte(), x.byte())):
        with pytest.raises(ValueError):
            call()


def test_gemm_epilogue_refuses(lib):
    def desc(rows, cols):
        d = nv.QTensorStruct()
        d.rows, d.cols, d.layout_mask, d.block_dim = rows, cols, 1, 1
        d.row_codes = d.row_scales = d.row_tensor_scale = P
        return d

    def call(m=32, n=48, k=64, kb=64, epilogue=True, d=P, dt=1, ldd=48, **e):
        a, b, s = desc(m, k), desc(n, kb), nv.EpilogueStruct(**e)
        return lib.nvfp4_gemm_epilogue(ctypes.byref(a), ctypes.byref(b), 1, ctypes.byref(s) if epilogue else None, d, dt, ldd, None, 0, None)

    def c(rows=32, cols=48, codes=P, scales=P):
        return ctypes.pointer(nv.CheckpointStruct(rows, cols, codes, scales))
    assert ctypes.sizeof(nv.EpilogueStruct) == 48
    assert call(epilogue=False) == -1 and call(d=None) == -1 and call(dt=2) == -1 and call(dt=3) == -1 and call(activation=4) == -1 and call(activation=-1) == -1
    assert call(kb=80) == -4 and call(ldd=40) == -2 and call(ldd=52) == -2 and call(d=P + 8) == -1       # as nvfp4_gemm
    assert call(bias=P + 4) == -1
    assert call(residual=P, ldr=40) == -2 and call(residual=P, ldr=50) == -2 and call(residual=P + 8, ldr=48) == -1 and call(residual=P, ldr=48, residual_dtype=2) == -1
    assert call(keep=c(cols=64)) == -4 and call(keep=c(rows=16)) == -4 and call(keep=c(codes=None)) == -1 and call(keep=c(codes=P + 4)) == -1
    assert call(grad_of=c(rows=48)) == -4 and call(grad_of=c(scales=None)) == -1
    for other in (dict(bias=P), dict(residual=P, ldr=48), dict(keep=c())):
        assert call(grad_of=c(), **other) == -1                                                            # one form or the other
