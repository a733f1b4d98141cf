"""CPU: the calls at the ends of a training step refuse bad arguments before anything is enqueued; the binding refuses what it can see; the list of gradients covers
every element once."""
import ctypes
import os
import struct
import subprocess

import numpy as np
import pytest
import torch

from paper_2509_25149_amd import binding as nv

P = 0x10000      # fake, aligned, never dereferenced by the checks


@pytest.fixture(scope="module")
def lib():
    return nv.load_library()


def test_struct_layouts_match_the_header(tmp_path):
    structs = {"nvfp4_grad": nv.GradStruct, "nvfp4_grad_list": nv.GradListStruct}
    lines = []
    for name, mirror in structs.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f[0]}));' for f in mirror._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "nvfp4.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0;\n}\n")
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include"), str(src), "-o", str(exe)], check=True)
    got = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert got == [v for m in structs.values() for v in [ctypes.sizeof(m)] + [getattr(m, f[0]).offset for f in m._fields_]]


def test_embedding_refuses(lib):
    def fwd(ids=P, it=1, n=32, table=P, tt=1, vocab=100, cols=64, ldt=64, scale=1.0, out=P, ot=1, ldo=64):
        return lib.nvfp4_embedding_forward(ids, it, n, table, tt, vocab, cols, ldt, scale, out, ot, ldo, None)
    assert fwd(ids=None) == -1 and fwd(ids=P + 4) == -1 and fwd(ids=P + 2, it=0) == -1 and fwd(it=2) == -1 and fwd(it=-1) == -1
    assert fwd(table=None) == -1 and fwd(table=P + 8) == -1 and fwd(out=None) == -1 and fwd(out=P + 4) == -1 and fwd(tt=2) == -1 and fwd(ot=-1) == -1
    assert fwd(scale=float("inf")) == -1 and fwd(scale=float("nan")) == -1
    assert fwd(n=-1) == -2 and fwd(n=1 << 30) == -2 and fwd(vocab=0) == -2 and fwd(vocab=(1 << 31) - 1) == -2 and fwd(cols=24) == -2 and fwd(cols=0) == -2
    assert fwd(cols=32784, ldt=32784, ldo=32784) == -2 and fwd(ldt=56) == -2 and fwd(ldt=68) == -2 and fwd(ldo=60) == -2

    def bwd(dout=P, dt=1, ldd=64, ids=P, it=1, n=2000, vocab=100, cols=64, scale=1.0, dtable=P, ldt=64, acc=0, ws=P, size=1 << 24):
        return lib.nvfp4_embedding_backward(dout, dt, ldd, ids, it, n, vocab, cols, scale, dtable, ldt, acc, ws, size, None)
    assert bwd(dout=None) == -1 and bwd(dout=P + 8) == -1 and bwd(dt=2) == -1 and bwd(ids=None) == -1 and bwd(ids=P + 4) == -1 and bwd(it=5) == -1
    assert bwd(dtable=None) == -1 and bwd(dtable=P + 4) == -1 and bwd(scale=float("nan")) == -1
    assert bwd(n=-1) == -2 and bwd(vocab=-1) == -2 and bwd(cols=40) == -2 and bwd(ldd=56) == -2 and bwd(ldt=63) == -2
    need = nv.embedding_workspace_bytes(2000, 100, 64)
    assert bwd(ws=None) == -6 and bwd(size=need - 1) == -6 and bwd(ws=P + 8) == -6
    w = ctypes.c_size_t()
    assert lib.nvfp4_embedding_workspace_bytes(32, 100, 24, ctypes.addressof(w)) == -2 and lib.nvfp4_embedding_workspace_bytes(32, 100, 64, None) == -1
    assert nv.embedding_workspace_bytes(0, 100, 64) == 0 and nv.embedding_workspace_bytes(512, 100, 64) == 0 and nv.embedding_workspace_bytes(513, 100, 64) >= 2 * 513 * 4


def test_logprob_refuses(lib):
    def fwd(z=P, dt=1, ld=104, rows=4, cols=100, scale=1.0, t=P, it=1, lp=P, st=P, lse=P, h=P, top=2, ti=P, tl=P, ws=None, size=0):
        return lib.nvfp4_logprob_forward(z, dt, ld, rows, cols, scale, t, it, lp, st, lse, h, top, ti, tl, ws, size, None)
    assert fwd(z=None) == -1 and fwd(z=P + 8) == -1 and fwd(dt=2) == -1 and fwd(it=2) == -1 and fwd(t=P + 4) == -1 and fwd(t=None) == -1
    for scale in (0.0, -1.0, float("inf"), float("nan")):
        assert fwd(scale=scale) == -1
    assert fwd(lp=P + 2) == -1 and fwd(st=P + 1) == -1 and fwd(lse=P + 2) == -1 and fwd(h=P + 3) == -1 and fwd(ti=P + 2) == -1 and fwd(tl=P + 2) == -1
    assert fwd(ti=None) == -1 and fwd(tl=None) == -1
    assert fwd(rows=-1) == -2 and fwd(cols=0) == -2 and fwd(cols=1 << 30, ld=1 << 30) == -2 and fwd(ld=96) == -2 and fwd(ld=100) == -2
    assert fwd(top=-1) == -2 and fwd(top=33) == -2 and fwd(cols=5, top=6) == -2
    assert nv.logprob_workspace_bytes(4, 100, 2) == 0 and nv.logprob_workspace_bytes(1, 131072, 8) > nv.logprob_workspace_bytes(1, 131072, 0) > 0
    big = dict(rows=1, cols=131072, ld=131072)
    need = nv.logprob_workspace_bytes(1, 131072, 2)
    assert fwd(**big) == -6 and fwd(ws=P, size=need - 1, **big) == -6 and fwd(ws=P + 8, size=need, **big) == -6
    w = ctypes.c_size_t()
    assert lib.nvfp4_logprob_workspace_bytes(1, 4, 5, ctypes.addressof(w)) == -2 and lib.nvfp4_logprob_workspace_bytes(1, 4, 4, None) == -1

    def bwd(z=P, dt=1, ld=104, rows=4, cols=100, scale=1.0, t=P, it=1, st=P, g=P, gl=None, ge=None, h=None, dz=2 * P, ot=1, ldd=104):
        return lib.nvfp4_logprob_backward(z, dt, ld, rows, cols, scale, t, it, st, g, gl, ge, h, dz, ot, ldd, None)
    assert bwd(z=None) == -1 and bwd(dz=None) == -1 and bwd(dz=P + 8) == -1 and bwd(ot=2) == -1 and bwd(st=None) == -1 and bwd(t=None) == -1 and bwd(ge=P) == -1
    assert bwd(g=P + 2) == -1 and bwd(gl=P + 2) == -1 and bwd(ge=P + 2, h=P) == -1 and bwd(ge=P, h=P + 2) == -1 and bwd(scale=-1.0) == -1
    assert bwd(ldd=96) == -2 and bwd(ldd=100) == -2 and bwd(ld=100) == -2 and bwd(cols=0) == -2

    assert bwd(dz=P, ot=0) == -1 and bwd(dz=P, ldd=112) == -1                                # over the logits, but laid out otherwise

    def both(z=P, dt=1, ld=104, rows=4, cols=100, scale=1.0, t=P, it=1, g=P, lp=P, st=P, lse=P, dz=2 * P, ot=1, ldd=104, ws=None, size=0):
        return lib.nvfp4_logprob_with_gradient(z, dt, ld, rows, cols, scale, t, it, g, lp, st, lse, dz, ot, ldd, ws, size, None)
    assert both(dz=P, ot=0) == -1 and both(dz=P, ldd=112) == -1 and both(z=None) == -1 and both(t=None) == -1 and both(g=None) == -1 and both(st=P + 2) == -1 and both(dz=None) == -1 and both(ot=3) == -1 and both(lse=P + 2) == -1
    assert both(ldd=96) == -2 and both(rows=-1) == -2 and both(rows=1, cols=131072, ld=131072, ldd=131072) == -6


def grad(data=P, out=None, rows=1, cols=100, ld=100, ld_out=100, dt=0, ot=0):
    return nv.GradStruct(data, out, rows, cols, ld, ld_out, dt, ot)


def build(lib, grads, room=1 << 22, host=True):
    array = (nv.GradStruct * max(1, len(grads)))(*grads)
    buf, lst = ctypes.create_string_buffer(room), nv.GradListStruct()
    rc = lib.nvfp4_grad_list_build(array, len(grads), ctypes.addressof(buf) if host else None, room, ctypes.byref(lst))
    return rc, buf, lst


def test_logprob_refuses_a_scale_whose_base_2_form_overflows(lib):
    """The kernels work with scale * log2(e): infinite, it would make a NaN of the largest logit's distance 0.  No rows: nothing is read, whatever the answer."""
    most = 2.0 ** 127
    for scale, rc in ((3.4e38, -1), (2.4e38, -1), (float(np.nextafter(np.float32(most), np.float32(np.inf))), -1), (most, 0), (1e-45, 0)):
        logits = (None, 1, 104, 0, 100, scale, None, 1)
        assert lib.nvfp4_logprob_forward(*logits, None, None, None, None, 0, None, None, None, 0, None) == rc
        assert lib.nvfp4_logprob_backward(*logits, None, None, None, None, None, None, 1, 104, None) == rc
        assert lib.nvfp4_logprob_with_gradient(*logits, None, None, None, None, None, 1, 104, None, 0, None) == rc


def test_the_list_of_gradients_refuses(lib):
    size = lambda *g: lib.nvfp4_grad_list_sizes((nv.GradStruct * len(g))(*g), len(g), None, None)
    assert size(grad()) == 0 and lib.nvfp4_grad_list_sizes(None, 1, None, None) == -1 and lib.nvfp4_grad_list_sizes(None, -1, None, None) == -1
    assert size(grad(data=None)) == -1 and size(grad(data=P + 2)) == -1 and size(grad(data=P + 2, dt=1, ot=1)) == 0 and size(grad(data=P + 1, dt=1, ot=1)) == -1
    assert size(grad(dt=2)) == -1 and size(grad(ot=3)) == -1 and size(grad(ot=1)) == -1 and size(grad(out=P + 2)) == -1
    assert size(grad(out=P, ot=1)) == -1 and size(grad(out=P, rows=2, ld_out=200)) == -1        # in its place, but laid out otherwise
    assert size(grad(rows=-1)) == -2 and size(grad(cols=-1)) == -2 and size(grad(rows=2, ld=99)) == -2 and size(grad(out=P * 2, rows=2, ld_out=99)) == -2
    assert size(grad(rows=1 << 30, cols=1 << 30, ld=1 << 30)) == -2 and size(grad(cols=1 << 41)) == -2
    assert size(grad(data=None, cols=0)) == 0 and size(grad(data=None, rows=0)) == 0
    apart = grad(data=P + 400)
    assert build(lib, [grad(), apart])[0] == 0 and build(lib, [grad(), grad(data=P + 396)])[0] == -1 and build(lib, [grad(), grad()])[0] == -1
    assert build(lib, [grad(out=2 * P), grad(out=3 * P)])[0] == 0 and build(lib, [grad(out=2 * P), grad(out=2 * P + 8)])[0] == -1
    assert build(lib, [grad(rows=4, cols=10, ld=20), grad(data=P + 40, rows=4, cols=10, ld=20)])[0] == 0       # side by side
    assert build(lib, [grad()], room=64)[0] == -6 and build(lib, [grad()], host=False)[0] == -1
    assert build(lib, [])[0] == 0

    good = build(lib, [grad()])[2]
    good.table = P
    ref = ctypes.byref(good)
    assert lib.nvfp4_grad_sumsq(None, P, P, 1 << 20, None) == -1 and lib.nvfp4_grad_sumsq(ref, None, P, 1 << 20, None) == -1
    assert lib.nvfp4_grad_sumsq(ref, P + 4, P, 1 << 20, None) == -1 and lib.nvfp4_grad_sumsq(ref, P, None, 0, None) == -6 and lib.nvfp4_grad_sumsq(ref, P, P, 7, None) == -6
    assert lib.nvfp4_grad_clip(None, P, 1.0, P, None) == -1 and lib.nvfp4_grad_clip(ref, None, 1.0, P, None) == -1 and lib.nvfp4_grad_clip(ref, P, -1.0, P, None) == -1
    assert lib.nvfp4_grad_clip(ref, P, float("nan"), P, None) == -1 and lib.nvfp4_grad_clip(ref, P, 1.0, P + 2, None) == -1
    unset = build(lib, [grad()])[2]
    assert lib.nvfp4_grad_sumsq(ctypes.byref(unset), P, P, 1 << 20, None) == -1                # the table has not been copied to the device


def test_units_of_work_cover_every_element_once(lib):
    """The table, read as the kernels do."""
    shapes = [(1, 1, 1), (1, 8191, 8191), (1, 8193, 8193), (0, 5, 5), (3, 100, 104), (70, 101, 300), (1000, 20, 24), (5, 20000, 20008), (64, 8192, 8200), (2, 300, 300), (1, 5_000_000, 5_000_000),
              (4_100_000, 10, 12)]
    grads, at = [], P
    for rows, cols, ld in shapes:
        grads.append(grad(data=at, rows=rows, cols=cols, ld=ld))
        at += max(rows * ld * 4, 64) // 64 * 64 + 64
    rc, buf, lst = build(lib, grads)
    assert rc == 0 and lst.tensors == len(shapes)
    owner = np.frombuffer(buf, np.int32, lst.units, len(shapes) * 64)
    seen = 0
    for i, (rows, cols, ld) in enumerate(shapes):
        data, out, c, l, lo, r, first, ur, uc, flags, _ = struct.unpack_from("<QQqqqiiiiii", buf, i * 64)
        mine = np.flatnonzero(owner == i)
        if rows * cols == 0:
            assert len(mine) == 0
            continue
        assert out == data == grads[i].data and (r, c) in ((rows, cols), (1, rows * cols)) and (r == 1 or l == ld == lo)
        assert flags == 0 and first == mine[0] and (uc % 8 == 0 or uc == c)
        across, down = -(-c // uc), -(-r // ur)
        assert list(mine) == list(range(first, first + across * down)) and ur * uc <= 1 << 24
        covered = sum(min(ur, r - (u // across) * ur) * min(uc, c - (u % across) * uc) for u in range(across * down))
        assert covered == rows * cols
        seen += len(mine)
    assert seen == lst.units < 40000


def test_the_binding_refuses():
    x, i = torch.zeros(4, 32), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: nv.nvfp4_embedding_forward(i, x), lambda: nv.nvfp4_embedding_backward(x, i, 9), lambda: nv.nvfp4_logprob_forward(x, i),
                 lambda: nv.nvfp4_logprob_backward(x, i, x), lambda: nv.nvfp4_logprob_with_gradient(x, i, torch.zeros(4)), lambda: nv.Gradients([x])):
        with pytest.raises((ValueError, RuntimeError, AssertionError)):
            call()


def test_a_workspace_that_is_no_plain_memory_is_refused(monkeypatch):
    """An expanded view says more elements than it has memory for."""
    monkeypatch.setattr(nv, "_here", lambda *tensors: None)
    whole = torch.empty(64, dtype=torch.float32)
    assert nv._scratch(whole, 256, whole.device)[:2] == (whole.data_ptr(), 256)
    for bad in (torch.empty(1).expand(64), torch.empty(1, 8).expand(8, 8), whole[::2]):
        with pytest.raises(ValueError):
            nv._scratch(bad, 64, bad.device)
