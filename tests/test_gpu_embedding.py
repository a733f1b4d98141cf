"""Embedding lookup and its gradient on the GPU."""
import numpy as np
import pytest
import torch

import block_math as bm
import ends_math as em
from paper_2509_25149_amd import binding as nv

pytestmark = pytest.mark.gpu
F32, BF16, I32, I64 = torch.float32, torch.bfloat16, torch.int32, torch.int64
OUT = {F32: nv.OUT_F32, BF16: nv.OUT_BF16}


def tokens(n, vocab, seed, kind="zipf"):
    r = np.random.default_rng(seed)
    if kind == "zipf":
        ids = np.minimum((vocab + 1.0) ** r.random(n), vocab).astype(np.int64) - 1
    elif kind == "one":
        ids = np.full(n, vocab // 2)
    elif kind == "none":
        ids = np.full(n, -1)
    else:
        ids = r.integers(0, vocab, n)
    if kind in ("zipf", "uniform") and n > 4:
        ids[r.integers(0, n, max(1, n // 50))] = r.choice([-1, vocab, -100, 2 ** 31 - 1])
    return ids


@pytest.mark.parametrize("n,vocab,cols", [(0, 5, 16), (1, 1, 16), (1, 1000, 5120), (7, 3, 48), (300, 50257, 528), (1040, 5003, 2064), (65, 17, 32768)])
@pytest.mark.parametrize("tt,ot,it,scale,pad", [(BF16, BF16, I64, 1.0, 0), (F32, F32, I32, -0.7, 8), (BF16, F32, I32, 71.5, 8), (F32, BF16, I64, 1.0, 0)])
def test_lookup(n, vocab, cols, tt, ot, it, scale, pad):
    r = np.random.default_rng(n + cols)
    table = bm.tensor(r.standard_normal((vocab, cols)), tt, pad)
    ids = tokens(n, vocab, 1)
    t64, there = bm.f64(table), (ids >= 0) & (ids < vocab)
    ref = np.where(there[:, None], t64[np.clip(ids, 0, vocab - 1)] * np.float32(scale).astype(np.float64), 0.0)
    out = nv.nvfp4_embedding_forward(em.index(ids, it), table, scale=scale, out_dtype=OUT[ot])
    assert out.dtype == ot and out.shape == (n, cols)
    bm.within(out, ref, em.U * np.abs(ref) + bm.rounding(ref, ot))
    own = bm.tensor(np.zeros((n, cols)), ot, 24)
    assert nv.nvfp4_embedding_forward(em.index(ids, it), table, scale=scale, out=own) is own and torch.equal(own, out)
    assert n == 0 or torch.isnan(own.as_strided((n, 24), own.stride(), cols)).all()


# tokens: below and above what one launch does (512) and what is ranked by counting (12288), words of 64, chunk limits, tiles (2048); columns: strips of 512; 32 tiles;
# tables above and below 8 MB, with more and fewer than four rows to a token
@pytest.mark.parametrize("n,vocab,cols", [(1, 1, 16), (63, 70, 2064), (64, 300, 2048), (65, 65, 4112), (129, 270000, 64), (255, 2000, 16), (256, 40000, 64), (257, 66, 528), (511, 66, 48), (512, 66, 528), (512, 40000, 64), (513, 66, 528), (1023, 2000, 16), (1024, 66, 528), (1025, 66, 528), (1100, 300000, 64), (1500, 6001, 48), (2, 300, 528), (15, 4, 16), (16, 9, 48), (17, 9, 512), (33, 5, 1040), (1040, 5003, 272), (2047, 40, 32),
                                          (2049, 100, 16), (4099, 131072, 16), (8192, 700, 64), (12287, 700, 64), (12288, 700, 64), (12289, 700, 64), (20000, 511, 32), (20000, 513, 32), (33000, 300000, 16), (65536, 900, 16), (65537, 900, 16), (140000, 1 << 20, 16)])
@pytest.mark.parametrize("kind", ["zipf", "one", "none", "uniform"])
def test_gradient(n, vocab, cols, kind):
    r = np.random.default_rng(n * 3 + vocab)
    ids = tokens(n, vocab, 2, kind)
    for dt, it, scale, pad in ((F32, I64, 1.0, 8), (BF16, I32, -1.5, 0)):
        dout = bm.tensor(r.standard_normal((n, cols)), dt, pad)
        ref, tol = em.embedding_gradient(bm.f64(dout), ids, vocab, scale)
        idt = em.index(ids, it)
        got = nv.nvfp4_embedding_backward(dout, idt, vocab, scale=scale)
        bm.within(got, ref, tol + em.U * np.abs(ref))
        assert torch.equal(got, nv.nvfp4_embedding_backward(dout, idt, vocab, scale=scale))      # in a fixed order
        before = bm.tensor(r.standard_normal((vocab, cols)), F32, 16)
        old = bm.f64(before)
        wide = before.as_strided((vocab, 16), before.stride(), cols)
        assert nv.nvfp4_embedding_backward(dout, idt, dtable=before, scale=scale, accumulate=True) is before
        untouched = np.ones(vocab, bool)
        untouched[ids[(ids >= 0) & (ids < vocab)]] = False
        bm.within(before, old + ref, tol + 2 * em.U * (np.abs(old) + np.abs(ref)) * ~untouched[:, None])
        assert torch.isnan(wide).all()
        # stored over what was there, rows without a token too
        assert torch.equal(nv.nvfp4_embedding_backward(dout, idt, dtable=before, scale=scale), got) and torch.isnan(wide).all()


def test_gradient_without_tokens():
    dout, ids = torch.empty(0, 48, device="cuda"), torch.empty(0, dtype=I64, device="cuda")
    assert torch.equal(nv.nvfp4_embedding_backward(dout, ids, 70), torch.zeros(70, 48, device="cuda"))
    before = torch.ones(70, 48, device="cuda")
    nv.nvfp4_embedding_backward(dout, ids, dtable=before, accumulate=True)
    assert bool((before == 1).all())


def test_gradient_agrees_with_differences():
    n, vocab, cols, scale = 40, 9, 32, 1.5
    r = np.random.default_rng(5)
    table, w, ids = r.standard_normal((vocab, cols)), r.standard_normal((n, cols)).astype(np.float32), tokens(n, vocab, 3)
    there = (ids >= 0) & (ids < vocab)
    f = lambda t: (np.where(there[:, None], t[np.clip(ids, 0, vocab - 1)] * scale, 0.0) * w).sum()
    got = bm.f64(nv.nvfp4_embedding_backward(bm.tensor(w, F32), em.index(ids, I64), vocab, scale=scale))
    for _ in range(4):
        v = r.standard_normal(table.shape)
        diff = (f(table + 1e-3 * v) - f(table - 1e-3 * v)) / 2e-3      # exact but for binary64's rounding: f is linear
        assert abs((got * v).sum() - diff) <= 1e-5 * np.sqrt((got ** 2).sum())


def test_a_table_of_more_than_2_to_the_31_elements():
    vocab, cols = 430_000, 5008
    table = torch.zeros(vocab, cols, dtype=BF16, device="cuda")
    rows = torch.tensor([0, vocab - 1, vocab // 2, vocab], device="cuda")
    table[rows[:3]] = torch.tensor([[1.0], [2.0], [3.0]], dtype=BF16, device="cuda")
    out = nv.nvfp4_embedding_forward(rows, table)
    assert [float(v) for v in out.float().mean(1)] == [1, 2, 3, 0]
    del table
    d = nv.nvfp4_embedding_backward(out, rows, vocab)
    assert [float(v) for v in d[rows[:3]].mean(1)] == [1, 2, 3] and float(d.sum(dtype=torch.float64)) == 6 * cols


def test_scratch_memory_and_another_stream():
    n, vocab, cols = 9000, 800, 528
    dout, ids = bm.tensor(np.random.default_rng(1).standard_normal((n, cols)), BF16), em.index(tokens(n, vocab, 4), I32)
    want = nv.nvfp4_embedding_backward(dout, ids, vocab)
    need = nv.embedding_workspace_bytes(n, vocab, cols)
    buf = torch.full((need + 4096,), 0xAB, dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        got = nv.nvfp4_embedding_backward(dout, ids, vocab, workspace=buf[:need])
    s.synchronize()
    assert torch.equal(got, want) and bool((buf[need:] == 0xAB).all())
