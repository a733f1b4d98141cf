"""Calls with the binding's own scratch memory: captured into graphs that are replayed beside other work, and from two host threads on one stream."""
import threading

import pytest
import torch

from paper_2509_25149_amd import binding as nv

pytestmark = pytest.mark.gpu
SMALL, LARGE = (1040, 2064), (4112, 8208)
RC = nv.LAYOUT_ROW | nv.LAYOUT_COL


def matrix(rows, cols, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(rows, cols, generator=g, device="cuda").bfloat16()


class Case:
    """One call on inputs of its own; `run` gives its outputs."""

    def __init__(self, name, rows, cols, seed):
        self.name, self.x = name, matrix(rows, cols, seed)
        if name != "quantize":
            self.dy = matrix(rows, cols, seed + 1)
            self.norm = nv.nvfp4_rmsnorm_forward(self.x, checkpoint=True)

    def run(self):
        if self.name == "quantize":
            q = nv.nvfp4_quantize(self.x, RC, rht_on_col=True, rht_seed=5)
            return [q.row_codes, q.row_scales, q.row_ts, q.col_codes, q.col_scales, q.col_ts]
        if self.name == "rmsnorm_backward":
            return list(nv.nvfp4_rmsnorm_backward(self.dy, self.norm.checkpoint, self.norm.rstd))
        return list(nv.nvfp4_activation_backward(self.dy, self.norm.checkpoint, nv.ACT_GELU))


NAMES = ["quantize", "rmsnorm_backward", "activation_backward"]


def same(got, want):
    return all(torch.equal(g.view(torch.uint8), w.view(torch.uint8)) for g, w in zip(got, want))


@pytest.mark.parametrize("name", NAMES)
def test_replays_neither_lose_their_workspace_nor_write_into_what_came_after(name):
    assert name == "quantize" or nv.rowsum_workspace_bytes(*SMALL) > 0
    case, larger = Case(name, *SMALL, 1), Case(name, *LARGE, 3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = [t.clone() for t in case.run()]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = case.run()
        want_larger = [t.clone() for t in larger.run()]                  # needs more scratch memory than there was
        live = [torch.full((1 << 16,), 0xAB, dtype=torch.uint8, device="cuda") for _ in range(256)]
        live.append(torch.full((nv.rowsum_workspace_bytes(*SMALL),), 0xAB, dtype=torch.uint8, device="cuda"))
        for _ in range(4):
            for t in out:
                t.view(torch.uint8).zero_()
            graph.replay()
            got_larger = larger.run()                                    # behind the replay
            side.synchronize()
            assert same(out, want) and same(got_larger, want_larger)
            assert all(bool((t == 0xAB).all()) for t in live)


@pytest.mark.parametrize("name", NAMES)
def test_two_graphs_captured_on_one_stream_run_side_by_side(name):
    cases = [Case(name, *SMALL, seed) for seed in (7, 17)]
    want = [[t.clone() for t in c.run()] for c in cases]
    capture, streams, graphs, outs = torch.cuda.Stream(), [torch.cuda.Stream() for _ in cases], [], []
    torch.cuda.synchronize()
    for c in cases:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=capture):
            outs.append(c.run())
    for _ in range(8):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert all(same(o, w) for o, w in zip(outs, want))
        for o in outs:
            for t in o:
                t.view(torch.uint8).zero_()
        torch.cuda.synchronize()


@pytest.mark.parametrize("name", NAMES)
def test_two_threads_on_one_stream(name):
    cases = [Case(name, *SMALL, seed) for seed in (7, 17)]
    want = [[t.clone() for t in c.run()] for c in cases]
    torch.cuda.synchronize()
    wrong = []

    def work(c, w):
        for _ in range(50):
            if not same(c.run(), w):
                wrong.append(c.name)
    threads = [threading.Thread(target=work, args=a) for a in zip(cases, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
