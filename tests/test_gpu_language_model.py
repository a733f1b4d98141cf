"""The ends of a training step together: examples/language_model.py, the calls in turn on their own results, captured into graphs, on other streams and from two threads."""
import importlib.util
import math
import os
import threading

import pytest
import torch

from paper_2509_25149_amd import binding as nv

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("language_model", os.path.join(ROOT, "examples", "language_model.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("tokens,d_model,d_ffn,vocab", [(256, 512, 1024, 4096), (528, 272, 1040, 5008)])
def test_a_step_is_near_the_model_in_64_bits(example, tokens, d_model, d_ffn, vocab):
    """The block adds to its input of size 1 (sqrt(d) 0.02 * sqrt(d) < 1) what two quantized products leave, off by some 0.2 of itself (see test_gpu_mlp_block); logits
    near 0.02 sqrt(d) move the loss little.  Gradients through the quantized products as there, the others by less.  A missing factor or sum is off by 0.5 and more."""
    errors = example.main(tokens, d_model, d_ffn, vocab)
    assert errors["loss"] < 0.05
    for name, off in errors.items():
        assert off < 0.4, (name, errors)


def test_micro_batches_accumulate_and_the_clipped_norm_is_the_bound(example):
    model = example.LanguageModel(1008, 272, 528)
    g = torch.Generator(device="cuda").manual_seed(3)
    ids, targets = (torch.randint(-1, 1008, (256,), generator=g, device="cuda") for _ in range(2))
    loss = model.step(ids, targets, 5)
    once = {k: v.clone() for k, v in model.grads.items()}
    assert torch.equal(loss, model.step(ids, targets, 5))
    for name, grad in model.grads.items():
        # twice the same terms: exact but for the table's, where the second pass's two additions start from a sum (each rounds once)
        bound = 0 if name != "table" else 2.0 ** -22 * once[name].abs() + 2.0 ** -22 * once[name].abs().max()
        assert bool(((grad - 2 * once[name]).abs() <= bound).all()), name
    norm64 = math.sqrt(sum(float(v.double().square().sum()) for v in model.grads.values()))
    assert abs(float(model.clip(norm64 / 8)) - norm64) <= 2.0 ** -23 * norm64
    after = math.sqrt(sum(float(v.double().square().sum()) for v in model.grads.values()))
    assert abs(after - norm64 / 8) <= 2.0 ** -22 * norm64 / 8


def logits_of(rows, cols, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (2 * torch.randn(rows, cols, generator=g, device="cuda")).bfloat16(), torch.randint(-1, cols, (rows,), generator=g, device="cuda")


class Embedding:
    def __init__(self, n, vocab, cols, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.ids, self.dout, self.vocab = torch.randint(-1, vocab, (n,), generator=g, device="cuda"), torch.randn(n, cols, generator=g, device="cuda").bfloat16(), vocab

    def run(self):
        return [nv.nvfp4_embedding_backward(self.dout, self.ids, self.vocab, scale=3.0)]


class LogProb:
    def __init__(self, rows, cols, seed):
        self.z, self.t = logits_of(rows, cols, seed)

    def run(self):
        r = nv.nvfp4_logprob_forward(self.z, self.t, entropy=True, top=5, for_backward=True)
        g = torch.full_like(r.logprob, -0.25)
        return [r.logprob, r.lse, r.entropy, r.top_index, r.top_logprob, nv.nvfp4_logprob_backward(self.z, self.t, r.stats, g_logprob=g, g_entropy=g, entropy=r.entropy),
                nv.nvfp4_logprob_with_gradient(self.z, self.t, g).dlogits]


class Clip:
    def __init__(self, sizes, seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.tensors = [torch.randn(n, generator=g, device="cuda") for n in sizes]
        self.outs = [torch.empty_like(t) for t in self.tensors]
        self.list = nv.Gradients(self.tensors, self.outs)

    def run(self):
        return [nv.nvfp4_grad_clip(self.list, nv.nvfp4_grad_sumsq(self.list), 1.0)] + self.outs


# (small, larger): calls with scratch memory, the second needing more of it
CASES = {"embedding": (lambda s: Embedding(1240, 700, 272, s), lambda s: Embedding(9000, 3000, 528, s)), "logprob": (lambda s: LogProb(3, 70000, s), lambda s: LogProb(90, 131072, s)),
         "clip": (lambda s: Clip([5000, 70000, 3], s), lambda s: Clip([1 << 20] * 8, s))}


def same(got, want):
    return len(got) == len(want) and all(torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)) for a, b in zip(got, want))


@pytest.mark.parametrize("name", CASES)
def test_replays_of_a_captured_call(name):
    case, larger = CASES[name][0](1), CASES[name][1](2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = [t.clone() for t in case.run()]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = case.run()
        want_larger = [t.clone() for t in larger.run()]
        live = [torch.full((1 << 16,), 0xAB, dtype=torch.uint8, device="cuda") for _ in range(64)]
        for _ in range(4):
            for t in out:
                t.zero_()
            graph.replay()
            got_larger = larger.run()
            side.synchronize()
            assert same(out, want) and same(got_larger, want_larger) and all(bool((t == 0xAB).all()) for t in live)


@pytest.mark.parametrize("name", CASES)
def test_two_graphs_captured_on_one_stream_run_side_by_side(name):
    cases = [CASES[name][0](s) for s in (7, 17)]
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
                t.zero_()
        torch.cuda.synchronize()


@pytest.mark.parametrize("name", CASES)
def test_two_threads_on_one_stream(name):
    cases = [CASES[name][0](s) for s in (7, 17)]
    want = [[t.clone() for t in c.run()] for c in cases]
    torch.cuda.synchronize()
    wrong = []

    def work(c, w):
        for _ in range(50):
            if not same(c.run(), w):
                wrong.append(name)
    threads = [threading.Thread(target=work, args=a) for a in zip(cases, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_the_binding_refuses_what_does_not_fit():
    z, t = logits_of(4, 96, 1)
    f = torch.zeros(4, device="cuda")
    table = torch.zeros(10, 32, device="cuda")
    stats = torch.zeros(4, 2, device="cuda")
    for call in (lambda: nv.nvfp4_logprob_forward(z, t[:3]), lambda: nv.nvfp4_logprob_forward(z, t.float()), lambda: nv.nvfp4_logprob_forward(z, t[None]), lambda: nv.nvfp4_logprob_forward(z.half()),
                 lambda: nv.nvfp4_logprob_forward(z.t()), lambda: nv.nvfp4_logprob_forward(z, t, top=33), lambda: nv.nvfp4_logprob_forward(z, t, top=-1), lambda: nv.nvfp4_logprob_forward(z, t, scale=0.0),
                 lambda: nv.nvfp4_logprob_forward(z[:, 1:], t), lambda: nv.nvfp4_logprob_forward(torch.zeros(4, 50, device="cuda"), t), lambda: nv.nvfp4_logprob_forward(z, t.cpu()),
                 lambda: nv.nvfp4_logprob_backward(z, t, stats[:, :1], g_logprob=f), lambda: nv.nvfp4_logprob_backward(z, None, stats, g_logprob=f),
                 lambda: nv.nvfp4_logprob_backward(z, t, stats, g_logprob=f[0].expand(4)), lambda: nv.nvfp4_logprob_backward(z, t, stats, g_entropy=f),
                 lambda: nv.nvfp4_logprob_backward(z, t, stats, g_logprob=f, out=z[:3]), lambda: nv.nvfp4_logprob_backward(z, t, stats, g_logprob=f, out=z, out_dtype=nv.OUT_F32),
                 lambda: nv.nvfp4_logprob_with_gradient(z, t, f[:3]), lambda: nv.nvfp4_embedding_forward(t, table[:, :24]), lambda: nv.nvfp4_embedding_forward(t[None], table),
                 lambda: nv.nvfp4_embedding_forward(t, table, out=torch.zeros(4, 48, device="cuda")), lambda: nv.nvfp4_embedding_forward(t, table, scale=math.inf),
                 lambda: nv.nvfp4_embedding_backward(table[:4], t), lambda: nv.nvfp4_embedding_backward(table[:4], t, accumulate=True, vocab=10),
                 lambda: nv.nvfp4_embedding_backward(table[:4], t, dtable=table.bfloat16()), lambda: nv.nvfp4_embedding_backward(table[:5], t, 10),
                 lambda: nv.nvfp4_embedding_backward(table[:1].expand(2000, 32).contiguous(), t.repeat(500), 10, workspace=torch.empty(16, dtype=torch.uint8, device="cuda")),
                 lambda: nv.nvfp4_grad_clip(nv.Gradients([f]), f, 1.0), lambda: nv.nvfp4_grad_clip(nv.Gradients([f]), torch.zeros(1, dtype=torch.float64, device="cuda"), -1.0),
                 lambda: nv.nvfp4_grad_sumsq(nv.Gradients([f]), out=f[:1])):
        with pytest.raises((ValueError, nv.NVFP4Error)):
            call()
    torch.cuda.synchronize()
