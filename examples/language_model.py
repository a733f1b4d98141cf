"""A training step of a language model, from token numbers to clipped gradients: the MLP block of mlp_block.py between its two ends.

    e = table[ids] * sqrt(d)                    nvfp4_embedding_forward
    y = the block                               mlp_block.py, its linear layers in NVFP4
    n = norm(y) * gamma                         nvfp4_rmsnorm_forward
    logits = n table^T                          a bf16 product (the recipe keeps the output head so); the head's weight is the table
    loss = -mean of the targets' ln p           nvfp4_logprob_with_gradient, which writes the logits' gradient over the logits

and back: the head's products, the norm's and the block's gradients, then the embedding's, which is added to what the head has left in the table's gradient.
All gradients are FP32 and accumulate over micro-batches.  Before the optimizer they are clipped to a common norm (nvfp4_grad_sumsq, nvfp4_grad_clip).

``python examples/language_model.py 8192 5120 20480 131072`` prints the time of a step, and how far its results are from the same model in 64 bits where those
fit the memory.
"""
import math
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))

from mlp_block import MlpBlock  # noqa: E402
from paper_2509_25149_amd import binding as nv  # noqa: E402


class LanguageModel:
    def __init__(self, vocab: int, d_model: int, d_ffn: int, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed + 1)
        self.block = MlpBlock(d_model, d_ffn, seed)
        self.table = (0.02 * torch.randn(vocab, d_model, generator=g, device="cuda")).bfloat16()
        self.gamma = 1.0 + 0.1 * torch.randn(d_model, generator=g, device="cuda")
        self.scale = math.sqrt(d_model)
        self.grads = dict(self.block.grads, table=torch.zeros(vocab, d_model, device="cuda"), out_gamma=torch.zeros(d_model, device="cuda"))
        self.list = nv.Gradients(self.grads.values())      # once: every step uses these tensors

    def parameters(self):
        return dict(self.block.parameters(), table=self.table, out_gamma=self.gamma)

    def step(self, ids: torch.Tensor, targets: torch.Tensor, sr_seed: int = 0) -> torch.Tensor:
        """One micro-batch: adds to the gradients of the mean loss over the targets inside the vocabulary; returns the loss."""
        g = self.grads
        e = nv.nvfp4_embedding_forward(ids, self.table, scale=self.scale)
        y, saved = self.block.forward(torch.zeros_like(e), e)
        norm = nv.nvfp4_rmsnorm_forward(y, self.gamma)
        vocab = self.table.shape[0]
        logits = torch.empty(len(ids), -(-vocab // 8) * 8, dtype=norm.y.dtype, device=ids.device)[:, :vocab]     # rows at multiples of 8, as the log probabilities take them
        torch.mm(norm.y, self.table.t(), out=logits)
        counted = ((targets >= 0) & (targets < vocab)).sum().clamp_min(1)
        weight = (-1.0 / counted).expand(targets.shape).contiguous()
        out = nv.nvfp4_logprob_with_gradient(logits, targets, weight, out=logits)
        dlogits = out.dlogits
        dn = torch.mm(dlogits, self.table)
        g["table"] += torch.mm(dlogits.t(), norm.y)
        dy, _ = nv.nvfp4_rmsnorm_backward(dn, y, norm.rstd, self.gamma, dgamma=g["out_gamma"], accumulate_dgamma=True)
        de = self.block.backward(dy, saved, sr_seed)
        nv.nvfp4_embedding_backward(de, ids, dtable=g["table"], scale=self.scale, accumulate=True)
        return (out.logprob * weight).sum()

    def clip(self, max_norm: float) -> torch.Tensor:
        """All gradients scaled so that their norm is at most max_norm; returns the norm that they had."""
        return nv.nvfp4_grad_clip(self.list, nv.nvfp4_grad_sumsq(self.list), max_norm)


def exact(model: LanguageModel, ids, targets, eps: float = 1e-5):
    """The same model with nothing quantized, in binary64 with autograd: loss and the parameters' gradients."""
    p = {name: t.double().requires_grad_() for name, t in model.parameters().items()}
    rms = lambda v: v * torch.rsqrt(v.square().mean(1, keepdim=True) + eps)
    vocab = p["table"].shape[0]
    there = ((ids >= 0) & (ids < vocab))[:, None]
    h = torch.where(there, p["table"][ids.clamp(0, vocab - 1)] * model.scale, 0.0)
    y = (rms(h) * p["gamma"] @ p["w1"] + p["b1"]).clamp_min(0).square() @ p["w2"] + p["b2"] + h
    logp = torch.log_softmax((rms(y) * p["out_gamma"]) @ p["table"].t(), 1)
    counted = (targets >= 0) & (targets < vocab)
    loss = -torch.where(counted, logp.gather(1, targets.clamp(0, vocab - 1)[:, None])[:, 0], 0.0).sum() / counted.sum().clamp_min(1)
    loss.backward()
    return loss.detach(), {name: t.grad for name, t in p.items()}


def main(tokens: int = 1024, d_model: int = 512, d_ffn: int = 2048, vocab: int = 8192):
    model = LanguageModel(vocab, d_model, d_ffn)
    g = torch.Generator(device="cuda").manual_seed(1)
    ids, targets = (torch.randint(0, vocab, (tokens,), generator=g, device="cuda") for _ in range(2))
    ids[tokens // 3] = targets[tokens // 2] = -1            # padding
    loss = model.step(ids, targets)
    errors = {}
    if tokens * vocab <= 1 << 26:
        loss64, grads = exact(model, ids, targets)
        off = lambda got, want: float((got.double() - want).norm() / want.norm())
        errors = dict(loss=off(loss, loss64), **{name: off(model.grads[name], grads[name]) for name in grads})
    model.clip(1.0)
    torch.cuda.synchronize()
    steps, began = 10, time.perf_counter()
    for step in range(steps):
        model.step(ids, targets, step)
        norm = model.clip(1.0)
    torch.cuda.synchronize()
    ms = (time.perf_counter() - began) / steps * 1e3
    print(f"language model, {tokens} tokens, {d_model} -> {d_ffn}, vocabulary {vocab}: {ms:.3f} ms a step, gradient norm {float(norm):.4f}")
    if errors:
        print("distance from the model in 64 bits:", ", ".join(f"{k} {v:.4f}" for k, v in errors.items()))
    return errors


if __name__ == "__main__":
    main(*(int(v) for v in sys.argv[1:5]))
