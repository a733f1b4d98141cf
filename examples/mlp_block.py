"""One MLP block of a transformer, trained in NVFP4: forward and backward through the library's calls, as a training program makes them.

    h = x + r                                   the residual stream (bf16)
    n = norm(h) * gamma                         nvfp4_rmsnorm_forward; the normalised rows are kept in 8 bits, not h
    z = n W1 + b1;  a = max(z, 0)^2             nvfp4_gemm_epilogue; z is kept in 8 bits, a is not kept
    y = a W2 + b2 + h                           nvfp4_gemm_epilogue

Kept for the backward pass: 1.06 bytes a value of the normalised rows and of z, a float per row, and the rotated 4-bit copies of
both products' inputs that the weight gradients contract over.  The backward pass reads these alone:

    dz = (dy W2^T) * act'(z)                    nvfp4_gemm_epilogue on the 8 bits of z
    dW2 = a^T dy, dW1 = n^T dz                  nvfp4_gemm, FP32, accumulated over micro-batches
    db2, db1                                    nvfp4_activation_backward
    dx = dr = norm's gradient of (dz W1^T) + dy nvfp4_rmsnorm_backward on the 8 bits of the normalised rows

Run it on a GPU (12B sizes: ``python examples/mlp_block.py 8192 5120 20480``); it prints the time of a step and how far the step's results
are from the same block in 64-bit arithmetic.
"""
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2509_25149_amd import binding as nv  # noqa: E402

RC = nv.LAYOUT_ROW | nv.LAYOUT_COL


def keep_col_copy(q: nv.QTensor) -> nv.QTensor:
    """Give a quantized tensor's row copy back: its memory, and its place in the descriptor, so that a call that asks for it is refused."""
    q.row_codes = q.row_scales = q.row_ts = None
    q.desc.row_codes = q.desc.row_scales = q.desc.row_tensor_scale = None
    q.desc.layout_mask &= ~nv.LAYOUT_ROW
    return q


class MlpBlock:
    """Parameters in FP32 or bf16, gradients in FP32; sizes multiples of 16."""

    def __init__(self, d_model: int, d_ffn: int, seed: int = 0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *size: torch.randn(*size, generator=g, device="cuda")
        self.d_model, self.d_ffn = d_model, d_ffn
        self.gamma = 1.0 + 0.1 * normal(d_model)
        self.w1, self.w2 = (0.02 * normal(d_model, d_ffn)).bfloat16(), (0.02 * normal(d_ffn, d_model)).bfloat16()
        self.b1, self.b2 = 0.02 * normal(d_ffn), 0.02 * normal(d_model)
        self.grads = {name: torch.zeros_like(p, dtype=torch.float32) for name, p in self.parameters().items()}
        self.rht_seed = 2025
        self.quantize_weights()

    def parameters(self):
        return dict(gamma=self.gamma, w1=self.w1, b1=self.b1, w2=self.w2, b2=self.b2)

    def quantize_weights(self):
        """Once per optimizer step: 16x16 blocks, both orientations from the same codes."""
        self.q1, self.q2 = nv.nvfp4_quantize(self.w1, RC, nv.BLOCK_16x16), nv.nvfp4_quantize(self.w2, RC, nv.BLOCK_16x16)

    def _workspace(self, tokens: int) -> torch.Tensor:
        need = nv.linear_workspace_bytes(tokens, self.d_model, self.d_ffn)
        if getattr(self, "workspace", None) is None or self.workspace.numel() < need:
            self.workspace = torch.empty(need, dtype=torch.uint8, device="cuda")
        return self.workspace

    def forward(self, x: torch.Tensor, r: torch.Tensor):
        """Returns y and what the backward pass needs."""
        tokens = x.shape[0]
        ws = self._workspace(tokens)
        norm = nv.nvfp4_rmsnorm_forward(x, self.gamma, residual=r, checkpoint=True)
        qn = nv.nvfp4_quantize(norm.y, RC, rht_on_col=True, rht_seed=self.rht_seed)
        z = nv.alloc_checkpoint(tokens, self.d_ffn)
        a = nv.nvfp4_gemm_epilogue(qn, self.q1, nv.OP_FPROP, bias=self.b1, activation=nv.ACT_RELU2, keep=z, workspace=ws)
        qa = nv.nvfp4_quantize(a, RC, rht_on_col=True, rht_seed=self.rht_seed)
        y = nv.nvfp4_gemm_epilogue(qa, self.q2, nv.OP_FPROP, bias=self.b2, residual=norm.h, workspace=ws)
        return y, (norm.checkpoint, norm.rstd, keep_col_copy(qn), z, keep_col_copy(qa))      # (the row copies have done their work)

    def backward(self, dy: torch.Tensor, saved, sr_seed: int = 0):
        """Adds to the gradients; returns the gradient of x and of r, which are one."""
        xhat, rstd, qn, z, qa = saved
        ws, g = self._workspace(dy.shape[0]), self.grads
        sr = dict(rounding=nv.ROUND_SR, rht_on_col=True, rht_seed=self.rht_seed)
        qdy = nv.nvfp4_quantize(dy, RC, sr_seed=2 * sr_seed, **sr)
        nv.nvfp4_activation_backward(dy, want_dz=False, dbias=g["b2"], accumulate_dbias=True)
        nv.nvfp4_gemm(qa, qdy, nv.OP_WGRAD, nv.OUT_F32_ACCUMULATE, out=g["w2"], workspace=ws)
        dz = nv.nvfp4_gemm_epilogue(qdy, self.q2, nv.OP_DGRAD, activation=nv.ACT_RELU2, grad_of=z, workspace=ws)
        qdz = nv.nvfp4_quantize(dz, RC, sr_seed=2 * sr_seed + 1, **sr)
        nv.nvfp4_activation_backward(dz, want_dz=False, dbias=g["b1"], accumulate_dbias=True)
        nv.nvfp4_gemm(qn, qdz, nv.OP_WGRAD, nv.OUT_F32_ACCUMULATE, out=g["w1"], workspace=ws)
        dn = nv.nvfp4_gemm(qdz, self.q1, nv.OP_DGRAD, nv.OUT_BF16, workspace=ws)
        dx, _ = nv.nvfp4_rmsnorm_backward(dn, xhat, rstd, self.gamma, dres=dy, dgamma=g["gamma"], accumulate_dgamma=True)
        return dx


def exact(block: MlpBlock, x, r, dy, eps: float = 1e-5):
    """The same block with nothing quantized, in binary64 with autograd: y, dx and the parameters' gradients."""
    p = {name: t.double().requires_grad_() for name, t in block.parameters().items()}
    x64 = x.double().requires_grad_()
    h = x64 + r.double()
    n = h * torch.rsqrt(h.square().mean(1, keepdim=True) + eps) * p["gamma"]
    z = n @ p["w1"] + p["b1"]
    y = z.clamp_min(0).square() @ p["w2"] + p["b2"] + h
    y.backward(dy.double())
    return y.detach(), x64.grad, {name: t.grad for name, t in p.items()}


def main(tokens: int = 1024, d_model: int = 1280, d_ffn: int = 5120):
    block = MlpBlock(d_model, d_ffn)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, r = (torch.randn(tokens, d_model, generator=g, device="cuda").bfloat16() for _ in range(2))
    dy = (1e-3 * torch.randn(tokens, d_model, generator=g, device="cuda")).bfloat16()
    y, saved = block.forward(x, r)
    dx = block.backward(dy, saved)
    off = lambda got, want: float((got.double() - want).norm() / want.norm())
    y64, dx64, grads = exact(block, x, r, dy)
    errors = dict(y=off(y, y64), dx=off(dx, dx64), **{name: off(block.grads[name], grads[name]) for name in grads})
    del y64, dx64, grads
    torch.cuda.synchronize()
    steps, began = 10, time.perf_counter()
    for step in range(steps):
        y, saved = block.forward(x, r)
        block.backward(dy, saved, step)
    torch.cuda.synchronize()
    ms = (time.perf_counter() - began) / steps * 1e3
    print(f"MLP block, {tokens} x {d_model} -> {d_ffn}: {ms:.3f} ms a step ({12 * tokens * d_model * d_ffn / ms * 1e-9:.0f} TFLOP/s of products)")
    print("distance from the block in 64 bits:", ", ".join(f"{k} {v:.3f}" for k, v in errors.items()))
    return errors


if __name__ == "__main__":
    main(*(int(v) for v in sys.argv[1:4]))
