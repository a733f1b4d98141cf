"""The two ends of a language model's training step, and what stands between its gradients and the optimizer, as measurable
cases: the embedding's lookup and gradient; log probabilities of given tokens with entropy, top alternatives and the gradient
of the logits; the norm over all gradients and clipping.

A case is one pass through ``paper_2509_25149_amd.binding``.  Sizes are those of the 12B model (model dimension 5120, FFN
dimension 20480, 8192 tokens) with a vocabulary of 131072, of the ragged layers measured elsewhere here, and single tokens.
Token numbers follow Zipf's law and 1 % of them are padding (-1), logits are N(0, 2^2) with the right token often
ahead, gradients 1e-3 N(0, 1).

With ``own`` false ``run`` computes the same results from elementary torch operations in 32 bits (64 for the sum of squares).
``exact`` computes them from the definitions in 64 bits.
"""
import math
import random

import numpy as np
import torch

own = False

TOKENS, D_MODEL, D_FFN, VOCAB = 8192, 5120, 20480, 131072
F32, BF16 = "f32", "bf16"
DTYPE = {F32: torch.float32, BF16: torch.bfloat16}
SIZE = {F32: 4, BF16: 2}
IDS = {"i32": torch.int32, "i64": torch.int64}


# ---------------------------------------------------------------- the cases

def listed():
    return [
        # The token that was just sampled, on its way back into the model: a launch and its latency.
        dict(name="embed_one_token", kind="embed", tokens=1, vocab=VOCAB, cols=D_MODEL, table=BF16, out=BF16, ids="i64", scale=1.0),
        # A sequence of the 12B model, rows scaled by the square root of their length.
        dict(name="embed_12b", kind="embed", tokens=TOKENS, vocab=VOCAB, cols=D_MODEL, table=BF16, out=BF16, ids="i64", scale=math.sqrt(D_MODEL)),
        # The embedding's gradient in a small ragged model.
        dict(name="embed_grad_ragged", kind="embed_grad", tokens=1040, vocab=5003, cols=2064, dout=F32, ids="i32", scale=1.0),
        # The same for a sequence of the 12B model: the whole gradient is written, rows without a token as zeros.
        dict(name="embed_grad_12b", kind="embed_grad", tokens=TOKENS, vocab=VOCAB, cols=D_MODEL, dout=BF16, ids="i64", scale=math.sqrt(D_MODEL)),
        # One decoded token: its log probability, the entropy and the best alternatives, over a vocabulary whose end is padding.
        dict(name="logprob_one_token", kind="logprob", rows=1, cols=VOCAB, x=F32, ids="i64", scale=1.0, entropy=True, top=8, masked=True),
        # A batch of decoded tokens over a vocabulary of odd size, at a temperature.
        dict(name="logprob_batch_top", kind="logprob", rows=64, cols=50257, x=BF16, ids="i64", scale=1.25, entropy=True, top=20, masked=False),
        # A sequence that is scored: log probabilities and entropies.
        dict(name="logprob_sequence", kind="logprob", rows=TOKENS, cols=VOCAB, x=BF16, ids="i64", scale=1.0, entropy=True, top=0, masked=True),
        # Gradient of a reinforcement-learning loss: of the log probability, of the normaliser and of the entropy.
        dict(name="logprob_grad_odd", kind="logprob_grad", rows=1040, cols=50257, x=F32, ids="i32", scale=1.0, entropy=True, lse=True, masked=False, out=F32),
        # A training step's loss and the logits' gradient on a ragged batch.
        dict(name="loss_ragged", kind="loss", rows=517, cols=50257, x=BF16, ids="i64", scale=1.0, masked=False, out=BF16),
        # The same for a sequence of the 12B model: the largest.
        dict(name="loss_sequence", kind="loss", rows=TOKENS, cols=VOCAB, x=BF16, ids="i64", scale=1.0, masked=True, out=BF16),
        # The gradients of a small model: many tensors, each a fraction of what fills the chip.
        dict(name="clip_many_small", kind="clip", tensors=384, lo=16, hi=70000, total=1 << 23, types="mixed", strided=True, max_norm=0.5, sizes=1),
        # The gradients of the 12B model's MLP block, accumulated in FP32.
        dict(name="clip_12b_block", kind="clip", tensors=5, lo=0, hi=0, total=0, types=F32, strided=False, max_norm=1.0, sizes=0),
    ]


def _size(rng, lo, hi, multiple=1):
    """Log-uniform in [lo, hi]; half of the sizes any multiple of the unit, half round ones."""
    n = lo * (hi / lo) ** rng.random()
    step = multiple if rng.random() < 0.5 else max(multiple, 256 if n >= 1024 else 64 if n >= 128 else multiple)
    return min(hi, max(lo, int(round(n / step)) * step))


def draw(rng):
    kind = rng.choice(["embed", "embed_grad", "embed_grad", "logprob", "logprob", "logprob_grad", "loss", "loss", "clip", "clip"])
    x, out, ids = rng.choice([BF16, BF16, F32]), rng.choice([BF16, F32]), rng.choice(["i32", "i64"])
    scale = rng.choice([1.0, 1.0, 0.7])
    if kind in ("embed", "embed_grad"):
        case = dict(kind=kind, tokens=_size(rng, 1, 4 * TOKENS), vocab=_size(rng, 500, VOCAB), cols=_size(rng, 64, D_MODEL, 16), ids=ids, scale=scale)
        return dict(case, table=x, out=out) if kind == "embed" else dict(case, dout=x)
    if kind == "clip":
        n = _size(rng, 1, 512)
        hi = _size(rng, 1000, 1 << 26)
        return dict(kind=kind, tensors=n, lo=rng.choice([1, 16, 5120]), hi=max(hi, 5120), total=1 << 27, types=rng.choice([F32, F32, BF16, "mixed"]),
                    strided=rng.random() < 0.3, max_norm=rng.choice([1.0, 1e-3, 1e4]), sizes=rng.randrange(1, 1 << 30))
    while True:
        rows, cols = _size(rng, 1, TOKENS), _size(rng, 100, 2 * VOCAB)
        if rows * cols * SIZE[x] <= TOKENS * VOCAB * 2 and rows * cols * (SIZE[x] + SIZE[out]) <= TOKENS * VOCAB * 4:
            break
    case = dict(kind=kind, rows=rows, cols=cols, x=x, ids=ids, scale=scale, masked=rng.random() < 0.3)
    if kind == "logprob":
        return dict(case, entropy=rng.random() < 0.5, top=rng.choice([0, 1, 5, 20, 32]) if rows * cols <= 1 << 26 else 0)
    if kind == "logprob_grad":
        return dict(case, entropy=rng.random() < 0.5, lse=rng.random() < 0.5, out=out)
    return dict(case, out=out)


# ---------------------------------------------------------------- inputs

class _Inputs:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda")

    def uniform(self, *shape):
        return torch.rand(*shape, generator=self.g, device="cuda", dtype=torch.float64)

    def tokens(self, n, vocab, dtype, missing):
        """Token k (from 0) about as often as 1 / (k + 1); a fraction `missing` of them -1."""
        ids = ((vocab + 1.0) ** self.uniform(n)).long().clamp(1, vocab) - 1
        return torch.where(self.uniform(n) < missing, torch.full_like(ids, -1), ids).to(dtype)

    def logits(self, case, targets, limit):
        rows, cols = case["rows"], case["cols"]
        ld = -(-cols // 8) * 8                                   # rows start at multiples of 16 bytes
        z = torch.empty(rows, ld, dtype=DTYPE[case["x"]], device="cuda")
        for r in range(0, rows, 1024):
            part = self.normal(min(1024, rows - r), ld) * 2.0
            t = targets[r:r + 1024].long().clamp_min(0)
            lift = torch.where(self.uniform(part.shape[0]) < 0.5, 8.0, 0.0).float()
            part.scatter_add_(1, t[:, None], lift[:, None])
            if case["masked"]:
                part[:, limit:] = -math.inf
            z[r:r + 1024] = part.to(z.dtype)
        return z[:, :cols]


def _block_shapes():
    return [(D_MODEL,), (D_MODEL, D_FFN), (D_FFN,), (D_FFN, D_MODEL), (D_MODEL,)]


def _shapes(case):
    """Shape, type and distance of rows (0: contiguous) of each tensor: vectors, and matrices of up to 64 rows."""
    if not case["sizes"]:
        return [(shape, case["types"], 0) for shape in _block_shapes()]
    r, out, total = random.Random(case["sizes"]), [], 0
    for i in range(case["tensors"]):
        n = int(case["lo"] * (case["hi"] / case["lo"]) ** r.random())
        n = max(1, min(n, case["total"] - total))
        total += n
        dtype = case["types"] if case["types"] != "mixed" else (F32, BF16)[i % 2]
        rows = r.choice([1, 1, 16, 64]) if n >= 1024 else 1
        shape = (rows, n // rows) if rows > 1 else (n,)
        out.append((shape, dtype, n // rows + 8 * r.randrange(1, 4) if rows > 1 and case["strided"] else 0))
        if total >= case["total"]:
            break
    return out


def _flat(tensors, dtype=None):
    """One buffer for each type, and the places of the tensors in it, as an optimizer or a reduction over GPUs takes them."""
    size, places = {}, []
    for t in tensors:
        at = size.get(t.dtype, 0)
        places.append(at)
        size[t.dtype] = at + -(-t.numel() // 64) * 64
    flat = {d: torch.zeros(n, dtype=dtype or d, device="cuda") for d, n in size.items()}
    return flat, [flat[t.dtype][at:at + t.numel()].view(t.shape) for t, at in zip(tensors, places)]


def _clipped(norm, flat):
    return {"norm": norm, **{"grads_" + str(d).split(".")[1]: t for d, t in flat.items()}}


def prepare(case, seed):
    gen, kind = _Inputs(seed), case["kind"]
    s = dict(case=case)
    if kind == "embed":
        s["ids"] = gen.tokens(case["tokens"], case["vocab"], IDS[case["ids"]], 0.01 if case["tokens"] > 1 else 0.0)
        s["table"] = (0.02 * gen.normal(case["vocab"], case["cols"])).to(DTYPE[case["table"]])
    elif kind == "embed_grad":
        s["ids"] = gen.tokens(case["tokens"], case["vocab"], IDS[case["ids"]], 0.01)
        s["dout"] = (1e-3 * gen.normal(case["tokens"], case["cols"])).to(DTYPE[case["dout"]])
    elif kind == "clip":
        s["grads"] = []
        for shape, dtype, ld in _shapes(case):
            t = torch.empty(shape[0], ld, dtype=DTYPE[dtype], device="cuda")[:, :shape[1]] if ld else torch.empty(shape, dtype=DTYPE[dtype], device="cuda")
            s["grads"].append(t.copy_(1e-3 * gen.normal(*shape)))
        s["flat"], s["outs"] = _flat(s["grads"])
        if own:   # the list of its gradients that a program keeps
            from paper_2509_25149_amd import binding as nv
            s["list"] = nv.Gradients(s["grads"], s["outs"])
    else:
        limit = case["cols"] - case["cols"] // 16 if case["masked"] else case["cols"]
        s["targets"] = gen.tokens(case["rows"], limit, IDS[case["ids"]], 0.02 if case["rows"] > 1 else 0.0)
        s["logits"] = gen.logits(case, s["targets"], limit)
        if kind != "logprob":
            s["g"] = (-1.0 / case["rows"]) * (0.5 + gen.uniform(case["rows"])).float()
        if kind == "logprob_grad":   # what the forward pass gave, as the framework keeps it
            s["g_lse"] = 1e-3 * gen.normal(case["rows"]) if case["lse"] else None
            s["g_entropy"] = 1e-3 * gen.normal(case["rows"]) if case["entropy"] else None
            m, logsum, entropy = [], [], []
            for r in range(0, case["rows"], 1024):
                a, b, c = _statistics(s["logits"][r:r + 1024].double(), case["scale"])
                m.append(a), logsum.append(b), entropy.append(c)
            s["stats"] = torch.stack([torch.cat(m), torch.cat(logsum)], 1).float()
            s["entropy"] = torch.cat(entropy).float() if case["entropy"] else None
    return s


# ---------------------------------------------------------------- one pass, plainly

def _statistics(z, scale):
    """Largest logit, log of the sum of exp(scale (z - largest)), entropy."""
    m = z.amax(1)
    d = (z - m[:, None]) * scale
    e = torch.exp(d)
    s = e.sum(1)
    logsum = torch.log(s)
    return m, logsum, logsum - torch.where(e > 0, e * d, torch.zeros_like(e)).sum(1) / s


def _named(**outputs):
    return {k: v for k, v in outputs.items() if v is not None}


def _at_target(z, m, logsum, targets, scale):
    """Log probability of the targets; 0 where there is none."""
    t = targets.long()
    at = (torch.gather(z, 1, t.clamp(0, z.shape[1] - 1)[:, None])[:, 0] - m) * scale - logsum
    return torch.where((t >= 0) & (t < z.shape[1]), at, torch.zeros_like(at))


def _gradient(z, m, logsum, targets, scale, g, g_lse=None, g_entropy=None, entropy=None):
    t = targets.long()
    g = torch.where((t >= 0) & (t < z.shape[1]), g.to(z.dtype), torch.zeros_like(m))
    logp = (z - m[:, None]) * scale - logsum[:, None]
    p = torch.exp(logp)
    factor = (-g if g_lse is None else g_lse.to(z.dtype) - g)[:, None]
    if g_entropy is not None:
        factor = factor - g_entropy.to(z.dtype)[:, None] * torch.where(p > 0, logp + entropy.to(z.dtype)[:, None], torch.zeros_like(p))
    dz = p * factor
    dz.scatter_add_(1, t.clamp(0, z.shape[1] - 1)[:, None], g[:, None])
    return dz * scale


def _plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "embed":
        ids = s["ids"].long()
        rows = s["table"][ids.clamp(0, case["vocab"] - 1)].float() * case["scale"]
        return _named(out=torch.where(((ids >= 0) & (ids < case["vocab"]))[:, None], rows, torch.zeros_like(rows)).to(DTYPE[case["out"]]))
    if kind == "embed_grad":
        ids = s["ids"].long()
        rows = torch.where(((ids >= 0) & (ids < case["vocab"]))[:, None], s["dout"].float(), torch.zeros((), device="cuda"))
        dtable = torch.zeros(case["vocab"], case["cols"], device="cuda")
        dtable.index_add_(0, ids.clamp(0, case["vocab"] - 1), rows)
        return _named(dtable=dtable * case["scale"])
    if kind == "clip":
        sumsq = torch.stack([t.double().square().sum() for t in s["grads"]]).sum()
        norm = sumsq.sqrt()
        coef = torch.where(norm > case["max_norm"], case["max_norm"] / norm, torch.ones_like(norm)).float()
        for t, o in zip(s["grads"], s["outs"]):
            o.copy_(t.float() * coef)
        return _clipped(norm.float().reshape(1), s["flat"])
    z, scale = s["logits"].float(), case["scale"]
    if kind == "logprob_grad":
        dz = _gradient(z, s["stats"][:, 0], s["stats"][:, 1], s["targets"], scale, s["g"], s["g_lse"], s["g_entropy"], s["entropy"])
        return _named(dlogits=dz.to(DTYPE[case["out"]]))
    if kind == "loss":
        m = z.amax(1)
        logsum = torch.log(torch.exp((z - m[:, None]) * scale).sum(1))
        return _named(logprob=_at_target(z, m, logsum, s["targets"], scale), lse=m * scale + logsum,
                      dlogits=_gradient(z, m, logsum, s["targets"], scale, s["g"]).to(DTYPE[case["out"]]))
    m, logsum, entropy = _statistics(z, scale)
    out = _named(logprob=_at_target(z, m, logsum, s["targets"], scale), lse=m * scale + logsum, entropy=entropy if case["entropy"] else None)
    if case["top"]:
        v, i = torch.sort(z, dim=1, descending=True, stable=True)
        out.update(top_index=i[:, :case["top"]].int(), top_logprob=(v[:, :case["top"]] - m[:, None]) * scale - logsum[:, None])
    return out


# ---------------------------------------------------------------- one pass, through the framework

def run(state):
    if not own:
        return _plain(state)
    from paper_2509_25149_amd import binding as nv
    case, kind = state["case"], state["case"]["kind"]
    out_type = {F32: nv.OUT_F32, BF16: nv.OUT_BF16}
    if kind == "embed":
        return _named(out=nv.nvfp4_embedding_forward(state["ids"], state["table"], scale=case["scale"], out_dtype=out_type[case["out"]]))
    if kind == "embed_grad":
        return _named(dtable=nv.nvfp4_embedding_backward(state["dout"], state["ids"], case["vocab"], scale=case["scale"]))
    if kind == "clip":
        norm = nv.nvfp4_grad_clip(state["list"], nv.nvfp4_grad_sumsq(state["list"]), case["max_norm"])
        return _clipped(norm, state["flat"])
    if kind == "logprob_grad":
        return _named(dlogits=nv.nvfp4_logprob_backward(state["logits"], state["targets"], state["stats"], g_logprob=state["g"], g_lse=state["g_lse"],
                                                        g_entropy=state["g_entropy"], entropy=state["entropy"], scale=case["scale"],
                                                        out_dtype=out_type[case["out"]]))
    if kind == "loss":
        r = nv.nvfp4_logprob_with_gradient(state["logits"], state["targets"], state["g"], scale=case["scale"], out_dtype=out_type[case["out"]])
        return _named(logprob=r.logprob, lse=r.lse, dlogits=r.dlogits)
    r = nv.nvfp4_logprob_forward(state["logits"], state["targets"], scale=case["scale"], entropy=case["entropy"], top=case["top"])
    return _named(logprob=r.logprob, lse=r.lse, entropy=r.entropy, top_index=r.top_index, top_logprob=r.top_logprob)


# ---------------------------------------------------------------- 64 bits

def exact(case, seed):
    s, kind, f64, scale = prepare(case, seed), case["kind"], torch.float64, case.get("scale")
    if kind == "embed":
        out = torch.zeros(case["tokens"], case["cols"], dtype=f64, device="cuda")
        there = (s["ids"] >= 0).nonzero()[:, 0]
        out[there] = torch.index_select(s["table"], 0, s["ids"][there].long()).to(f64) * scale
        return _named(out=out)
    if kind == "embed_grad":
        there = (s["ids"] >= 0).nonzero()[:, 0]
        return _named(dtable=torch.zeros(case["vocab"], case["cols"], dtype=f64, device="cuda").index_add_(0, s["ids"][there].long(), s["dout"][there].to(f64) * scale))
    if kind == "clip":
        norm = math.sqrt(sum(float(torch.linalg.vector_norm(t.to(f64))) ** 2 for t in s["grads"]))
        coef = min(1.0, case["max_norm"] / norm)
        flat, outs = _flat(s["grads"], f64)
        for t, o in zip(s["grads"], outs):
            o.copy_(t.to(f64) * coef)
        return _clipped(torch.tensor([norm], dtype=f64, device="cuda"), flat)
    parts = []
    for r in range(0, case["rows"], 512):
        z = s["logits"][r:r + 512].to(f64)
        t = s["targets"][r:r + 512].long()
        counted, row = t >= 0, torch.arange(z.shape[0], device="cuda")
        y = z * scale
        if kind == "logprob_grad":
            lse = s["stats"][r:r + 512, 0].to(f64) * scale + s["stats"][r:r + 512, 1].to(f64)     # the forward pass's, as it was handed on
        else:
            lse = torch.logsumexp(y, 1)
        logp = y - lse[:, None]
        p = torch.exp(logp)
        part = {}
        if kind == "logprob":
            part.update(logprob=torch.where(counted, logp[row, t.clamp_min(0)], 0.0), lse=lse)
            if case["entropy"]:
                part["entropy"] = -torch.nan_to_num(p * logp, nan=0.0).sum(1)
            if case["top"]:
                key = np.argsort(-z.cpu().numpy(), axis=1, kind="stable")[:, :case["top"]]
                key = torch.from_numpy(key).cuda()
                part.update(top_index=key.int(), top_logprob=torch.gather(logp, 1, key))
        else:
            g = torch.where(counted, s["g"][r:r + 512].to(f64), 0.0)
            dz = -g[:, None] * p
            if kind == "loss":
                part.update(logprob=torch.where(counted, logp[row, t.clamp_min(0)], 0.0), lse=lse)
            else:
                if s["g_lse"] is not None:
                    dz = dz + s["g_lse"][r:r + 512].to(f64)[:, None] * p
                if s["g_entropy"] is not None:
                    h = s["entropy"][r:r + 512].to(f64)[:, None]
                    dz = dz - s["g_entropy"][r:r + 512].to(f64)[:, None] * torch.nan_to_num(p * (logp + h), nan=0.0)
            dz[row, t.clamp_min(0)] += g
            part["dlogits"] = dz * scale
        parts.append(part)
    return {k: torch.cat([p[k] for p in parts]) for k in parts[0]}


# ---------------------------------------------------------------- what a pass cannot do without

def _distinct(n, vocab):
    """Expected number of different tokens among n."""
    k = np.arange(1, vocab + 1, dtype=np.float64)
    p = np.log1p(1 / k) / math.log(vocab + 1.0)
    return float((-np.expm1(n * np.log1p(-np.minimum(p, 1 - 1e-12)))).sum())


def work(case):
    kind = case["kind"]
    if kind == "embed":
        n = case["tokens"]
        return dict(bytes=case["cols"] * (_distinct(n, case["vocab"]) * SIZE[case["table"]] + n * SIZE[case["out"]]) + n * (4 if case["ids"] == "i32" else 8),
                    flops=n * case["cols"])
    if kind == "embed_grad":
        n = case["tokens"]
        return dict(bytes=case["cols"] * (n * SIZE[case["dout"]] + case["vocab"] * 4) + n * (4 if case["ids"] == "i32" else 8), flops=2 * n * case["cols"])
    if kind == "clip":
        count = {F32: 0, BF16: 0}
        for shape, dtype, _ in _shapes(case):
            count[dtype] += math.prod(shape)
        return dict(bytes=8 * count[F32] + 4 * count[BF16], flops=3 * (count[F32] + count[BF16]))
    n = case["rows"] * case["cols"]
    if kind == "logprob":
        return dict(bytes=n * SIZE[case["x"]] + case["rows"] * (16 + 8 * case["top"]), flops=(7 if case["entropy"] else 5) * n)
    return dict(bytes=n * (SIZE[case["x"]] + SIZE[case["out"]]) + case["rows"] * 24, flops=8 * n)
