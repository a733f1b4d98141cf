"""What stands next to the quantized linear layers in a transformer block, as measurable cases: the residual's addition
and root-mean-square norm in front of the first one, bias / activation / residual behind a product, the 8-bit
checkpoints of activations, and the backward pass that reads them.

A case is one call through ``paper_2509_25149_amd.binding``.  Sizes are those of the 12B model's MLP (model dimension
5120, FFN dimension 20480, 8192 tokens), of the small parity configuration (256 tokens, 512 -> 256), and ragged layers in
between.  Values are the synthetic stand-ins used elsewhere here: activations N(0, 1) with 0.1 % outliers of 50, weights
N(0, 0.02^2), gradients 1e-3 Student-t(3).

With ``own`` false ``run`` computes the same results from elementary torch operations in 32 bits.  ``exact`` computes them
from the definitions in 64 bits.  Tensors held in 8 bits come back as codes and scales, each viewed as the
numbers that its bytes stand for.
"""
import torch

own = False

TOKENS, D_MODEL, D_FFN = 8192, 5120, 20480      # the 12B model's MLP on one sequence
BLOCK = 16                                      # columns that share a scale, in 8 bits as in 4
F32, BF16 = "f32", "bf16"
DTYPE = {F32: torch.float32, BF16: torch.bfloat16}
EPS = 1e-5


# ---------------------------------------------------------------- the cases

def listed():
    return [
        # One new token on its way into a layer: residual added, normed, kept in 8 bits as well; a launch and its latency.
        dict(name="norm_one_token", kind="norm", rows=1, cols=D_MODEL, x=BF16, stream=BF16, y=BF16, residual=True, gamma=True, out8=True, pad=0),
        # The same for a whole sequence of the 12B model.
        dict(name="norm_12b", kind="norm", rows=TOKENS, cols=D_MODEL, x=BF16, stream=BF16, y=BF16, residual=True, gamma=True, out8=True, pad=0),
        # The norm's backward pass in a ragged layer with an FP32 residual stream that was kept as it is.
        dict(name="norm_bwd_ragged", kind="norm_bwd", rows=1040, cols=2064, x=BF16, stream=F32, saved8=False, gamma=True, dres=True, pad=0),
        # The same for a sequence of the 12B model, from the 8-bit checkpoint of the normalised rows.
        dict(name="norm_bwd_12b", kind="norm_bwd", rows=TOKENS, cols=D_MODEL, x=BF16, stream=BF16, saved8=True, gamma=True, dres=True, pad=0),
        # A small activation kept for the backward pass.
        dict(name="save_small", kind="save", rows=256, cols=512, x=BF16, pad=0),
        # The FFN's activation made again from its 8-bit checkpoint, for the weight gradient of the down-projection.
        dict(name="load_12b", kind="load", rows=TOKENS, cols=D_FFN, act="relu2", col_scale=False, x=BF16),
        # Gradient through the activation of a ragged layer, with the bias gradient.
        dict(name="act_bwd_ragged", kind="act_bwd", rows=1040, cols=1296, act="gelu", x=BF16, dbias=True, pad=0),
        # The same for the 12B FFN on a sequence: the largest that moves bytes only.
        dict(name="act_bwd_12b", kind="act_bwd", rows=TOKENS, cols=D_FFN, act="relu2", x=BF16, dbias=True, pad=0),
        # The small configuration's product with bias, activation and checkpoint: latency.
        dict(name="product_small", kind="product", m=256, n=256, k=512, fmt="nvfp4", bias=True, act="gelu", keep=True, grad=False, residual="", out=F32),
        # Inference of the down-projection with a handful of sequences in flight: the weight's bytes count.
        dict(name="product_few_tokens", kind="product", m=64, n=D_MODEL, k=D_FFN, fmt="nvfp4", bias=True, act="none", keep=False, grad=False, residual=BF16, out=BF16),
        # The 12B up-projection in training: bias, squared ReLU, checkpoint of what went into it.
        dict(name="product_12b", kind="product", m=TOKENS, n=D_FFN, k=D_MODEL, fmt="nvfp4", bias=True, act="relu2", keep=True, grad=False, residual="", out=BF16),
        # The gradient on its way back through the 12B down-projection and the activation, from the checkpoint: the largest.
        dict(name="product_grad_12b", kind="product", m=TOKENS, n=D_FFN, k=D_MODEL, fmt="nvfp4", bias=False, act="relu2", keep=False, grad=True, residual="", out=BF16),
    ]


def _size(rng, lo, hi, multiple):
    """Log-uniform in [lo, hi]; half of the sizes odd multiples of the unit, half round ones."""
    n = lo * (hi / lo) ** rng.random()
    step = multiple if rng.random() < 0.5 else max(multiple, 256 if n >= 1024 else 64 if n >= 128 else multiple)
    n = min(hi, max(lo, int(round(n / step)) * step))
    return n + multiple if n == 3072 else n     # (not a width of any layer here)


def draw(rng):
    kind = rng.choice(["norm", "norm", "norm_bwd", "norm_bwd", "save", "load", "act_bwd", "act_bwd", "product", "product", "product", "product"])
    x, stream = rng.choice([BF16, BF16, F32]), rng.choice([BF16, F32])
    pad = rng.choice([0, 0, 64])
    act = rng.choice(["relu2", "gelu", "silu"])
    if kind == "product":
        mx = rng.random() < 0.25
        while True:
            m, n = _size(rng, 16, TOKENS, 32 if mx else 16), _size(rng, 256, D_FFN, 32 if mx else 16)
            k = _size(rng, 256, D_FFN, 128 if mx else 16)
            if m * n * k <= TOKENS * D_FFN * D_MODEL:
                break
        case = dict(kind=kind, m=m, n=n, k=k, fmt="mxfp4" if mx else "nvfp4", out=rng.choice([BF16, F32]))
        if rng.random() < 0.25:
            return dict(case, bias=False, act=act, keep=False, grad=True, residual="")
        return dict(case, bias=rng.random() < 0.7, act=rng.choice(["none", act]), keep=rng.random() < 0.5, grad=False, residual=rng.choice(["", BF16, F32]))
    rows = _size(rng, 1, TOKENS, 1)
    if kind == "norm":
        return dict(kind=kind, rows=rows, cols=_size(rng, 256, D_FFN, 16), x=x, stream=stream, y=rng.choice([BF16, BF16, F32]), residual=rng.random() < 0.7,
                    gamma=rng.random() < 0.8, out8=rng.random() < 0.7, pad=pad)
    if kind == "norm_bwd":
        return dict(kind=kind, rows=rows, cols=_size(rng, 256, D_FFN, 16), x=x, stream=stream, saved8=rng.random() < 0.6, gamma=rng.random() < 0.8,
                    dres=rng.random() < 0.7, pad=pad)
    cols = _size(rng, 256, D_FFN, 16)
    if kind == "save":
        return dict(kind=kind, rows=rows, cols=cols, x=x, pad=pad)
    if kind == "load":
        return dict(kind=kind, rows=rows, cols=cols, act=rng.choice(["none", act]), col_scale=rng.random() < 0.5, x=x)
    return dict(kind=kind, rows=rows, cols=cols, act=act, x=x, dbias=rng.random() < 0.7, pad=pad)


# ---------------------------------------------------------------- 8 and 4 bits, plainly

def _encode8(v):
    """Codes (E4M3) and scales (powers of two) of a [rows, cols] tensor: the smallest power of two that brings a block's largest magnitude to at most 448."""
    blocks = v.reshape(v.shape[0], -1, BLOCK)
    m, e = torch.frexp(blocks.abs().amax(-1))                                    # amax = m 2^e, 0.5 <= m < 1; 448 = 0.875 * 2^9
    e = torch.where(m > 0, torch.where(m <= 0.875, e - 9, e - 8), torch.full_like(e, -127)).clamp(-127, 127)
    codes = (blocks * torch.exp2(-e.to(v.dtype))[..., None]).to(torch.float32).to(torch.float8_e4m3fn).reshape(v.shape)
    return codes, (e + 127).to(torch.uint8).view(torch.float8_e8m0fnu)


def _decode8(codes, scales, dtype):
    return (codes.to(dtype).reshape(codes.shape[0], -1, BLOCK) * scales.to(dtype)[..., None]).reshape(codes.shape)


_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _encode4(v, fmt, tile):
    """A K-contiguous operand [outer, K] in 4 bits: packed codes, scale bytes, tensor scale.  tile: rows that share a block scale (a weight's 16)."""
    outer, k = v.shape
    block = 32 if fmt == "mxfp4" else 16
    amax_t = v.abs().amax()
    s_enc = torch.ones_like(amax_t) if fmt == "mxfp4" else 2688.0 / amax_t
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=v.device)
    codes = torch.empty(outer, k // 2, dtype=torch.uint8, device=v.device)
    scales = torch.empty(outer, k // block, dtype=torch.uint8, device=v.device)
    for r in range(0, outer, 1024):
        part = v[r:r + 1024]
        amax = part.abs().reshape(-1, tile, k // block, block).amax((1, 3))
        if fmt == "mxfp4":
            e = torch.ceil(torch.log2((amax / 6.0).clamp_min(2.0 ** -126)))
            stored, factor = (e + 127).to(torch.uint8), torch.exp2(e)
        else:
            s8 = (amax / 6.0 * s_enc).clamp_max(448.0).to(torch.float8_e4m3fn)
            stored, factor = s8.view(torch.uint8), s8.float() / s_enc
        stored, factor = (t.repeat_interleave(tile, 0) for t in (stored, factor))
        q = (part.reshape(-1, k // block, block) / factor.clamp_min(1e-30)[..., None]).reshape(part.shape)
        c = torch.bucketize(q.abs(), edges).to(torch.uint8) | ((q < 0).to(torch.uint8) << 3)
        codes[r:r + 1024] = c[:, 0::2] | (c[:, 1::2] << 4)
        scales[r:r + 1024] = stored
    ts = torch.stack([1.0 / s_enc, amax_t if fmt != "mxfp4" else torch.zeros_like(amax_t)]).float()
    return codes, scales, ts


def _decode4(codes, scales, ts, fmt, dtype):
    values = torch.tensor(_E2M1 + [-x for x in _E2M1], dtype=dtype, device=codes.device)
    v = torch.stack([values[(codes & 15).int()], values[(codes >> 4).int()]], -1).reshape(codes.shape[0], -1)
    s = torch.exp2(scales.to(dtype) - 127) if fmt == "mxfp4" else scales.view(torch.float8_e4m3fn).to(dtype)
    return (v.reshape(v.shape[0], s.shape[1], -1) * s[..., None]).reshape(v.shape) * ts[0].to(dtype)


# ---------------------------------------------------------------- inputs

class _Inputs:
    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)

    def normal(self, *shape):
        return torch.randn(*shape, generator=self.g, device="cuda")

    def activation(self, rows, cols):
        v = self.normal(rows, cols)
        return torch.where(torch.rand(rows, cols, generator=self.g, device="cuda") < 1e-3, v * 50.0, v)

    def gradient(self, rows, cols):
        z = self.normal(rows, cols)
        chi = self.normal(rows, cols).square() + self.normal(rows, cols).square() + self.normal(rows, cols).square()
        return 1e-3 * z / (chi / 3.0).clamp_min(1e-6).sqrt()


def _placed(v, dtype, pad):
    """The tensor in its type, its rows `pad` elements further apart than they are long."""
    rows, cols = v.shape
    out = torch.zeros(rows, cols + pad, dtype=DTYPE[dtype], device=v.device)[:, :cols]
    out.copy_(v)
    return out


def prepare(case, seed):
    gen, kind = _Inputs(seed), case["kind"]
    s = dict(case=case)
    if kind == "product":
        m, n, k, fmt = case["m"], case["n"], case["k"], case["fmt"]
        left = gen.gradient(m, k) if case["grad"] else gen.activation(m, k)
        s["a"] = _encode4(left.bfloat16().float(), fmt, 1)
        s["b"] = _encode4((0.02 * gen.normal(n, k)).bfloat16().float(), fmt, 1 if fmt == "mxfp4" else 16)
        s["bias"] = 0.02 * gen.normal(n) if case["bias"] else None
        s["residual"] = _placed(gen.activation(m, n), case["residual"], 0) if case["residual"] else None
        s["saved"] = _encode8(gen.activation(m, n)) if case["grad"] else None
        if own:   # the handles and the scratch memory that a program keeps for its layers
            _handles(s)
        return s
    rows, cols = case["rows"], case["cols"]
    if kind == "norm":
        s["x"] = _placed(gen.activation(rows, cols), case["x"], case["pad"])
        s["residual"] = _placed(gen.activation(rows, cols), case["stream"], case["pad"]) if case["residual"] else None
        s["gamma"] = 1.0 + 0.1 * gen.normal(cols) if case["gamma"] else None
    elif kind == "norm_bwd":
        h = _placed(gen.activation(rows, cols), case["stream"], case["pad"])
        s["rstd"] = torch.rsqrt(h.float().square().mean(1) + EPS)
        s["saved"] = _encode8(h.float() * s["rstd"][:, None]) if case["saved8"] else h
        s["dy"] = _placed(gen.gradient(rows, cols), case["x"], case["pad"])
        s["dres"] = _placed(gen.gradient(rows, cols), case["stream"], case["pad"]) if case["dres"] else None
        s["gamma"] = 1.0 + 0.1 * gen.normal(cols) if case["gamma"] else None
    elif kind == "save":
        s["x"] = _placed(gen.activation(rows, cols), case["x"], case["pad"])
    else:
        s["saved"] = _encode8(gen.activation(rows, cols))
        if kind == "load":
            s["col_scale"] = 1.0 + 0.1 * gen.normal(cols) if case["col_scale"] else None
        else:
            s["da"] = _placed(gen.gradient(rows, cols), case["x"], case["pad"])
    if own and isinstance(s.get("saved"), tuple):
        _handles(s)
    return s


def _handles(s):
    """The framework's descriptors over the very tensors that prepare() made."""
    from paper_2509_25149_amd import binding as nv
    case = s["case"]
    if isinstance(s.get("saved"), tuple):
        codes, scales = s["saved"]
        s["saved8"] = nv.Checkpoint8(codes.view(torch.uint8), scales.view(torch.uint8))
    if case["kind"] == "product":
        def operand(packed, outer):
            q = nv.QTensor(nv.QTensorStruct(), outer, case["k"])
            q.row_codes, q.row_scales, q.row_ts = packed
            q.desc.rows, q.desc.cols, q.desc.layout_mask = outer, case["k"], nv.LAYOUT_ROW
            q.desc.block_dim = nv.BLOCK_MX32 if case["fmt"] == "mxfp4" else nv.BLOCK_1x16
            q.desc.row_codes, q.desc.row_scales, q.desc.row_tensor_scale = (t.data_ptr() for t in packed)
            return q
        s["qa"], s["qb"] = operand(s["a"], case["m"]), operand(s["b"], case["n"])
        s["workspace"] = torch.empty(nv.gemm_workspace_bytes(case["m"], case["n"], case["k"]), dtype=torch.uint8, device="cuda")


# ---------------------------------------------------------------- one pass, plainly

_C1, _C3 = 1.5957691216057308, 0.07135481282988394     # GELU in its tanh form: z times the logistic function of c1 z + c3 z^3


def _act(z, act):
    if act == "relu2":
        return z.clamp_min(0).square()
    if act == "silu":
        return z * torch.sigmoid(z)
    if act == "gelu":
        return z * torch.sigmoid(z * (_C1 + _C3 * z * z))
    return z


def _act_grad(z, act):
    if act == "relu2":
        return 2 * z.clamp_min(0)
    if act == "silu":
        g = torch.sigmoid(z)
        return g + z * g * (1 - g)
    if act == "gelu":
        g = torch.sigmoid(z * (_C1 + _C3 * z * z))
        return g + z * g * (1 - g) * (_C1 + 3 * _C3 * z * z)
    return torch.ones_like(z)


def _named(**outputs):
    return {k: v for k, v in outputs.items() if v is not None}


def _plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "norm":
        h = s["x"].float()
        if s["residual"] is not None:
            h = h + s["residual"].float()
        rstd = torch.rsqrt(h.square().mean(1) + EPS)
        xhat = h * rstd[:, None]
        y = xhat if s["gamma"] is None else xhat * s["gamma"]
        codes, scales = _encode8(xhat) if case["out8"] else (None, None)
        return _named(y=y.to(DTYPE[case["y"]]), h=h.to(DTYPE[case["stream"]]) if s["residual"] is not None else None, rstd=rstd, codes=codes, scales=scales)
    if kind == "norm_bwd":
        rstd = s["rstd"][:, None]
        xhat = _decode8(*s["saved"], torch.float32) if case["saved8"] else s["saved"].float() * rstd
        dy = s["dy"].float()
        g = dy if s["gamma"] is None else dy * s["gamma"]
        dx = rstd * (g - xhat * (g * xhat).mean(1, keepdim=True))
        if s["dres"] is not None:
            dx = dx + s["dres"].float()
        return _named(dx=dx.to(DTYPE[case["stream"]]), dgamma=(dy * xhat).sum(0))
    if kind == "save":
        codes, scales = _encode8(s["x"].float())
        return _named(codes=codes, scales=scales)
    if kind == "load":
        v = _act(_decode8(*s["saved"], torch.float32), case["act"])
        return _named(out=(v if s["col_scale"] is None else v * s["col_scale"]).to(DTYPE[case["x"]]))
    if kind == "act_bwd":
        dz = s["da"].float() * _act_grad(_decode8(*s["saved"], torch.float32), case["act"])
        return _named(dz=dz.to(DTYPE[case["x"]]), dbias=dz.sum(0) if case["dbias"] else None)
    z = torch.matmul(_decode4(*s["a"], case["fmt"], torch.float32), _decode4(*s["b"], case["fmt"], torch.float32).t())
    if case["grad"]:
        return _named(out=(z * _act_grad(_decode8(*s["saved"], torch.float32), case["act"])).to(DTYPE[case["out"]]))
    if s["bias"] is not None:
        z = z + s["bias"]
    codes, scales = _encode8(z) if case["keep"] else (None, None)
    d = _act(z, case["act"])
    if s["residual"] is not None:
        d = d + s["residual"].float()
    return _named(out=d.to(DTYPE[case["out"]]), codes=codes, scales=scales)


# ---------------------------------------------------------------- one pass, through the framework

def _bytes8(ckpt):
    return (ckpt.codes.view(torch.float8_e4m3fn), ckpt.scales.view(torch.float8_e8m0fnu)) if ckpt is not None else (None, None)


def run(state):
    if not own:
        return _plain(state)
    from paper_2509_25149_amd import binding as nv
    case, kind = state["case"], state["case"]["kind"]
    out_type = {F32: nv.OUT_F32, BF16: nv.OUT_BF16}
    act = {"none": nv.ACT_NONE, "relu2": nv.ACT_RELU2, "gelu": nv.ACT_GELU, "silu": nv.ACT_SILU}
    if kind == "norm":
        h_type = out_type[case["stream"]]
        r = nv.nvfp4_rmsnorm_forward(state["x"], state["gamma"], residual=state["residual"], eps=EPS, y_dtype=out_type[case["y"]], h_dtype=h_type,
                                     checkpoint=case["out8"])
        codes, scales = _bytes8(r.checkpoint)
        return _named(y=r.y, h=r.h if state["residual"] is not None else None, rstd=r.rstd, codes=codes, scales=scales)
    if kind == "norm_bwd":
        dx, dgamma = nv.nvfp4_rmsnorm_backward(state["dy"], state["saved8"] if case["saved8"] else state["saved"], state["rstd"], state["gamma"],
                                               dres=state["dres"], dx_dtype=out_type[case["stream"]])
        return _named(dx=dx, dgamma=dgamma)
    if kind == "save":
        codes, scales = _bytes8(nv.nvfp4_checkpoint_save(state["x"]))
        return _named(codes=codes, scales=scales)
    if kind == "load":
        return _named(out=nv.nvfp4_checkpoint_load(state["saved8"], act[case["act"]], col_scale=state["col_scale"], out_dtype=out_type[case["x"]]))
    if kind == "act_bwd":
        dz, dbias = nv.nvfp4_activation_backward(state["da"], state["saved8"], act[case["act"]], bias_grad=case["dbias"])
        return _named(dz=dz, dbias=dbias)
    keep = nv.alloc_checkpoint(case["m"], case["n"]) if case["keep"] else None
    d = nv.nvfp4_gemm_epilogue(state["qa"], state["qb"], nv.OP_DGRAD, bias=state["bias"], activation=act[case["act"]], residual=state["residual"], keep=keep,
                               grad_of=state["saved8"] if case["grad"] else None, out_dtype=out_type[case["out"]], workspace=state["workspace"])
    codes, scales = _bytes8(keep)
    return _named(out=d, codes=codes, scales=scales)


# ---------------------------------------------------------------- 64 bits

def _exact8(v):
    """Codes and scales of binary64 values, as numbers: the definition by comparison of magnitudes."""
    blocks = v.reshape(v.shape[0], -1, BLOCK)
    amax = blocks.abs().amax(-1)
    e = torch.ceil(torch.log2(amax.clamp_min(2.0 ** -118) / 448.0))
    e = torch.where(448.0 * torch.exp2(e - 1) >= amax, e - 1, torch.where(448.0 * torch.exp2(e) < amax, e + 1, e)).clamp(-127, 127)
    e = torch.where(amax == 0, torch.full_like(e, -127.0), e)
    a = (blocks / torch.exp2(e)[..., None]).abs()
    step = torch.exp2(torch.floor(torch.log2(a.clamp_min(2.0 ** -6))) - 3)      # three bits behind the leading one; below 2^-6 the step stays
    q = torch.round(a / step) * step                                             # ties to even
    return torch.copysign(q, blocks).reshape(v.shape), torch.exp2(e)


def _exact_act(z, act):
    if act == "relu2":
        return torch.where(z > 0, z * z, torch.zeros_like(z))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.tanh((2 / torch.pi) ** 0.5 * (z + 0.044715 * z ** 3)))
    return z


def _exact_act_grad(z, act):
    if act == "relu2":
        return torch.where(z > 0, 2 * z, torch.zeros_like(z))
    if act == "silu":
        e = torch.exp(-z.abs())                                                  # g' = e / (1 + e)^2 either side of zero
        return 1 / (1 + torch.exp(-z)) + z * e / (1 + e) ** 2
    if act == "gelu":
        t = torch.tanh((2 / torch.pi) ** 0.5 * (z + 0.044715 * z ** 3))
        return 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * (2 / torch.pi) ** 0.5 * (1 + 3 * 0.044715 * z * z)
    return torch.ones_like(z)


def exact(case, seed):
    s, kind, f64 = prepare(case, seed), case["kind"], torch.float64
    if kind == "product":
        a, b = (_decode4(*s[name], case["fmt"], f64) for name in ("a", "b"))
        z = torch.cat([a[r:r + 1024] @ b.t() for r in range(0, a.shape[0], 1024)])
        if case["grad"]:
            return _named(out=z * _exact_act_grad(_decode8(*s["saved"], f64), case["act"]))
        if s["bias"] is not None:
            z += s["bias"].to(f64)
        codes, scales = _exact8(z) if case["keep"] else (None, None)
        d = _exact_act(z, case["act"])
        return _named(out=d if s["residual"] is None else d + s["residual"].to(f64), codes=codes, scales=scales)
    if kind == "norm":
        h = s["x"].to(f64) + (s["residual"].to(f64) if s["residual"] is not None else 0.0)
        rstd = 1 / torch.sqrt((h * h).sum(1) / h.shape[1] + EPS)
        xhat = h * rstd[:, None]
        codes, scales = _exact8(xhat) if case["out8"] else (None, None)
        return _named(y=xhat * s["gamma"].to(f64) if s["gamma"] is not None else xhat, h=h if s["residual"] is not None else None, rstd=rstd, codes=codes,
                      scales=scales)
    if kind == "norm_bwd":
        rstd, dy = s["rstd"].to(f64)[:, None], s["dy"].to(f64)
        xhat = _decode8(*s["saved"], f64) if case["saved8"] else s["saved"].to(f64) * rstd
        g = dy * s["gamma"].to(f64) if s["gamma"] is not None else dy
        dx = rstd * g - rstd * xhat * ((g * xhat).sum(1, keepdim=True) / g.shape[1])
        return _named(dx=dx + s["dres"].to(f64) if s["dres"] is not None else dx, dgamma=(dy * xhat).sum(0))
    if kind == "save":
        codes, scales = _exact8(s["x"].to(f64))
        return _named(codes=codes, scales=scales)
    z = _decode8(*s["saved"], f64)
    if kind == "load":
        v = _exact_act(z, case["act"])
        return _named(out=v * s["col_scale"].to(f64) if s["col_scale"] is not None else v)
    dz = s["da"].to(f64) * _exact_act_grad(z, case["act"])
    return _named(dz=dz, dbias=dz.sum(0) if case["dbias"] else None)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    size, eight = {F32: 4, BF16: 2}, 1 + 1 / BLOCK
    kind = case["kind"]
    if kind == "product":
        m, n, k = case["m"], case["n"], case["k"]
        operand = 0.5 + (1 / 32 if case["fmt"] == "mxfp4" else 1 / 16)
        per = size[case["out"]] + (eight if case["keep"] else 0) + (eight if case["grad"] else 0) + (size[case["residual"]] if case["residual"] else 0)
        return dict(bytes=(m + n) * k * operand + m * n * per + (4 * n if case["bias"] else 0), flops=2 * m * n * k)
    rows, cols = case["rows"], case["cols"]
    if kind == "norm":
        per = size[case["x"]] + size[case["y"]] + (2 * size[case["stream"]] if case["residual"] else 0) + (eight if case["out8"] else 0)
        return dict(bytes=rows * cols * per + 4 * rows + 4 * cols, flops=6 * rows * cols)
    if kind == "norm_bwd":
        per = size[case["x"]] + size[case["stream"]] + (eight if case["saved8"] else size[case["stream"]]) + (size[case["stream"]] if case["dres"] else 0)
        return dict(bytes=rows * cols * per + 4 * rows + 8 * cols, flops=9 * rows * cols)
    if kind == "act_bwd":
        return dict(bytes=rows * cols * (2 * size[case["x"]] + eight) + (4 * cols if case["dbias"] else 0), flops=4 * rows * cols)
    return dict(bytes=rows * cols * (size[case["x"]] + eight), flops=3 * rows * cols)
