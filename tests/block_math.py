"""What surrounds the linear layers, in binary64 numpy straight from the formulas: 8-bit checkpoints, activations, norm.  Used by the tests only."""
import numpy as np
import torch

ACTS = {"none": 0, "relu2": 1, "gelu": 2, "silu": 3}
E4M3 = np.array([(c & 7) * 2.0 ** -9 if c >> 3 == 0 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)])   # code -> value; 126 is 448


def encode(v):
    """(codes, scale bytes) of a finite [rows, cols] array."""
    v = np.asarray(v, np.float64)
    blocks = v.reshape(v.shape[0], -1, 16)
    amax = np.abs(blocks).max(-1)
    e = np.full(amax.shape, -127)
    for k in range(-127, 128):                                # the smallest e that covers the block, by trying all
        e = np.where((amax > 448.0 * 2.0 ** (k - 1)) & (k > -127), k, e)
    a = np.abs(blocks) / np.exp2(e.astype(np.float64))[..., None]
    hi = np.clip(np.searchsorted(E4M3, a), 1, 126)            # nearest of two neighbours, the even code at a tie
    lo = hi - 1
    dl, dh = a - E4M3[lo], E4M3[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    code = code | (np.signbit(blocks).astype(np.int64) << 7)
    return code.reshape(v.shape).astype(np.uint8), (e + 127).astype(np.uint8)


def decode(codes, scales):
    codes, scales = np.asarray(codes), np.asarray(scales)
    table = np.concatenate([E4M3, [np.nan], -E4M3, [np.nan]])
    s = np.where(scales == 255, np.nan, np.exp2(scales.astype(np.float64) - 127))
    return (table[codes].reshape(codes.shape[0], -1, 16) * s[..., None]).reshape(codes.shape)


def logistic_argument(z, name):
    return z if name == "silu" else 2 * np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3)


def act(z, name):
    if name == "relu2":
        return np.where(z > 0, z * z, 0.0)
    if name == "none":
        return z
    with np.errstate(over="ignore"):
        return z / (1 + np.exp(-logistic_argument(z, name)))     # (1 + tanh(u)) / 2 = 1 / (1 + exp(-2 u)), without the cancellation far below 0


def slope(z, name):
    if name == "relu2":
        return np.where(z > 0, 2 * z, 0.0)
    if name == "none":
        return np.ones_like(z)
    p = logistic_argument(z, name)
    dp = np.ones_like(z) if name == "silu" else 2 * np.sqrt(2 / np.pi) * (1 + 3 * 0.044715 * z * z)
    with np.errstate(over="ignore"):
        s = 1 / (1 + np.exp(-p))
        return s + z * s * (1 / (1 + np.exp(p))) * dp


def act_tolerance(z, name):
    """How far an FP32 evaluation of act may be from the true value: the logistic function takes exp2 and a reciprocal of an ulp each, and the
    rounding of its argument p (three operations and the change of base) moves exp(p) by |p| of those."""
    if name in ("none", "relu2"):
        return 2.0 ** -23 * np.abs(act(z, name))
    return 2.0 ** -22 * (4 + np.abs(logistic_argument(z, name))) * np.abs(act(z, name)) + 1e-37


def slope_tolerance(z, name):
    if name in ("none", "relu2"):
        return 2.0 ** -23 * np.abs(slope(z, name))
    p = logistic_argument(z, name)
    dp = np.ones_like(z) if name == "silu" else 2 * np.sqrt(2 / np.pi) * (1 + 3 * 0.044715 * z * z)
    with np.errstate(over="ignore"):
        s, t = 1 / (1 + np.exp(-p)), 1 / ((1 + np.exp(-p)) * (1 + np.exp(p)))
    return 2.0 ** -22 * (4 + 2 * np.abs(p)) * (s + np.abs(z) * t * dp) + 1e-37


def rounding(ref, dtype):
    """Half a unit in the last place of the output's type (8 or 24 significant bits), relative, with room for the FP32 value being rounded a little off."""
    return (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -24) * np.abs(ref) * 1.01 + 1e-37


def norm(x, residual, gamma, eps):
    h = x if residual is None else x + residual
    rstd = 1 / np.sqrt((h * h).mean(1) + eps)
    xhat = h * rstd[:, None]
    return h, rstd, xhat, xhat if gamma is None else xhat * gamma


def norm_backward(dy, xhat, rstd, gamma, dres):
    g = dy if gamma is None else dy * gamma
    dx = rstd[:, None] * (g - xhat * (g * xhat).mean(1, keepdims=True))
    return dx if dres is None else dx + dres, (dy * xhat).sum(0)


def f64(t):
    return t.detach().cpu().double().numpy()


def tensor(v, dtype, pad=0):
    """On the GPU, rows `pad` elements further apart than they are long; what lies between is NaN."""
    v = torch.as_tensor(np.asarray(v, np.float32))
    wide = torch.full((v.shape[0], v.shape[1] + pad), float("nan"), dtype=dtype, device="cuda")
    wide[:, :v.shape[1]] = v.to("cuda", dtype)
    return wide[:, :v.shape[1]]


def within(got, ref, tol):
    got = f64(got) if isinstance(got, torch.Tensor) else got
    off = np.abs(got - ref) - tol
    worst = np.unravel_index(np.argmax(off), off.shape) if off.size else None
    assert off.size == 0 or off[worst] <= 0, (worst, got[worst], ref[worst], tol[worst])
