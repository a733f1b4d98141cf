"""The ends of a training step in binary64 numpy straight from the formulas, and how far FP32 may be from them.  Used by the tests only."""
import numpy as np
import torch

U = 2.0 ** -24      # half a unit in the last place of FP32, relative


def logits_statistics(z, scale):
    """(largest, ln sum exp(scale (z - largest)), p, ln p, entropy) of each row; a row without a value above -infinity has p = 0, ln p = -infinity, entropy 0."""
    z = np.asarray(z, np.float64)
    m = z.max(1)
    empty = np.isneginf(m)
    base = np.where(empty, 0.0, m)
    with np.errstate(over="ignore", divide="ignore", invalid="ignore"):
        d = scale * (z - base[:, None])
        e = np.exp(d)
        s = e.sum(1)
        logsum = np.where(empty, np.inf, np.log(s))
        logp = d - logsum[:, None]
        p = np.exp(logp)
        entropy = -np.where(p > 0, p * logp, 0.0).sum(1)
    return base, logsum, p, logp, np.where(empty, 0.0, entropy)


def sum_error(z, scale):
    """Relative error of a row's sum of exponentials: an exponent's three roundings (difference, factor, product) move a term by 4 |D| u, D = scale (z - max), and its rescalings, whose
    exponents add up to less than |D|, by as much again; exp2 is good to 2 u; a term goes through at most 160 additions and factors (chains of 8, turns over the row, a tree)."""
    m, logsum, p, logp, _ = logits_statistics(z, scale)
    with np.errstate(invalid="ignore"):
        mean = np.where(p > 0, p * np.abs(logp + logsum[:, None]), 0.0).sum(1)
        square = np.where(p > 0, p * (logp + logsum[:, None]) ** 2, 0.0).sum(1)
    return (8 * mean + 160) * U, mean, square


def entropy_error(z, scale):
    rel, mean, square = sum_error(z, scale)
    logsum = logits_statistics(z, scale)[1]
    return 8 * U * (square + mean) + 2 * rel * mean + rel + 4 * U * (np.abs(logsum) + mean)


def logits_gradient(z, scale, targets, g, g_lse, g_entropy):
    """(dlogits, tolerance before the output is rounded), the statistics handed on from an FP32 forward pass included."""
    m, logsum, p, logp, entropy = logits_statistics(z, scale)
    rows, cols = p.shape
    zero = np.zeros(rows)
    counted = (targets >= 0) & (targets < cols) if targets is not None else np.zeros(rows, bool)
    g = np.where(counted & np.isfinite(logsum), g if g is not None else zero, 0.0)
    gl, gh = (zero if v is None else v for v in (g_lse, g_entropy))
    with np.errstate(invalid="ignore"):
        ph = np.where(p > 0, p * (logp + entropy[:, None]), 0.0)
        dz = p * (gl - g)[:, None] - gh[:, None] * ph
        rel = np.where(p > 0, 8 * U * np.abs(logp) + sum_error(z, scale)[0][:, None] + 4 * U * (2 + np.abs(logsum))[:, None], 0.0)
        size = p * (np.abs(gl) + np.abs(g))[:, None] + np.abs(gh)[:, None] * np.where(p > 0, p * (np.abs(logp) + entropy[:, None]), 0.0)
        tol = scale * (size * (rel + 8 * U) + np.abs(gh)[:, None] * p * (entropy_error(z, scale) if g_entropy is not None else zero)[:, None]
                       + np.abs(gh)[:, None] * np.where(p > 0, p * rel * np.maximum(1, np.abs(logp)), 0.0))
    if targets is not None:
        at = np.clip(targets, 0, cols - 1)
        dz[np.arange(rows), at] += g
        tol[np.arange(rows), at] += 4 * U * scale * np.abs(g)
    return scale * dz, np.nan_to_num(tol, nan=0.0) + 1e-37


def best(z, top):
    """Columns of the largest, the lowest columns first among equal ones; a NaN is below -infinity."""
    key = np.where(np.isnan(z), -np.inf, np.asarray(z, np.float64))
    order = np.lexsort((np.arange(z.shape[1])[None].repeat(z.shape[0], 0), np.isnan(z), -key), axis=1)
    return order[:, :top]


def embedding_gradient(dout, ids, vocab, scale):
    """(dtable, tolerance): a row of n tokens is a sum of n terms in some fixed order, times the scale."""
    ids = np.asarray(ids)
    there = (ids >= 0) & (ids < vocab)
    sums, size, count = np.zeros((vocab, dout.shape[1])), np.zeros((vocab, dout.shape[1])), np.zeros(vocab)
    np.add.at(sums, ids[there], dout[there])
    np.add.at(size, ids[there], np.abs(dout[there]))
    np.add.at(count, ids[there], 1)
    return scale * sums, (count + 2)[:, None] * U * abs(scale) * size + 1e-37


def index(values, dtype):
    return torch.as_tensor(np.asarray(values)).to("cuda", dtype)
