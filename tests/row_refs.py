"""The row operators (layer norm, bias + GELU, distillation) in numpy, in 64 bits and from their formulas, and how far an fp32
computation of each may be off.

Bounds.  u = 2^-24 is the rounding of fp32.  A sum of n terms that at least 64 lanes share out is off by at most depth(n) u times the
sum of the absolute terms, depth(n) = n / 64 + 16 (a lane's own chain, then the tree); a sum over rows by rows / 8 + 64 at most, or n
where that is less (any order).  Functions (exp, log, erf, tanh, square root, division) are taken as good to 4 u of their value, and
what their arguments are off by is passed on by the derivative.  A result of type bf16 (8 significant bits) is off by 2^-8 of its value
more, its one rounding."""
from __future__ import annotations

import math

import numpy as np

U = 2.0 ** -24


def depth(n):
    return n / 64 + 16


def row_depth(n):
    return min(n, n / 8 + 64)


def stored(value, bound, bf16):
    """The bound of a result after it has been rounded to its type (and what denormal results lose)."""
    return (bound * 1.01 + (2.0 ** -8 if bf16 else U) * np.abs(value)) + (2.0 ** -133 if bf16 else 2.0 ** -149)


def _or(v, other):
    return np.float64(other) if v is None else v.astype(np.float64)


def layer_norm(x, residual=None, weight=None, bias=None, eps=1e-5):
    """{name: (value, bound)}"""
    n = x.shape[1]
    x = x.astype(np.float64)
    t = x if residual is None else x + residual.astype(np.float64)
    mean = t.mean(1, keepdims=True)
    d = t - mean
    var = (d * d).mean(1, keepdims=True)
    rstd = 1 / np.sqrt(var + eps)
    w, b = _or(weight, 1.0), _or(bias, 0.0)
    xh = d * rstd
    y = xh * w + b
    off_t = U * np.abs(t)
    off_mean = (depth(n) + 2) * U * np.abs(t).mean(1, keepdims=True)
    off_d = off_t + off_mean + U * np.abs(d)
    off_var = (2 * np.abs(d) * off_d + off_d ** 2).mean(1, keepdims=True) + (depth(n) + 4) * U * var
    rel_rstd = 0.5 * off_var * rstd ** 2 + 6 * U
    off_y = np.abs(w) * (off_d * rstd + np.abs(xh) * rel_rstd) * 1.01 + 4 * U * (np.abs(xh * w) + np.abs(b))
    return {"y": (y, off_y), "total": (t, off_t), "mean": (mean[:, 0], off_mean[:, 0]), "rstd": (rstd[:, 0], (rel_rstd * rstd * 1.01)[:, 0])}


def layer_norm_backward(dy, x, mean, rstd, weight=None, dtotal=None):
    rows, n = x.shape
    dy, x, mean, rstd = (a.astype(np.float64) for a in (dy, x, mean[:, None], rstd[:, None]))
    w, more = _or(weight, 1.0), _or(dtotal, 0.0)
    h = (x - mean) * rstd
    d = dy * w
    m1, m2 = d.mean(1, keepdims=True), (d * h).mean(1, keepdims=True)
    dx = rstd * (d - m1 - h * m2) + more
    off_h = 3 * U * np.abs(h)                                    # the difference of two given numbers is one rounding off
    off_d = U * np.abs(d)
    off_m1 = off_d.mean(1, keepdims=True) + (depth(n) + 2) * U * np.abs(d).mean(1, keepdims=True)
    off_m2 = (depth(n) + 8) * U * np.abs(d * h).mean(1, keepdims=True)
    off_dx = rstd * (off_d + off_m1 + np.abs(h) * off_m2 + np.abs(m2) * off_h + 6 * U * (np.abs(d) + np.abs(m1) + np.abs(h * m2))) + 2 * U * (np.abs(dx) + np.abs(more))
    dw, db = dy * h, dy
    return {"dx": (dx, off_dx), "dweight": (dw.sum(0), ((row_depth(rows) + 6) * U * np.abs(dw)).sum(0)),
            "dbias": (db.sum(0), (row_depth(rows) * U * np.abs(db)).sum(0))}


_erf = np.vectorize(math.erf, otypes=[np.float64])
_erfc = np.vectorize(math.erfc, otypes=[np.float64])


def _gelu(x, bias, tanh):
    """u, the share of it that passes, and the derivative of y"""
    u = x.astype(np.float64) + _or(bias, 0.0)
    if tanh:
        c = math.sqrt(2 / math.pi)
        inner = c * (u + 0.044715 * u ** 3)
        th = np.tanh(inner)
        share = 1 / (1 + np.exp(np.minimum(-2 * inner, 700.0)))
        return u, share, share + u * 0.5 * (1 - th * th) * c * (1 + 3 * 0.044715 * u ** 2)
    share = 0.5 * _erfc(-u / math.sqrt(2))
    return u, share, share + u * np.exp(-0.5 * u * u) / math.sqrt(2 * math.pi)


# The share is taken as good to 8 u of 1 (it is not held to its own size where it vanishes), the derivative to as much of each of its
# two terms, the second of which has a factor u; an argument that is off by u |u| moves them by at most as much again.
def bias_gelu(x, bias=None, tanh=False):
    u, share, _ = _gelu(x, bias, tanh)
    return {"y": (u * share, 12 * U * np.abs(u))}


def bias_gelu_backward(dy, x, bias=None, tanh=False):
    u, _, slope = _gelu(x, bias, tanh)
    dy = dy.astype(np.float64)
    dx = dy * slope
    off = np.abs(dy) * 16 * U * (1 + np.minimum(np.abs(u), 20.0))
    rows = x.shape[0]
    return {"dx": (dx, off), "dbias": (dx.sum(0), off.sum(0) + (row_depth(rows) * U * np.abs(dx)).sum(0))}


def distill(logits, teacher, index, T, row_weight=None, grad=True):
    """Row by row.  Rows for which the formula has no finite value are left NaN or Inf, as the formula gives them."""
    rows, vocab = logits.shape
    out = {k: (np.zeros(rows), np.zeros(rows)) for k in ("loss", "row_max", "row_sum")}
    out["dlogits"] = (np.zeros((rows, vocab)), np.zeros((rows, vocab)))
    T = float(np.float32(T))
    for r in range(rows):
        z = logits[r].astype(np.float64)
        have = (index[r] >= 0) & (index[r] < vocab) & ~(teacher[r] == -np.inf)
        at, t = index[r][have].astype(np.int64), teacher[r][have].astype(np.float64)
        w = 1.0 if row_weight is None else float(row_weight[r])
        with np.errstate(all="ignore"):
            m = np.fmax.reduce(z)
            a = (z - m) / T
            e = np.exp(a)
            s = e.sum()
            reach = np.where(e > 0, np.abs(a) * e, 0.0).sum() / s           # how far the arguments' roundings move the sum
            rel_s = U * (depth(vocab) + 8 + 3 * reach)
            out["row_max"][0][r], out["row_sum"][0][r], out["row_sum"][1][r] = m, s, rel_s * s
            if not len(at):
                continue
            b = (t - t.max()) / T
            ps = np.exp(b).sum()
            log_p, log_q = b - np.log(ps), a[at] - np.log(s)
            p = np.exp(log_p)
            rel_p = U * (3 * np.abs(b) + depth(len(at)) + 16 + 3 * (np.exp(b) * np.abs(b)).sum() / ps)
            off_log = U * (3 * np.abs(b) + 3 * np.abs(a[at]) + 8 + 4 * np.abs(log_p) + 4 * np.abs(log_q)) + rel_s + rel_p
            term = np.where(np.isneginf(log_q), np.inf, p * (log_p - log_q))
            out["loss"][0][r] = T * T * term.sum()
            out["loss"][1][r] = T * T * ((rel_p * np.abs(term) + p * off_log).sum() + (depth(len(at)) + 4) * U * np.abs(term).sum())
            if not grad or w == 0:
                continue
            q = e / s
            share = np.bincount(at, weights=p, minlength=vocab)
            off = q * (rel_s + U * (3 * np.where(e > 0, np.abs(a), 0.0) + 16)) + np.bincount(at, weights=p * rel_p, minlength=vocab) + (depth(len(at)) + 4) * U * share
            out["dlogits"][0][r] = w * T * (q - share)
            # what is below the least normal number of fp32 may be lost on the way
            out["dlogits"][1][r] = abs(w) * T * (off + 2.0 ** -126) + 4 * U * np.abs(out["dlogits"][0][r])
    return out
