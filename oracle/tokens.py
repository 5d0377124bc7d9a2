"""64-bit oracle of the token operators (embedding, vocabulary loss, distillation from top logits), in numpy, from the formulas.

Shares no code with the library.  Next to the values stand error bounds (names with _err) for fp32 arithmetic on operands as they are
stored: a sum of n products is off by at most n roundings of 2^-24 of the sum of their magnitudes, an exponential by its argument's error."""
from __future__ import annotations

import numpy as np

EPS32 = 2.0 ** -24
# fp32 numbers end at 2^-126 (the matrix cores and exp2 know none below): a probability, a term of one, or a product may be off by this much, whatever its size.
# exp(-90) = 2^-129.8 for one is 0 in fp32, which no number of roundings allows for.
LEAST = 2.0 ** -126


def embed(tokens, weight, scale=1.0):
    """y [n, d] for tokens [n]; 0 where a token is outside the table."""
    t, w = np.asarray(tokens, np.int64), np.asarray(weight, np.float64)
    live = (t >= 0) & (t < w.shape[0])
    return np.where(live[:, None], w[np.where(live, t, 0)] * scale, 0.0)


def embed_backward(tokens, dy, vocab, scale=1.0, before=None):
    """(dweight, bound).  before: what the sums are added to, for tokens that occur."""
    t, dy = np.asarray(tokens, np.int64), np.asarray(dy, np.float64)
    dw, size, count = np.zeros((vocab, dy.shape[1])), np.zeros((vocab, dy.shape[1])), np.zeros(vocab)
    for i in np.flatnonzero((t >= 0) & (t < vocab)):
        dw[t[i]] += dy[i]
        size[t[i]] += np.abs(dy[i])
        count[t[i]] += 1
    dw, err = dw * scale, (count[:, None] + 2) * EPS32 * size * abs(scale)
    if before is not None:
        dw, err = dw + before, err + EPS32 * (np.abs(dw) + np.abs(before))
    return dw, err, count


def _softmax(z):
    with np.errstate(invalid="ignore"):
        top = z.max(1, keepdims=True)
        e = np.exp(z - top)
        s = e.sum(1, keepdims=True)
        return e / s, (top + np.log(s))[:, 0]


def head_loss(h, weight, labels, row_weight=None, half=EPS32, least=0.0, pairs=False):
    """A dict: loss, lse, dh, dweight and their bounds.  half: what rounding dz to its type is off by at most, relative to the value, where v is not the row's label; least: and absolutely, in units of the
    largest row weight (a type without small numbers).  pairs: the logits are products of pairs of fp16 terms: a number scaled to at most 2^14 is the sum of
    its terms up to 2^-22 of itself (two roundings of 2^-11) and 2^-25 (half fp16's smallest step; the largest lies above 2^13: 2^-38 of it), and of
    a product the terms' smallest part, 2^-22, is left out; three products are summed for each."""
    h, w, labels = np.asarray(h, np.float64), np.asarray(weight, np.float64), np.asarray(labels, np.int64)
    n, d = h.shape
    v = w.shape[0]
    live = (labels >= 0) & (labels < v)
    g = np.where(live, 1.0 if row_weight is None else np.asarray(row_weight, np.float64), 0.0)
    z = h @ w.T
    zerr = (2 * d + 32) * EPS32 * (np.abs(h) @ np.abs(w).T)
    if pairs:
        finite = lambda x: np.where(np.isfinite(x), np.abs(x), 0.0)                                  # noqa: E731
        zerr = 3 * zerr + 3 * 2.0 ** -22 * (np.abs(h) @ np.abs(w).T)
        zerr = zerr + 2.0 ** -38 * 1.01 * (finite(h).max(1, keepdims=True) * np.abs(w).sum(1)[None] + finite(w).max() * np.abs(h).sum(1)[:, None])
    p, lse = _softmax(z)
    # the sum over v: a tile's lane adds up to 128 terms, then the tiles are joined; arguments are rounded, as are the exponentials
    spread = np.abs(z - lse[:, None])
    perr = zerr + (8 + 2 * spread) * EPS32
    lse_err = (p * perr).sum(1) + (160 + v / 2048) * EPS32 + 2 * EPS32 * np.abs(lse)
    at = np.where(live, labels, 0)
    rows = np.arange(n)
    loss = np.where(live, lse - z[rows, at], 0.0)
    loss_err = np.where(live, lse_err + zerr[rows, at] + 2 * EPS32 * (np.abs(lse) + np.abs(z[rows, at])), 0.0)
    hot = np.zeros_like(p)
    hot[rows[live], labels[live]] = 1.0
    dz = g[:, None] * (p - hot)
    off = np.abs(g)[:, None] * (p * (perr + lse_err[:, None]) + 2 * EPS32 * (p + hot))
    # a row's own label is most of its gradient: it is kept in two terms at least (what rounding leaves is rounded once more)
    off = off + (np.abs(dz) + off) * np.where(hot > 0, max(half * half, EPS32), half) + np.where(g[:, None] != 0, least * np.abs(g).max(initial=0.0), 0.0) + 2 * LEAST * np.abs(g)[:, None]
    hl = np.where(live[:, None], h, 0.0)
    dh, dw = dz @ w, dz.T @ hl
    dh_err = off @ np.abs(w) + (2 * v + 64) * EPS32 * (np.abs(dz) @ np.abs(w)) + v * LEAST
    dw_err = off.T @ np.abs(hl) + (2 * n + 64) * EPS32 * (np.abs(dz).T @ np.abs(hl)) + n * LEAST
    return {"loss": loss, "loss_err": loss_err, "lse": lse, "lse_err": lse_err, "dh": dh, "dh_err": dh_err, "dweight": dw, "dweight_err": dw_err}


def topk_distill(logits, teacher, at, temperature=1.0, row_weight=None):
    """A dict: loss, dlogits and their bounds."""
    z, t, at = np.asarray(logits, np.float64) / temperature, np.asarray(teacher, np.float64) / temperature, np.asarray(at, np.int64)
    n, v = z.shape
    g = np.ones(n) if row_weight is None else np.asarray(row_weight, np.float64)
    with np.errstate(invalid="ignore"):
        known = (at >= 0) & (at < v) & (t > -np.inf)
    some = known.any(1)
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        p, lse = _softmax(z)
        tm = np.where(some, np.where(known, t, -np.inf).max(1), 0.0)[:, None]
        e = np.where(known, np.exp(np.where(known, t, 0.0) - tm), 0.0)
        share = np.where(some, e.sum(1), 1.0)[:, None]
        q = e / share
        log_q = t - tm - np.log(share)
        zj = np.take_along_axis(z, np.where(known, at, 0), 1)
        loss = np.where(q > 0, q * (log_q - zj + lse[:, None]), 0.0).sum(1) * temperature ** 2
        # at least 256 threads sum a row, each in groups of at least four that are added one after the other, then a tree
        top = np.where(np.isfinite(z), np.abs(z), 0.0).max(1)
        lse_err = (32 + v / 1024 + 4 * top) * EPS32
        far = np.where(known, np.abs(t), 0.0)
        qerr = (16 + at.shape[1] / 64 + 6 * far.max(1, keepdims=True)) * EPS32
        size = np.where(q > 0, q * (np.abs(log_q) + np.abs(zj) + np.abs(lse)[:, None]), 0.0)
        loss_err = temperature ** 2 * ((size * ((at.shape[1] / 64 + 16) * EPS32 + qerr)).sum(1) + lse_err)
        dz = p.copy()
        derr = p * (lse_err[:, None] + (8 + 4 * np.where(np.isfinite(z), np.abs(z), 0.0)) * EPS32)
        for i, j in zip(*np.nonzero(known)):
            dz[i, at[i, j]] -= q[i, j]
            derr[i, at[i, j]] += q[i, j] * (qerr[i, 0] + at.shape[1] * EPS32)
        c = (g * temperature)[:, None]
        dz, derr = np.where(some[:, None], dz * c, 0.0), np.where(some[:, None], (derr + 4 * EPS32 * np.abs(dz) + 2 * LEAST) * np.abs(c), 0.0)
    return {"loss": np.where(some, loss, 0.0), "loss_err": np.where(some, loss_err, 0.0), "dlogits": dz, "dlogits_err": derr}
