"""64-bit oracle of the sequence operators (root-mean-square norm, gated recurrence, AdamW), in numpy, from the formulas.

Shares no code with the library.  The recurrence goes token by token; its backward pass is the chain rule written
out, and tests compare it with differences of the forward pass.  Next to the values stand error bounds for fp32
arithmetic: what a sum of products of correctly typed operands can be off when every operation rounds to 2^-24, carried through the
same recurrence as the values (a step's error decays with the state)."""
from __future__ import annotations

import numpy as np

EPS32 = 2.0 ** -24
E4M3_MAX = 448.0
TINY = 2.0 ** -100


def sigmoid(x):
    e = np.exp(-np.abs(x))
    return np.where(x >= 0, 1.0, e) / (1.0 + e)


# ------------------------------------------------------------------------------------------------------------ e4m3
def e4m3_values():
    """The 256 values of the codes (OCP e4m3: no infinities, 0x7f and 0xff are NaN)."""
    c = np.arange(256)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c >> 7, -v, v)


def e4m3_spacing(x):
    """Distance of the e4m3 values around |x| <= 448."""
    return 2.0 ** (np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -6))) - 3)


# ------------------------------------------------------------------------------------------------------------ norm
def rmsnorm(x, weight, residual=None, eps=1e-6):
    """(y, s, scale): y unrounded, s = x + residual, scale of the 8-bit output's rows."""
    s = np.asarray(x, np.float64) + (0.0 if residual is None else np.asarray(residual, np.float64))
    y = s / np.sqrt((s * s).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
    return y, s, np.maximum(np.abs(y).max(-1), TINY) / E4M3_MAX


def rmsnorm_backward(s, weight, dy, dtotal=None, eps=1e-6):
    """(dx, dweight, bound of dx's fp32 error, bound of dweight's)."""
    s, w, dy = (np.asarray(v, np.float64) for v in (s, weight, dy))
    r = 1.0 / np.sqrt((s * s).mean(-1, keepdims=True) + eps)
    g, xh = dy * w, s * r
    dx = r * (g - xh * (g * xh).mean(-1, keepdims=True))
    size = r * (np.abs(g) + np.abs(xh) * np.abs(g * xh).mean(-1, keepdims=True))
    if dtotal is not None:
        dx, size = dx + dtotal, size + np.abs(dtotal)
    rows = s.reshape(-1, s.shape[-1]).shape[0]
    dw, total = (dy * xh).reshape(rows, -1).sum(0), np.abs(dy * xh).reshape(rows, -1).sum(0)
    # a thread adds up to 32 products before the tree, roots and quotients add a few roundings
    return dx, dw, 64 * EPS32 * size, (64 + rows / 32) * EPS32 * total


# ------------------------------------------------------------------------------------------------------ recurrence
def recurrence(u, gate, out_gate=None, bias=None, lengths=None, state=None):
    """Token by token.  Returns a dict: y, state (the last one), h [b, t+1, d] (h[:, 0] the initial state), and bounds
    y_err, state_err, h_err of fp32 arithmetic."""
    u, gate = np.asarray(u, np.float64), np.asarray(gate, np.float64)
    b, t, d = u.shape
    x = gate + (0.0 if bias is None else np.asarray(bias, np.float64))
    a, z = sigmoid(x), sigmoid(-x)
    live = np.ones((b, t), bool) if lengths is None else np.arange(t)[None] < np.clip(np.asarray(lengths), 0, t)[:, None]
    h, err = np.zeros((b, t + 1, d)), np.zeros((b, t + 1, d))
    if state is not None:
        h[:, 0] = state
    for i in range(t):
        on = live[:, i, None]
        step = a[:, i] * h[:, i] + z[:, i] * u[:, i]
        # exp's argument is rounded: |x| units; the rest of a sigmoid, the product and the sum, the pairs' own products: 8
        with np.errstate(invalid="ignore"):
            off = a[:, i] * err[:, i] + (8 + 2 * np.abs(x[:, i])) * EPS32 * (np.abs(a[:, i] * h[:, i]) + np.abs(z[:, i] * u[:, i]))
        h[:, i + 1], err[:, i + 1] = np.where(on, step, h[:, i]), np.where(on, off, err[:, i])
    if out_gate is None:
        gain = np.ones_like(u)
        gerr = np.zeros_like(u)
    else:
        o = np.asarray(out_gate, np.float64)
        gain = o * sigmoid(o)
        gerr = (6 + np.abs(o)) * EPS32 * np.abs(gain)
    m = live[:, :, None]
    with np.errstate(invalid="ignore"):
        y = np.where(m, h[:, 1:] * gain, 0.0)
        yerr = np.where(m, err[:, 1:] * np.abs(gain) + np.abs(h[:, 1:]) * gerr, 0.0)
    return {"y": y, "y_err": yerr, "state": h[:, t], "state_err": err[:, t], "h": h, "h_err": err, "a": a, "z": z, "live": live}


def recurrence_backward(u, gate, dy, out_gate=None, bias=None, lengths=None, state=None, dstate_out=None):
    """Gradients du, dgate, dout_gate, dbias, dstate and their bounds (names with _err)."""
    f = recurrence(u, gate, out_gate, bias, lengths, state)
    u, dy = np.asarray(u, np.float64), np.asarray(dy, np.float64)
    b, t, d = u.shape
    x = np.asarray(gate, np.float64) + (0.0 if bias is None else np.asarray(bias, np.float64))
    a, z, m = f["a"], f["z"], f["live"][:, :, None]
    u, dy, x = np.where(m, u, 0.0), np.where(m, dy, 0.0), np.where(m, x, 0.0)
    a, z = np.where(m, a, 1.0), np.where(m, z, 0.0)
    rel = (8 + 2 * np.abs(x)) * EPS32
    if out_gate is not None:
        o = np.where(m, np.asarray(out_gate, np.float64), 0.0)
        s = sigmoid(o)
        c, cerr = dy * o * s, (8 + np.abs(o)) * EPS32 * np.abs(dy * o * s)
    else:
        c, cerr = dy, np.zeros_like(dy)
    e = np.zeros((b, d)) if dstate_out is None else np.asarray(dstate_out, np.float64).copy()
    eerr = np.zeros((b, d))
    dh, dherr = np.zeros_like(u), np.zeros_like(u)
    for i in range(t - 1, -1, -1):
        dh[:, i] = c[:, i] + e
        dherr[:, i] = cerr[:, i] + eerr + 2 * EPS32 * (np.abs(c[:, i]) + np.abs(e))
        e = a[:, i] * dh[:, i]
        eerr = a[:, i] * dherr[:, i] + np.where(m[:, i], rel[:, i] * np.abs(e), 0.0)
    before, berr = f["h"][:, :-1], f["h_err"][:, :-1]
    out = {"du": z * dh, "du_err": z * dherr + rel * np.abs(z * dh), "dstate": e, "dstate_err": eerr}
    diff = before - u
    out["dgate"] = np.where(m, dh * diff * a * z, 0.0)
    out["dgate_err"] = np.where(m, a * z * (np.abs(dh) * (berr + EPS32 * np.abs(diff)) + dherr * np.abs(diff)) + 2 * rel * np.abs(out["dgate"]), 0.0)
    out["dbias"] = out["dgate"].sum((0, 1))
    out["dbias_err"] = out["dgate_err"].sum((0, 1)) + (64 + b * t / 64) * EPS32 * np.abs(out["dgate"]).sum((0, 1))
    if out_gate is not None:
        slope = s * (1.0 + o * (1.0 - s))
        size = s * (1.0 + np.abs(o) * (1.0 - s))
        h = f["h"][:, 1:]
        out["dout_gate"] = np.where(m, dy * h * slope, 0.0)
        # 1 + o (1 - s) cancels around o = -1.28, and 1 - s has 2^-24 of 1 as its error
        out["dout_gate_err"] = np.where(m, np.abs(dy) * (f["h_err"][:, 1:] * np.abs(slope) + np.abs(h) * ((8 + np.abs(o)) * EPS32 * size + 2 * EPS32 * s * np.abs(o))), 0.0)
    return out


# ----------------------------------------------------------------------------------------------------------- AdamW
def element_hash(n, seed, first=0):
    """The 32-bit random number of each of n elements (the definition: products modulo 2^32, xor-shifts)."""
    x = (np.arange(first, first + n, dtype=np.uint64) * np.uint64(0x9E3779B1) + np.uint64((seed * 0x632BE5AB) & 0xFFFFFFFF)) & np.uint64(0xFFFFFFFF)
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x21F0AAAD)) & np.uint64(0xFFFFFFFF)
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0x735A2D97)) & np.uint64(0xFFFFFFFF)
    return (x ^ (x >> np.uint64(15))).astype(np.int64)


def adamw(p, g, m, v, lr, step, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.0, grad_scale=1.0):
    """(p, m, v) after one step on 64-bit states."""
    b1, b2 = betas
    g = np.asarray(g, np.float64) * grad_scale
    m, v = b1 * np.asarray(m, np.float64) + (1 - b1) * g, b2 * np.asarray(v, np.float64) + (1 - b2) * g * g
    p = np.asarray(p, np.float64)
    return p - lr * weight_decay * p - lr * (m / (1 - b1 ** step)) / (np.sqrt(v / (1 - b2 ** step)) + eps), m, v
