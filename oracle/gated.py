"""fp64 CPU oracle of the gated FC shard.

TEST INFRASTRUCTURE, as oracle/train.py.  It shares no code with the HIP library.

y = act(x Wg + bg) * (x Wu + bu) and the gradients of sum(dy * y) with respect to
x, both weights and both biases, each from its definition.  ``bounds`` says how far
a result formed from fp32 sums may be off, element by element.
"""
from __future__ import annotations

import numpy as np
from scipy import special

ACTS = ("sigmoid", "silu", "gelu", "gelu_tanh", "relu")
U = 2.0 ** -24                         # half a step of fp32
HALF16 = 2.0 ** -8                     # of bf16


def act(name, a):
    """act(a) and its derivative in float64."""
    a = np.asarray(a, np.float64)
    s = special.expit
    if name == "sigmoid":
        return s(a), s(a) * s(-a)
    if name == "silu":
        return a * s(a), s(a) + a * s(a) * s(-a)
    if name == "gelu":
        return a * special.ndtr(a), special.ndtr(a) + a * np.exp(-a * a / 2) / np.sqrt(2 * np.pi)
    if name == "gelu_tanh":
        r = np.sqrt(2 / np.pi)
        t = np.tanh(r * (a + 0.044715 * a ** 3))
        return a * (1 + t) / 2, (1 + t) / 2 + a * (1 - t * t) / 2 * r * (1 + 3 * 0.044715 * a * a)
    return np.maximum(a, 0), (a > 0).astype(np.float64)


def forward(name, x, wg, wu, bg=None, bu=None):
    """(y, a, u)."""
    x, wg, wu = (np.asarray(t, np.float64) for t in (x, wg, wu))
    a = x @ wg + (0 if bg is None else np.asarray(bg, np.float64))
    u = x @ wu + (0 if bu is None else np.asarray(bu, np.float64))
    return act(name, a)[0] * u, a, u


def backward(name, x, wg, wu, a, u, dy):
    """(dx, dwg, dwu, dbg, dbu)."""
    x, wg, wu, dy = (np.asarray(t, np.float64) for t in (x, wg, wu, dy))
    f, df = act(name, a)
    da, du = dy * u * df, dy * f
    return da @ wg.T + du @ wu.T, x.T @ da, x.T @ du, da.sum(0), du.sum(0)


def bounds(name, x, wg, wu, bg, bu, dy, bf16):
    """Bounds on the errors of (y, dx, dwg, dwu, dbg, dbu) with fp32 sums.

    A sum of n products: each product of the split is off by at most 2^-24 of it
    (bf16 ones are exact), and at most n / 16 + 16 roundings or truncations of
    partial sums, each 2^-24 of at most the sum of magnitudes, are on a term's
    way (32 terms a matrix instruction, its truncation counted twice, splits and
    epilogues behind it).  The activation and its derivative are off by at most
    16 roundings of their own pieces (of the size of a, and a^3 for the tanh form's
    derivative), their slopes are at most 1.13 and 1.  Next to its corner the ReLU's
    derivative may be either.  bf16 results add half a step, and there is room for
    another one of da and du in the bf16 dx (more than their two parts need)."""
    absx = np.abs(np.asarray(x, np.float64))
    awg, awu = (np.abs(np.asarray(w, np.float64)) for w in (wg, wu))
    y, a, u = forward(name, x, wg, wu, bg, bu)
    f, df = act(name, a)

    def off(n, magnitude):
        return (n / 16 + 16) * U * magnitude
    k = absx.shape[1]
    ea = off(k, absx @ awg + (0 if bg is None else np.abs(bg)))
    eu = off(k, absx @ awu + (0 if bu is None else np.abs(bu)))
    ef = 1.13 * ea + 16 * U * np.maximum(1, np.abs(a))
    ey = (np.abs(f) + ef) * eu + ef * np.abs(u) + 4 * U * np.abs(y)
    if bf16:
        ey = ey + HALF16 * (np.abs(y) + ey)
    if dy is None:
        return (ey,)
    edf = ea + 16 * U * (1 + np.abs(a) ** 3)
    if name == "relu":
        edf = (np.abs(a) <= ea).astype(np.float64)
    ady = np.abs(np.asarray(dy, np.float64))
    ada, adu = ady * np.abs(u) * np.abs(df), ady * np.abs(f)
    eda = ady * ((np.abs(u) + eu) * edf + eu * np.abs(df)) + 4 * U * ada
    edu = ady * ef + 4 * U * adu
    m, n = ady.shape
    out = [ey]
    ga, gu = eda, edu
    if bf16:
        ga, gu = eda + HALF16 * (ada + eda), edu + HALF16 * (adu + edu)
    ex = ga @ awg.T + gu @ awu.T + off(2 * n, (ada + ga) @ awg.T + (adu + gu) @ awu.T)
    if bf16:
        dx = backward(name, x, wg, wu, a, u, dy)[0]
        ex = ex + HALF16 * (np.abs(dx) + ex)
    out.append(ex)
    for e, v in ((eda, ada), (edu, adu)):
        out.append(absx.T @ e + off(m, absx.T @ (v + e)))
    for e, v in ((eda, ada), (edu, adu)):
        out.append(e.sum(0) + off(m, (v + e).sum(0)))
    return tuple(out)
