"""fp64 CPU oracle of the token log-probabilities, entropies and alternatives.

TEST INFRASTRUCTURE, as oracle/train.py.  It shares no code with the HIP library.

With p = softmax(z): logp = log p at the target, entropy = -sum p log p (0 log 0 is 0),
the `top` largest logits, of equal ones the lower class first; the gradient of
sum(dlogp logp) + sum(dentropy entropy) + sum(dtop top_values).
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24                         # half a step of fp32
HALF16 = 2.0 ** -8                     # of bf16
TINY = 2.0 ** -120                     # where the exponential's smallest results are lost


def forward(z, targets=None, top=0, probs=False):
    """A dict of logp, entropy, stats, top_ids, top_values and (for the bounds) lp, all log-probabilities."""
    z = np.asarray(z, np.float64)
    m, classes = z.shape
    with np.errstate(invalid="ignore", divide="ignore"):
        most = z.max(1, keepdims=True)
        none = np.all(z == -np.inf, 1, keepdims=True)
        x = np.exp(z - np.where(none, 0, most))
        # Without the largest term, 1: the logarithm of a sum next to 1 keeps its bits.
        np.put_along_axis(x, z.argmax(1)[:, None], np.where(np.isnan(most), np.nan, 0.0), 1)
        ls = np.where(most == np.inf, np.nan, np.where(none, -np.inf, np.log1p(x.sum(1, keepdims=True))))
        lp = np.where((z == -np.inf) & ~np.isnan(ls), -np.inf, z - most - ls)
        p = np.exp(lp)
        plp = np.where(lp == -np.inf, 0.0, p * np.where(lp == -np.inf, 0, lp))
        got = {"lp": lp, "entropy": 0.0 - plp.sum(1), "stats": np.concatenate([most, ls], 1)}
    if targets is not None:
        logp = np.zeros(m)
        for i, t in enumerate(targets):
            logp[i] = 0.0 if t < 0 else np.nan if t >= classes else lp[i, t]
        got["logp"] = logp
    if top:
        # NaN above all, then larger logits, then lower classes (the sort is stable).
        order = np.argsort(np.where(np.isnan(z), -np.inf, -z), axis=1, kind="stable")
        first = np.argsort(~np.isnan(np.take_along_axis(z, order, 1)), axis=1, kind="stable")
        ids = np.take_along_axis(order, first, 1)[:, :top]
        got["top_ids"] = ids.astype(np.int32)
        v = np.take_along_axis(lp, ids, 1)
        got["top_values"] = np.exp(v) if probs else v
    return got


def backward(z, f, targets=None, dlogp=None, dentropy=None, dtop=None, probs=False):
    """f: what forward gave."""
    lp = f["lp"]
    m, classes = lp.shape
    p = np.exp(lp)
    with np.errstate(invalid="ignore"):
        g = np.zeros_like(p)                   # gradient on the log-probabilities
        bad = np.zeros(m, bool)
        if dlogp is not None:
            for i, t in enumerate(targets):
                if t >= classes:
                    bad[i] = True
                elif t >= 0:
                    g[i, t] += dlogp[i]
        if dtop is not None:
            for i in range(m):
                for k, c in enumerate(f["top_ids"][i]):
                    g[i, c] += dtop[i, k] * (p[i, c] if probs else 1.0)
        if dentropy is not None:
            finite = np.where(lp == -np.inf, 0, lp)
            g -= np.asarray(dentropy, np.float64)[:, None] * p * (finite + 1)
        dz = g - p * g.sum(1, keepdims=True)
    dz[f["stats"][:, 1] == -np.inf] = 0.0      # rows of -inf alone
    dz[bad] = np.nan
    dz[np.isnan(f["stats"][:, 1])] = np.nan
    return dz


def bounds(z, f, targets=None, dlogp=None, dentropy=None, dtop=None, probs=False, bf16=False):
    """Bounds on the errors of the forward's outputs and dz, rows of finite logits and -inf.

    t = z - M is off by U |t|; exp(t) by 3 U |t| (t, log2 e and their product) and 2 U of its own, of itself.
    On a term's way lie at most R roundings: 64 terms of a lane, 6 sums of lanes, 8 stretches a lane and 6
    sums again, and 8 products where stretches are joined.  log1p, exp and expm1 are off by 4 U of their
    results."""
    R = 64 + 6 + 8 + 6 + 8
    lp = f["lp"]
    t = np.where(lp == -np.inf, 0.0, lp + f["stats"][:, 1:])
    x = np.exp(lp + np.where(np.isfinite(f["stats"][:, 1:]), f["stats"][:, 1:], 0))
    a = np.abs(t)
    S = np.maximum(x.sum(1), TINY)
    own = x * (a > 0)                          # the largest is not summed
    eO = (own * (3 * a + 2 + R) * U).sum(1) + TINY
    ls = np.where(np.isfinite(f["stats"][:, 1]), f["stats"][:, 1], 0)
    els = eO / S + 4 * U * ls
    h = (x * a).sum(1) / S
    es = (x * a * (3 * a + 5 + R) * U).sum(1)
    eh = els + es / S + h * eO / S + 4 * U * h + U * np.abs(f["entropy"]) + TINY
    fin = np.where(lp == -np.inf, 0.0, lp)
    elp = els[:, None] + U * a + U * np.abs(fin)
    got = {"stats": np.stack([np.zeros(len(ls)), els], 1), "entropy": eh}
    p = np.exp(lp)
    rows = np.arange(len(ls))[:, None]
    if targets is not None:
        c = np.clip(targets, 0, lp.shape[1] - 1)[:, None]
        got["logp"] = np.where(targets >= 0, elp[rows, c][:, 0], 0)
    ep = p * (elp + 3 * U * np.abs(fin) + 4 * U) + TINY
    if "top_ids" in f:
        got["top_values"] = (ep if probs else elp)[rows, f["top_ids"]]
    if dlogp is None and dentropy is None and dtop is None:
        return got
    g, eg = np.zeros_like(p), np.zeros_like(p)
    if dlogp is not None:
        for i, c in enumerate(targets):
            if 0 <= c < p.shape[1]:
                g[i, c] += abs(dlogp[i])
    terms = 3
    if dtop is not None:
        terms += dtop.shape[1]
        for i in range(len(ls)):
            for k, c in enumerate(f["top_ids"][i]):
                g[i, c] += abs(dtop[i, k]) * (p[i, c] if probs else 1.0)
                eg[i, c] += abs(dtop[i, k]) * (ep[i, c] + U * p[i, c]) if probs else 0.0
    dh = np.abs(dentropy)[:, None] if dentropy is not None else np.zeros((len(ls), 1))
    H = np.abs(f["entropy"])[:, None]
    size = g.sum(1, keepdims=True) + dh * H
    eall = terms * U * size + eg.sum(1, keepdims=True) + dh * eh[:, None]
    inner = size + g + dh * np.abs(fin)
    e = ep * inner + p * (eall + eg + dh * elp + 4 * U * inner)
    e = e + (g + eg) * (ep + 6 * U * (1 - p)) + terms * U * g + eg
    if bf16:
        dz = np.abs(backward(z, f, targets, dlogp, dentropy, dtop, probs))
        e = e + HALF16 * (np.where(np.isfinite(dz), dz, 0) + e)
    got["dz"] = e + TINY
    return got
