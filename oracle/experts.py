"""fp64 CPU oracle of the expert rows: sorting by expert, laying out, bringing back.

TEST INFRASTRUCTURE, as oracle/train.py.  It shares no code with the HIP library.
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24                         # half a step of fp32
HALF16 = 2.0 ** -8                     # of bf16


def sort(ids, first, experts):
    """(place, offsets): expert after expert, the tokens of each in their order."""
    place = np.full(ids.shape, -1, np.int32)
    offsets = np.zeros(experts + 1, np.int32)
    row = 0
    for e in range(experts):
        offsets[e] = row
        for t, j in np.argwhere(ids == first + e):
            place[t, j] = row
            row += 1
    offsets[experts] = row
    return place, offsets


def gather(x, place, rows):
    """rows: what the sorted rows hold before."""
    xs = np.array(rows, np.float64)
    for t, j in np.argwhere(place >= 0):
        xs[place[t, j]] = x[t]
    return xs


def combine(ys, place, weights=None, add=None):
    y = np.zeros((place.shape[0], ys.shape[1])) if add is None else np.array(add, np.float64)
    for t, j in np.argwhere(place >= 0):
        y[t] += (1.0 if weights is None else float(weights[t, j])) * np.asarray(ys[place[t, j]], np.float64)
    return y


def combine_backward(dy, ys, place, weights, rows):
    dys, dw = np.array(rows, np.float64), np.zeros(place.shape)
    for t, j in np.argwhere(place >= 0):
        dys[place[t, j]] = (1.0 if weights is None else float(weights[t, j])) * np.asarray(dy[t], np.float64)
        dw[t, j] = np.asarray(dy[t], np.float64) @ np.asarray(ys[place[t, j]], np.float64)
    return dys, dw


def bounds(dy, ys, place, weights, rows, bf16, add=None):
    """Bounds on the errors of (y, dys, dw).  y: `top` fused products, each sum rounded once in fp32; dys: one
    product; dw: at most width / 64 + 8 products a lane and 6 sums of lanes.  bf16 adds half a step of the
    result (not of dw, which is fp32)."""
    w = None if weights is None else np.abs(weights)
    half = HALF16 if bf16 else 0.0
    y = np.abs(combine(ys, place, weights, add))
    ey = place.shape[1] * U * combine(np.abs(ys), place, w, None if add is None else np.abs(add))
    ey = ey + half * (y + ey)
    dys, dw = combine_backward(np.abs(dy), np.abs(ys), place, w, np.zeros_like(rows))
    edys = U * dys
    if weights is None:
        edys = np.zeros_like(dys)
    else:
        edys = edys + half * (dys + edys)
    return ey, edys, (dy.shape[1] / 64 + 14) * U * dw
