"""fp64 CPU oracle of the embedding shard.

TEST INFRASTRUCTURE, as oracle/train.py.  It shares no code with the HIP library.
Element by element from the definition: a token's row of the table, scaled; a row's
gradient the sum over the tokens that name it.
"""
from __future__ import annotations

import numpy as np

U = 2.0 ** -24                         # half a step of fp32
HALF16 = 2.0 ** -8                     # of bf16


def forward(table, ids, first, scale):
    table = np.asarray(table, np.float64)
    y = np.zeros((len(ids), table.shape[1]))
    for i, t in enumerate(ids):
        if first <= t < first + table.shape[0]:
            y[i] = scale * table[t - first]
    return y


def backward(dy, ids, first, vocab, scale, old=None):
    dy = np.asarray(dy, np.float64)
    d = np.zeros((vocab, dy.shape[1])) if old is None else np.array(old, np.float64)
    for i, t in enumerate(ids):
        if first <= t < first + vocab:
            d[t - first] += scale * dy[i]
    return d


def forward_bound(y, scale, bf16):
    """One product, rounded once to fp32 and once to bf16; rows as they are with a scale of 1."""
    if scale == 1:
        return np.zeros_like(y)
    e = U * np.abs(y)
    return e + HALF16 * (np.abs(y) + e) if bf16 else e


def backward_bound(dy, ids, first, vocab, scale, old=None):
    """c terms in fp32 have at most c - 1 roundings each of at most the sum of magnitudes; the scale and the
    sum with what was there add one each."""
    dy = np.abs(np.asarray(dy, np.float64))
    size = backward(dy, ids, first, vocab, abs(scale))
    count = backward(np.ones((len(ids), 1)), ids, first, vocab, 1.0)
    e = (count + 1) * U * size
    if old is not None:
        e = e + np.where(count > 0, U, 0) * (np.abs(np.asarray(old, np.float64)) + size + e)
    return e
