"""CPU oracle of the AdamW step: the update in float64, and the moments in bytes.

TEST INFRASTRUCTURE, as oracle/train.py.  It shares no code with the HIP library.

* Update: first and second moments are running means of the gradient (times a
  per-tensor scale) and of its square; the parameter shrinks by lr * decay and
  moves by lr times the bias-corrected first moment over the root of the
  bias-corrected second one plus eps.
* Bytes: a magnitude's rank is the number of its fp32 pattern without the lower
  20 bits, rounded up if 16 random bits (at weights 16 .. 2^19, and 8) carry into
  it.  A block of 256 has the largest rank as its reference; a byte holds how far
  below it a value's rank lies.  Since the rank follows from a pattern, ``moments``
  forms the two sums in fp32, each product rounded before the sum.
"""
from __future__ import annotations

import numpy as np

BLOCK = 256


def update(w, g, m, v, t, lr, beta1, beta2, eps, scale=1.0, decay=0.0):
    """(w, m, v) after update number t, in float64."""
    w, g, m, v = (np.asarray(a, np.float64) for a in (w, g, m, v))
    g = g * scale
    m = beta1 * m + (1.0 - beta1) * g
    v = beta2 * v + (1.0 - beta2) * g * g
    m_hat, v_hat = m / (1.0 - beta1 ** t), v / (1.0 - beta2 ** t)
    return w - lr * decay * w - lr * m_hat / (np.sqrt(v_hat) + eps), m, v


def moments(g, m, v, beta1, beta2, scale=1.0):
    """The new moments in fp32, from fp32 ones, as the library rounds them."""
    f = np.float32
    with np.errstate(all="ignore"):
        g = np.asarray(g, f) * f(scale)
        return (np.asarray(m, f) * f(beta1) + g * f(1.0 - beta1),
                np.asarray(v, f) * f(beta2) + (g * g) * f(1.0 - beta2))


def _mix(x):
    x = np.asarray(x, np.uint32)
    with np.errstate(over="ignore"):
        for shift, odd in ((16, 0x9E3779B9), (15, 0xB7E15163)):
            x = (x ^ (x >> np.uint32(shift))) * np.uint32(odd)
    return x ^ (x >> np.uint32(16))


def noise(n, first, t, seed):
    """The 16 random bits of both moments of n elements."""
    golden = 0x9E3779B9
    key = _mix((seed + t * golden) & 0xFFFFFFFF)
    number = np.uint64(first) + np.arange(n, dtype=np.uint64)
    low = (number & np.uint64(0xFFFFFFFF)).astype(np.uint32)
    high = (number >> np.uint64(32)).astype(np.uint32)
    with np.errstate(over="ignore"):
        h = _mix(low ^ key ^ high * np.uint32(golden))
    return (h & np.uint32(0xFFFF)).astype(np.int64), (h >> np.uint32(16)).astype(np.int64)


def _ranks(x, random):
    bits = np.abs(np.asarray(x, np.float32)).view(np.uint32).astype(np.int64)
    rank = np.minimum((bits + 16 * random + 8) // (1 << 20), 0x7F7)
    rank[np.isinf(x)] = 0x7F8
    rank[np.isnan(x)] = 0x7FC
    return rank


def _tops(rank):
    pad = np.zeros((-len(rank)) % BLOCK, np.int64)
    return np.concatenate([rank, pad]).reshape(-1, BLOCK).max(axis=1)


def pack(m, v, random):
    """(m bytes, m references, v bytes, v references); random: noise()."""
    out = []
    for x, r, steps, least in ((m, random[0], 127, 0), (v, random[1], 255, 1)):
        x = np.asarray(x, np.float32)
        rank = _ranks(x, r)
        top = _tops(rank)
        code = np.maximum(rank - np.repeat(top, BLOCK)[:len(x)] + steps, least)
        if steps == 127:
            code = code + 128 * ((code > 0) & (x < 0))
        else:
            code = np.where(x == 0, 0, code)
        out += [code.astype(np.uint8), top.astype(np.int16)]
    return out


def unpack(mb, mt, vb, vt):
    """fp32 values of both moments."""
    def values(code, top, steps):
        rank = np.repeat(top.astype(np.int64), BLOCK)[:len(code)] + code - steps
        rank = np.where((code > 0) & (rank > 0), rank, 0)
        return (rank << 20).astype(np.uint32).view(np.float32)
    mb, vb = mb.astype(np.int64), vb.astype(np.int64)
    m = values(mb % 128, mt, 127)
    return np.where(mb > 127, -m, m).astype(np.float32), values(vb, vt, 255)
