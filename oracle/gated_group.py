"""fp64 CPU oracle of the model-parallel part of a training step with gated layers
and AdamW updates.

TEST INFRASTRUCTURE, as oracle/train.py.  It shares no code with the HIP library.

K modulo iterations on the full (unsplit) dense layers: an MP group's column shards
side by side are the full layer, and the K-way sums of the shard and modulo layers
are the full layer's products.  Iteration k gathers block k of every worker's local
batch, in worker order; the loss is the mean negative log-likelihood over the
gathered rows; the gradients, divided by K, update the layers before iteration k + 1.
"""
from __future__ import annotations

import numpy as np

from . import adamw, gated
from .train import log_softmax_nll


def iterations(local, layers, labels, opt):
    """local [K][B][F]; layers: dicts of ``w`` and ``b`` (pairs for a gated layer, with
    its ``act``; else ``relu``); labels [K][B]; opt: lr, beta1, beta2, eps, decay (of the
    weights).  Returns (records of every iteration, layers after them, dlocal)."""
    K, B, _ = local.shape
    s = B // K
    f = np.float64
    layers = [dict(d, w=[np.array(w, f) for w in d["w"]], b=[np.array(b, f) for b in d["b"]])
              for d in layers]
    state = [{key: [(np.zeros_like(p), np.zeros_like(p)) for p in d[key]] for key in ("w", "b")}
             for d in layers]
    dlocal = np.zeros(local.shape, f)
    records = []
    for k in range(K):
        x = np.concatenate([local[w][k * s:(k + 1) * s] for w in range(K)]).astype(f)
        xs, saved = [x], []
        for d in layers:
            if "act" in d:
                y, a, u = gated.forward(d["act"], xs[-1], d["w"][0], d["w"][1], d["b"][0], d["b"][1])
                saved.append((a, u))
            else:
                y = xs[-1] @ d["w"][0] + d["b"][0]
                y = np.maximum(y, 0) if d["relu"] else y
                saved.append(y)
            xs.append(y)
        _, loss, g = log_softmax_nll(xs[-1], labels[k], 1.0 / B)
        grads = [None] * len(layers)
        for j in reversed(range(len(layers))):
            d = layers[j]
            if "act" in d:
                g, dwg, dwu, dbg, dbu = gated.backward(d["act"], xs[j], d["w"][0], d["w"][1],
                                                       *saved[j], g)
                grads[j] = {"w": [dwg, dwu], "b": [dbg, dbu]}
            else:
                g = g * (saved[j] > 0) if d["relu"] else g
                grads[j] = {"w": [xs[j].T @ g], "b": [g.sum(0)]}
                g = g @ d["w"][0].T
        for w in range(K):
            dlocal[w][k * s:(k + 1) * s] = g[w * s:(w + 1) * s]
        records.append({"logits": xs[-1], "loss": loss, "grads": grads})
        for d, st, gr in zip(layers, state, grads):
            for key in ("w", "b"):
                for i in range(len(d[key])):
                    d[key][i], m, v = adamw.update(
                        d[key][i], gr[key][i], *st[key][i], k + 1, opt["lr"], opt["beta1"],
                        opt["beta2"], opt["eps"], 1.0 / K, opt["decay"] if key == "w" else 0.0)
                    st[key][i] = (m, v)
    return records, layers, dlocal
