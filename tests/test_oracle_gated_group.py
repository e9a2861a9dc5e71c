"""Pin of oracle/gated_group.py: the same iterations in torch float64 with autograd
and torch's AdamW."""
import numpy as np
import torch

from oracle import gated_group as GG


def test_iterations_equal_torch_autograd_and_adamw():
    r = np.random.default_rng(4)
    K, B, F, H, C = 2, 6, 9, 8, 4
    local = r.normal(size=(K, B, F))
    labels = r.integers(0, C, size=(K, B))
    layers = [dict(act="silu", w=[r.normal(size=(F, H)) for _ in range(2)],
                   b=[r.normal(size=H) for _ in range(2)]),
              dict(relu=True, w=[r.normal(size=(H, H))], b=[r.normal(size=H)]),
              dict(relu=False, w=[r.normal(size=(H, C))], b=[r.normal(size=C)])]
    opt = dict(lr=1e-2, beta1=0.8, beta2=0.95, eps=1e-5, decay=0.1)
    rec, new, dlocal = GG.iterations(local, layers, labels, opt)
    P = [{key: [torch.tensor(p, requires_grad=True) for p in d[key]] for key in ("w", "b")}
         for d in layers]
    o = torch.optim.AdamW([dict(params=[p for q in P for p in q["w"]], weight_decay=0.1),
                           dict(params=[p for q in P for p in q["b"]], weight_decay=0.0)],
                          lr=1e-2, betas=(0.8, 0.95), eps=1e-5)
    s = B // K
    for k in range(K):
        x = torch.tensor(np.concatenate([local[w][k * s:(k + 1) * s] for w in range(K)]),
                         requires_grad=True)
        h = torch.nn.functional.silu(x @ P[0]["w"][0] + P[0]["b"][0]) * (x @ P[0]["w"][1] + P[0]["b"][1])
        h = torch.relu(h @ P[1]["w"][0] + P[1]["b"][0])
        z = h @ P[2]["w"][0] + P[2]["b"][0]
        loss = torch.nn.functional.cross_entropy(z, torch.tensor(labels[k]), reduction="none")
        o.zero_grad()
        loss.mean().backward()
        np.testing.assert_allclose(rec[k]["logits"], z.detach().numpy(), rtol=1e-10, atol=1e-12)
        np.testing.assert_allclose(rec[k]["loss"], loss.detach().numpy(), rtol=1e-10, atol=1e-12)
        for w in range(K):
            np.testing.assert_allclose(dlocal[w][k * s:(k + 1) * s],
                                       x.grad[w * s:(w + 1) * s].numpy(), rtol=1e-9, atol=1e-13)
        for q in P:
            for p in q["w"] + q["b"]:
                p.grad /= K
        o.step()
    for d, q in zip(new, P):
        for key in ("w", "b"):
            for a, b in zip(d[key], q[key]):
                np.testing.assert_allclose(a, b.detach().numpy(), rtol=1e-10, atol=1e-12)
