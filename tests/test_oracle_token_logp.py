"""Pins of the token log-probabilities' oracle: torch in float64, autograd, central
differences, rows with nothing left, and the bounds that the GPU tests use.  No GPU."""
import numpy as np
import pytest
import torch

from oracle import token_logp as L
from oracle import train


def _case(m=12, classes=30, seed=0, masked=True):
    r = np.random.default_rng(seed)
    z = r.normal(size=(m, classes)) * 3
    t = r.integers(0, classes, m)
    if masked:
        z[r.uniform(size=z.shape) < 0.2] = -np.inf
        z[np.arange(m), t] = r.normal(size=m)
    t[::5] = -1
    return z, t, r.normal(size=m), r.normal(size=m), r.normal(size=(m, 4))


def test_against_torch_and_the_loss():
    z, t, _, _, _ = _case(masked=False)
    f = L.forward(z, t, 4)
    lp = torch.log_softmax(torch.from_numpy(z), 1)
    ref = torch.where(torch.from_numpy(t) >= 0, lp[torch.arange(12), torch.from_numpy(t)], 0.0)
    np.testing.assert_allclose(f["logp"], ref.numpy(), rtol=1e-12)
    np.testing.assert_allclose(f["entropy"], torch.distributions.Categorical(logits=lp).entropy().numpy(), rtol=1e-12)
    v, i = torch.topk(lp, 4)
    np.testing.assert_array_equal(f["top_ids"], i.numpy())
    np.testing.assert_allclose(f["top_values"], v.numpy(), rtol=1e-12)
    np.testing.assert_allclose(f["stats"].sum(1), torch.logsumexp(torch.from_numpy(z), 1).numpy(), rtol=1e-13)
    good = np.where(t < 0, 0, t)
    _, loss, dz = train.log_softmax_nll(z, good, 0.25)
    g = L.forward(z, good)
    np.testing.assert_allclose(g["logp"], -loss, rtol=1e-12)
    np.testing.assert_allclose(L.backward(z, g, good, -0.25 * np.ones(12)), dz, rtol=1e-9, atol=1e-15)


@pytest.mark.parametrize("probs", [False, True])
def test_gradient_against_autograd_and_differences(probs):
    z, t, dl, dh, dt = _case(masked=False)
    f = L.forward(z, t, 4, probs)
    got = L.backward(z, f, t, dl, dh, dt, probs)

    def value(z):
        lp = torch.log_softmax(z, 1)
        p = lp.exp()
        ids = torch.from_numpy(f["top_ids"]).long()
        top = (p if probs else lp).gather(1, ids)
        valid = torch.from_numpy(t >= 0)
        logp = torch.where(valid, lp[torch.arange(12), torch.from_numpy(np.maximum(t, 0))], 0.0)
        return (torch.from_numpy(dl) * logp).sum() - (torch.from_numpy(dh) * (p * lp).sum(1)).sum() \
            + (torch.from_numpy(dt) * top).sum()
    zt = torch.from_numpy(z.copy()).requires_grad_()
    value(zt).backward()
    np.testing.assert_allclose(got, zt.grad.numpy(), rtol=1e-9, atol=1e-13)
    for i, c in ((0, 3), (5, 7), (11, 29)):
        h = np.zeros_like(z)
        h[i, c] = 1e-6
        num = (value(torch.from_numpy(z + h)) - value(torch.from_numpy(z - h))) / 2e-6
        assert abs(float(num) - got[i, c]) < 1e-7


def test_masked_classes_are_as_if_they_were_not_there():
    z, t, dl, dh, dt = _case()
    f = L.forward(z, t, 4)
    dz = L.backward(z, f, t, dl, dh, dt)
    assert np.all(dz[z == -np.inf] == 0) and np.all(np.isfinite(dz))
    for i in range(12):
        keep = np.flatnonzero(z[i] > -np.inf)
        ti = np.array([-1 if t[i] < 0 else np.flatnonzero(keep == t[i])[0]])
        g = L.forward(z[i:i + 1, keep], ti, 4)
        np.testing.assert_allclose(g["entropy"], f["entropy"][i:i + 1], rtol=1e-12)
        np.testing.assert_array_equal(keep[g["top_ids"][0]], f["top_ids"][i])
        np.testing.assert_allclose(L.backward(z[i:i + 1, keep], g, ti, dl[i:i + 1], dh[i:i + 1], dt[i:i + 1])[0],
                                   dz[i, keep], rtol=1e-9, atol=1e-13)


def test_rows_without_anything_ties_and_special_values():
    z = np.zeros((5, 6))
    z[0] = -np.inf
    z[2, 3] = np.nan
    z[3, 4] = np.inf
    z[4, 2] = -0.0
    t = np.array([1, 2, 0, 0, 9])
    f = L.forward(z, t, 3)
    assert f["logp"][0] == -np.inf and f["entropy"][0] == 0 and np.all(f["stats"][0] == -np.inf)
    assert list(f["top_ids"][0]) == [0, 1, 2] and np.all(f["top_values"][0] == -np.inf)
    assert list(f["top_ids"][1]) == [0, 1, 2] and list(f["top_ids"][4]) == [0, 1, 2]
    assert list(f["top_ids"][2]) == [3, 0, 1] and list(f["top_ids"][3]) == [4, 0, 1]
    assert np.all(np.isnan(f["logp"][2:])) and np.isnan(f["entropy"][2]) and np.isnan(f["entropy"][3])
    dz = L.backward(z, f, t, np.ones(5), np.ones(5))
    assert np.all(dz[0] == 0) and np.all(np.isfinite(dz[1])) and np.all(np.isnan(dz[2:]))


@pytest.mark.parametrize("bf16", [False, True])
@pytest.mark.parametrize("probs", [False, True])
def test_bounds_hold_for_fp32_arithmetic_and_see_a_lost_class(bf16, probs):
    z, t, dl, dh, dt = _case(20, 400, 3)
    dl, dh, dt = dl[:20], dh[:20], dt[:20]
    z, dl, dh, dt = (torch.from_numpy(a).float() for a in (z, dl, dh, dt))
    if bf16:
        z = z.bfloat16().float()
    f = L.forward(z.numpy(), t, 4, probs)
    args = (t, dl.numpy(), dh.numpy(), dt.numpy(), probs)
    lim = L.bounds(z.numpy(), f, *args, bf16=bf16)
    ref = dict(f, dz=L.backward(z.numpy(), f, *args))
    most = z.amax(1, keepdim=True)
    e = torch.exp(z - most)
    ls = torch.log(e.sum(1, keepdim=True))
    lp = z - most - ls
    p = lp.exp()
    ids = torch.from_numpy(f["top_ids"]).long()
    fin = torch.where(p > 0, lp, 0.0)
    h = -(p * fin).sum(1, keepdim=True)
    g = torch.zeros_like(z)
    rows = torch.arange(20)
    tt = torch.from_numpy(t)
    g[rows[tt >= 0], tt[tt >= 0]] = dl[tt >= 0]
    g.scatter_add_(1, ids, dt * (p.gather(1, ids) if probs else 1.0))
    dz = g - p * (g.sum(1, keepdim=True) + dh[:, None] * (fin + h))
    if bf16:
        dz = dz.bfloat16().float()
    got = {"stats": torch.cat([most, ls], 1), "entropy": h[:, 0], "dz": dz,
           "top_values": (p if probs else lp).gather(1, ids),
           "logp": torch.where(tt >= 0, lp[rows, tt.clamp(min=0)], 0.0)}
    for name, v in got.items():
        far = np.abs(v.double().numpy() - ref[name])
        assert np.all(far <= lim[name]), name
    lost = L.forward(np.where(np.arange(400) == 17, -np.inf, z.numpy()), t, 4, probs)
    assert np.mean(np.abs(lost["stats"][:, 1] - f["stats"][:, 1]) > lim["stats"][:, 1]) > 0.5
