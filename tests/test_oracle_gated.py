"""Pins of the gated shard's oracle: torch autograd in float64, central
differences, and column shards side by side."""
import numpy as np
import pytest
import torch

from oracle import gated as G

TORCH = {"sigmoid": torch.sigmoid, "silu": torch.nn.functional.silu,
         "gelu": torch.nn.functional.gelu,
         "gelu_tanh": lambda a: torch.nn.functional.gelu(a, approximate="tanh"),
         "relu": torch.relu}


def _case(m, k, n, seed=0):
    r = np.random.default_rng(seed)
    return (r.normal(size=(m, k)), r.normal(size=(k, n)) / np.sqrt(k), r.normal(size=(k, n)) / np.sqrt(k),
            r.normal(size=n), r.normal(size=n), r.normal(size=(m, n)))


@pytest.mark.parametrize("name", G.ACTS)
def test_against_torch_autograd(name):
    arrays = _case(7, 11, 5)
    t = [torch.from_numpy(a.copy()).requires_grad_(i < 5) for i, a in enumerate(arrays)]
    x, wg, wu, bg, bu, dy = t
    y = TORCH[name](x @ wg + bg) * (x @ wu + bu)
    y.backward(dy)
    gy, a, u = G.forward(name, *arrays[:5])
    np.testing.assert_allclose(gy, y.detach().numpy(), rtol=1e-12, atol=1e-14)
    got = G.backward(name, *arrays[:3], a, u, arrays[5])
    for g, p in zip(got, (x, wg, wu, bg, bu)):
        np.testing.assert_allclose(g, p.grad.numpy(), rtol=1e-11, atol=1e-13)


@pytest.mark.parametrize("name", G.ACTS[:4])
def test_derivative_against_differences(name):
    a = np.linspace(-9, 9, 181)
    h = 1e-5
    num = (G.act(name, a + h)[0] - G.act(name, a - h)[0]) / (2 * h)
    np.testing.assert_allclose(G.act(name, a)[1], num, atol=1e-9)
    slopes = np.abs(G.act(name, a)[1]), np.abs(np.diff(G.act(name, a)[1]) / (a[1] - a[0]))
    assert slopes[0].max() <= 1.13 and slopes[1].max() <= 1.0     # what bounds() takes


def test_column_shards_side_by_side():
    x, wg, wu, bg, bu, dy = _case(6, 9, 8)
    y, a, u = G.forward("silu", x, wg, wu, bg, bu)
    full = G.backward("silu", x, wg, wu, a, u, dy)
    parts = []
    for s in (slice(0, 4), slice(4, 8)):
        ys, as_, us = G.forward("silu", x, wg[:, s], wu[:, s], bg[s], bu[s])
        np.testing.assert_allclose(ys, y[:, s], rtol=1e-13)
        parts.append(G.backward("silu", x, wg[:, s], wu[:, s], as_, us, dy[:, s]))
    np.testing.assert_allclose(parts[0][0] + parts[1][0], full[0], rtol=1e-12, atol=1e-13)
    np.testing.assert_allclose(np.concatenate([p[1] for p in parts], 1), full[1], rtol=1e-12)


@pytest.mark.parametrize("name", G.ACTS)
@pytest.mark.parametrize("bf16", [False, True])
def test_bounds_hold_for_fp32_arithmetic_and_see_a_lost_term(name, bf16):
    x, wg, wu, bg, bu, dy = (a.astype(np.float32) for a in _case(40, 70, 30, 3))
    if bf16:
        x, wg, wu, dy = (torch.from_numpy(a).bfloat16().float().numpy() for a in (x, wg, wu, dy))
    t = [torch.from_numpy(a).requires_grad_(i < 5) for i, a in enumerate((x, wg, wu, bg, bu, dy))]
    y = TORCH[name](t[0] @ t[1] + t[3]) * (t[0] @ t[2] + t[4])
    y.backward(t[5])
    got = [y.detach()] + [p.grad for p in t[:5]]
    if bf16:
        got[:2] = [g.bfloat16().float() for g in got[:2]]
    ry, a, u = G.forward(name, x, wg, wu, bg, bu)
    ref = (ry,) + G.backward(name, x, wg, wu, a, u, dy)
    bound = G.bounds(name, x, wg, wu, bg, bu, dy, bf16)
    for g, r, b in zip(got, ref, bound):
        assert np.all(np.abs(g.numpy() - r) <= b)
    # A row less in the weight gradient, a column less in dx, are seen.
    lost = G.backward(name, x[:-1], wg, wu, a[:-1], u[:-1], dy[:-1])
    assert np.mean(np.abs(lost[2] - ref[3]) > bound[3]) > 0.3
    lost = G.backward(name, x, wg[:, :-1], wu[:, :-1], a[:, :-1], u[:, :-1], dy[:, :-1])
    assert np.mean(np.abs(lost[0] - ref[1]) > bound[1]) > 0.3
