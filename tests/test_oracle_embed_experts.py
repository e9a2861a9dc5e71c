"""Pins of the embedding's and the expert rows' oracles: torch autograd in float64,
shards side by side, and the bounds that the GPU tests use.  No GPU."""
import numpy as np
import pytest
import torch

from oracle import embed as E
from oracle import experts as X


def test_embedding_against_torch_autograd():
    r = np.random.default_rng(1)
    ids = r.integers(-2, 9, 40)
    table = torch.from_numpy(r.normal(size=(6, 5))).requires_grad_()
    inside = torch.from_numpy((ids >= 2) & (ids < 8))
    y = torch.nn.functional.embedding(torch.from_numpy(np.clip(ids - 2, 0, 5)), table) * 0.3 * inside[:, None]
    dy = r.normal(size=(40, 5))
    y.backward(torch.from_numpy(dy))
    np.testing.assert_allclose(E.forward(table.detach().numpy(), ids, 2, 0.3), y.detach().numpy(), rtol=1e-15)
    np.testing.assert_allclose(E.backward(dy, ids, 2, 6, 0.3), table.grad.numpy(), rtol=1e-12)
    old = r.normal(size=(6, 5))
    np.testing.assert_allclose(E.backward(dy, ids, 2, 6, 0.3, old), old + table.grad.numpy(), rtol=1e-12, atol=1e-14)


def test_vocabulary_shards_add_up():
    r = np.random.default_rng(2)
    ids, table, dy = r.integers(0, 9, 30), r.normal(size=(9, 4)), r.normal(size=(30, 4))
    parts = [E.forward(table[s:s + 3], ids, s, 2.0) for s in (0, 3, 6)]
    np.testing.assert_array_equal(sum(parts), E.forward(table, ids, 0, 2.0))
    grads = [E.backward(dy, ids, s, 3, 2.0) for s in (0, 3, 6)]
    np.testing.assert_array_equal(np.concatenate(grads), E.backward(dy, ids, 0, 9, 2.0))


def test_embedding_bounds_hold_and_see_a_lost_token():
    r = np.random.default_rng(3)
    ids, dy = r.integers(0, 5, 300), r.normal(size=(300, 16)).astype(np.float32)
    got = np.zeros((5, 16), np.float32)
    for i, t in enumerate(ids):
        got[t] += dy[i]
    got *= np.float32(0.3)
    scale = float(np.float32(0.3))
    ref, lim = E.backward(dy, ids, 0, 5, scale), E.backward_bound(dy, ids, 0, 5, scale)
    assert np.all(np.abs(got - ref) <= lim)
    lost = E.backward(dy[1:], ids[1:], 0, 5, scale)
    assert np.any(np.abs(lost - ref) > lim)


def _routing(r, n, top, whole):
    return np.stack([r.permutation(whole)[:top] for _ in range(n)]).astype(np.int32)


def test_experts_against_torch_autograd():
    r = np.random.default_rng(4)
    n, top, d = 30, 3, 5
    ids = _routing(r, n, top, 8)
    place, offsets = X.sort(ids, 2, 4)
    # Sorted by expert and, within one, by token.
    rows = np.argwhere((ids >= 2) & (ids < 6))
    want = sorted((ids[t, j], t * top + j) for t, j in rows)
    assert [place[s // top, s % top] for _, s in want] == list(range(len(want)))
    assert offsets[-1] == len(want) and all(
        offsets[e + 1] - offsets[e] == np.sum(ids == 2 + e) for e in range(4))
    x = torch.from_numpy(r.normal(size=(n, d))).requires_grad_()
    w = torch.from_numpy(r.uniform(size=(n, top))).requires_grad_()
    scale = torch.arange(1.0, 9.0, dtype=torch.float64)          # expert e multiplies by e + 1
    y = sum(w[:, j, None] * x * scale[torch.from_numpy(ids[:, j]).long(), None] *
            torch.from_numpy((place[:, j] >= 0).astype(float))[:, None] for j in range(top))
    dy = r.normal(size=(n, d))
    y.backward(torch.from_numpy(dy))
    xs = X.gather(x.detach().numpy(), place, np.zeros((n * top, d)))
    factor = np.zeros((n * top, 1))
    for e in range(4):
        factor[offsets[e]:offsets[e + 1]] = 3.0 + e
    ys = xs * factor
    np.testing.assert_allclose(X.combine(ys, place, w.detach().numpy()), y.detach().numpy(), rtol=1e-12, atol=1e-13)
    dys, dw = X.combine_backward(dy, ys, place, w.detach().numpy(), np.zeros_like(xs))
    np.testing.assert_allclose(dw, w.grad.numpy(), rtol=1e-12, atol=1e-13)
    np.testing.assert_allclose(X.combine(dys * factor, place), x.grad.numpy(), rtol=1e-12, atol=1e-13)


def test_workers_experts_add_up():
    r = np.random.default_rng(5)
    ids, x, w = _routing(r, 20, 2, 6), r.normal(size=(20, 3)), r.uniform(size=(20, 2))
    whole = X.combine(X.gather(x, *[X.sort(ids, 0, 6)[0], np.zeros((40, 3))]), X.sort(ids, 0, 6)[0], w)
    parts = 0
    for first in (0, 2, 4):
        place, _ = X.sort(ids, first, 2)
        parts = parts + X.combine(X.gather(x, place, np.zeros((40, 3))), place, w)
    np.testing.assert_allclose(parts, whole, rtol=1e-14)


@pytest.mark.parametrize("bf16", [False, True])
def test_expert_bounds_hold_and_see_a_lost_row(bf16):
    r = np.random.default_rng(6)
    n, top, d = 25, 4, 70
    place, _ = X.sort(_routing(r, n, top, 6), 0, 6)
    f = lambda *s: r.normal(size=s).astype(np.float32)
    dy, ys, w = f(n, d), f(n * top, d), r.uniform(size=(n, top)).astype(np.float32)
    if bf16:
        dy, ys = (torch.from_numpy(a).bfloat16().float().numpy() for a in (dy, ys))
    rows = np.zeros_like(ys)
    y32 = np.zeros((n, d), np.float32)
    dys32, dw32 = np.zeros_like(ys), np.zeros((n, top), np.float32)
    for t in range(n):
        for j in range(top):
            y32[t] += w[t, j] * ys[place[t, j]]
            dys32[place[t, j]] = w[t, j] * dy[t]
            dw32[t, j] = np.sum(dy[t] * ys[place[t, j]], dtype=np.float32)
    if bf16:
        y32, dys32 = (torch.from_numpy(a).bfloat16().float().numpy() for a in (y32, dys32))
    ey, edys, edw = X.bounds(dy, ys, place, w, rows, bf16)
    ref = (X.combine(ys, place, w),) + X.combine_backward(dy, ys, place, w, rows)
    # (Products and sums of numpy are rounded apart: twice the roundings of fused ones.)
    for got, want, lim in zip((y32, dys32, dw32), ref, (2 * ey, edys, 2 * edw)):
        assert np.all(np.abs(got - want) <= lim)
    lost = X.combine(ys, np.where(place == 3, -1, place), w)
    assert np.any(np.abs(lost - ref[0]) > ey)
