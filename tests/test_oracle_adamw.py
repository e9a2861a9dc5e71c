"""Pins of the AdamW oracle: torch's optimiser in float64, and what the moments
in bytes must satisfy (range, neighbours, an unbiased mean, special values)."""
import numpy as np
import pytest
import torch

from oracle import adamw as A


def test_update_equals_torch_adamw_over_several_steps():
    rng = np.random.default_rng(1)
    w = rng.normal(size=57)
    p = torch.nn.Parameter(torch.from_numpy(w.copy()))
    opt = torch.optim.AdamW([p], lr=3e-3, betas=(0.85, 0.99), eps=1e-6, weight_decay=0.1)
    m, v = np.zeros(57), np.zeros(57)
    for t in range(1, 8):
        g = rng.normal(size=57) * 10.0 ** rng.integers(-3, 3, 57)
        p.grad = torch.from_numpy(4.0 * g)
        opt.step()
        w, m, v = A.update(w, g, m, v, t, 3e-3, 0.85, 0.99, 1e-6, scale=4.0, decay=0.1)
        np.testing.assert_allclose(p.detach().numpy(), w, rtol=1e-12, atol=1e-14)


def _some(n, spread, seed):
    rng = np.random.default_rng(seed)
    m = (rng.normal(size=n) * 2.0 ** rng.integers(-spread, 1, n)).astype(np.float32)
    return m, (rng.normal(size=n) ** 2 * 2.0 ** rng.integers(-2 * spread, 1, n)).astype(np.float32)


@pytest.mark.parametrize("n", [1, 255, 256, 257, 1000])
def test_bytes_are_a_neighbour_of_the_value(n):
    m, v = _some(n, 4, n)
    got_m, got_v = A.unpack(*A.pack(m, v, A.noise(n, 5, 3, 7)))
    # Ranks are 1/8 of an octave's lower end apart, down to 15 and 31 octaves below
    # a block's largest value.
    for x, got, octaves in ((m, got_m, 15), (v, got_v, 31)):
        pad = np.concatenate([np.abs(x), np.zeros((-n) % 256, np.float32)]).reshape(-1, 256)
        within = np.abs(x) >= np.repeat(pad.max(axis=1), 256)[:n] * 2.0 ** -octaves
        assert within.mean() > 0.9
        assert np.all((np.abs(got - x) <= np.abs(x) / 8)[within])
        assert np.all((np.sign(got) == np.sign(x))[within])


def test_values_on_a_rank_are_kept():
    x = np.array([1.0, 1.125, 1.875, 2.0, 3.5, 2.0 ** -14], np.float32)
    for r in (0, 0xFFFF):
        noise = (np.full(6, r), np.full(6, r))
        m, v = A.unpack(*A.pack(-x, x, noise))
        assert np.array_equal(m, -x) and np.array_equal(v, x)


def test_rounding_is_right_on_average():
    n = 1 << 16
    for x in (1.01, 1.0625, 1.12, 1.999):
        one = np.full(n, x, np.float32)
        m, v = A.unpack(*A.pack(one, one, A.noise(n, 0, 1, 11)))
        # A sample of n choices between two values 1/8 apart at most: five
        # standard deviations of its mean, which are 1/16 / 256 each at most.
        assert abs(m.mean(dtype=np.float64) - x) < 5 / 16 / 256
        assert abs(v.mean(dtype=np.float64) - x) < 5 / 16 / 256
    a, b = A.noise(n, 0, 1, 11)
    assert abs(np.corrcoef(a, b)[0, 1]) < 5 / 256
    assert abs(np.corrcoef(a[1:], a[:-1])[0, 1]) < 5 / 256
    assert abs(np.corrcoef(a, A.noise(n, 0, 2, 11)[0])[0, 1]) < 5 / 256
    assert not np.array_equal(a, A.noise(n, 1 << 32, 1, 11)[0])


def test_range_zero_and_special_values():
    m = np.array([1.0, -2.0 ** -15, 2.0 ** -17, 0.0, -0.0], np.float32)
    v = np.array([1.0, 2.0 ** -31, 2.0 ** -40, 0.0, 2.0 ** -20], np.float32)
    none = (np.zeros(5, np.int64),) * 2
    got_m, got_v = A.unpack(*A.pack(m, v, none))
    assert np.array_equal(got_m, [1.0, -2.0 ** -15, 0, 0, 0])
    assert np.array_equal(got_v[[0, 1, 3, 4]], v[[0, 1, 3, 4]])
    assert got_v[2] == np.float32(1.25 * 2.0 ** -32)      # 254 ranks below the largest: not zero
    for bad in (np.inf, np.nan):
        m[1], v[1] = -bad, bad
        got_m, got_v = A.unpack(*A.pack(m, v, none))
        np.testing.assert_array_equal(np.abs(got_m[1]), bad)
        np.testing.assert_array_equal(got_v[1], bad)
        assert np.all(np.isfinite(np.delete(got_v, 1)))
    big = np.full(3, np.finfo(np.float32).max, np.float32)
    assert np.all(np.isfinite(A.unpack(*A.pack(big, big, (np.full(3, 0xFFFF),) * 2))[0]))


def test_second_moment_in_bytes_follows_a_change_of_the_gradient():
    """g doubles after 350 steps: v's mean must approach its new value (a v
    rounded to nearest would never move)."""
    n, beta2 = 4096, 0.99
    m, v = np.zeros(n, np.float32), np.zeros(n, np.float32)
    for t in range(1, 701):
        g = np.full(n, 1.0 if t <= 350 else 2.0, np.float32)
        nm, nv = A.moments(g, m, v, 0.9, beta2)
        m, v = A.unpack(*A.pack(nm, nv, A.noise(n, 0, t, 3)))
        if t == 350:
            # (1 - 0.99^350) and a mean over 4096 values each off by 1/8 at most.
            assert abs(v.mean() - (1 - beta2 ** 350)) < 0.02
    assert abs(v.mean() - 4.0) < 4 * 0.04
