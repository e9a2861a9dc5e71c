"""GPU parity of the token log-probabilities where single numbers decide: logits and
masks of any magnitude, over whole stretches of a row and alone; NaN in a row's first
class; the gradient of rows that are sure of their token; probabilities far below 1.
The shapes reach what tests/test_gpu_token_logp.py leaves: stretches of the longest
and the shortest kind, many blocks of the joining launch."""
import numpy as np
import pytest
import torch

from oracle import token_logp as L
from tests.helpers import print_case
from tests.test_gpu_token_logp import FWD, Case

pytestmark = pytest.mark.gpu

U = 2.0 ** -24                         # half a step of fp32
# Magnitudes on both sides of every limit that a kernel might draw, of both signs.
VALUES = [s * v for v in (9e5, 1.2e6, 1e8, 1e9, 1e10, 1e20, 9e29) for s in (1, -1)]
KINDS = 6


def _large(m, n, dtype):
    """Rows of ordinary logits with one of VALUES in one of KINDS ways."""
    r = np.random.default_rng(m + n)
    z = (r.normal(size=(m, n)) * 2).astype(np.float32)
    step = 1 << 16 if dtype == "bf16" else 1
    for i in range(m):
        at = i * 13 % (len(VALUES) * KINDS)         # 13: any six rows are of all kinds
        v, kind = np.float32(VALUES[at // KINDS]), at % KINDS
        if kind == 0:                               # all of them
            z[i] = v
        elif kind == 1:                             # a ruled-out tail
            z[i, n // 2:] = -abs(v)
        elif kind == 2:                             # one ahead of the others
            z[i, n // 3] = abs(v)
        elif kind == 3:                             # most of the row ruled out
            z[i, 100:] = -abs(v)
        elif kind == 4:                             # a few of the type's steps apart
            z[i] = (v.view(np.int32) + r.integers(0, 8, n) * step).astype(np.int32).view(np.float32)
        else:                                       # two ahead of the others, apart
            z[i, [n // 5, n - 2]] = abs(v)
    return z


# fp32 pieces of a lane's stretch / bf16: 84 x 1025 to 8192 a block a row, 84 x 50001 stretches
# of 4 / 13 of 8 in a block, 6 x 70000 of 1 / 1, 6 x 140000 of 2 / 1, 460 x 33000 of 8 / 8.
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,top", [(84, 700, 8), (84, 1025, 8), (84, 5000, 20), (84, 8192, 8), (84, 50001, 20),
                                     (6, 70000, 8), (6, 140000, 20), (460, 33000, 8)])
def test_logits_of_any_magnitude(m, n, top, dtype):
    print_case("token_logp magnitudes", m=m, n=n, top=top, dtype=dtype)
    c = Case(dtype, m, n, 0, 0, top, False, None, z=_large(m, n, dtype))
    c.fwd()
    c.bwd()
    c.check(FWD + ("top_ids", "dz"))
    c.untouched()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,top", [(8, 5000, 8), (8, 50001, 20), (8, 140000, 32)])
def test_stretches_ruled_out_whole(m, n, top, dtype):
    """Most stretches of -inf alone, in some rows all but fewer classes than are asked for."""
    print_case("token_logp ruled out", m=m, n=n, top=top, dtype=dtype)
    z = (np.random.default_rng(n).normal(size=(m, n)) * 2).astype(np.float32)
    z[0, n // 2:] = -np.inf
    z[1, :n // 2] = -np.inf
    z[2, 5:] = -np.inf
    z[3, :n - 3] = -np.inf
    z[4, 10:n - 10] = -np.inf
    z[5] = 0.25
    z[6] = 0.25
    z[6, n // 2:] = -np.inf
    t = [0, n - 1, 4, n - 2, -1, n // 2, 7, 8]
    c = Case(dtype, m, n, 0, 0, top, False, None, z=z, targets=t)
    c.fwd()
    c.bwd()
    c.check(FWD + ("top_ids", "dz"))
    c.untouched()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [300, 1025, 5000, 50001, 70000])
def test_nan_in_the_first_class(n, dtype):
    """NaN ranks above all classes, in class 0 too, and lower classes come first among equal ones."""
    print_case("token_logp first class", n=n, dtype=dtype)
    r = np.random.default_rng(n)
    z = r.normal(size=(6, n)).astype(np.float32)
    z[0, 0] = np.nan
    z[1] = np.nan
    z[2, [0, n // 2, n - 1]] = np.nan
    z[3, :] = -np.inf
    z[3, 0] = -np.nan
    z[4, 0] = np.inf
    z[4, 1] = np.nan
    c = Case(dtype, 6, n, 0, 0, 6, False, None, z=z)
    c.fwd()
    torch.cuda.synchronize()
    f = L.forward(c.z, None, 6)
    assert np.array_equal(c.d["top_ids"].cpu().numpy(), f["top_ids"])
    assert np.array_equal(torch.isnan(c.d["top_values"]).cpu().numpy(), np.isnan(f["top_values"]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [200, 2000, 50001])
@pytest.mark.parametrize("lead", [15, 22, 25, 28, 40])
def test_gradient_of_sure_rows(lead, n, dtype):
    """dz of a class `lead` ahead of the others: what is left where its own gradient g nearly cancels.
    With t = z - M < 0 of the others, x = exp(t), O = sum x and W = -sum x t: 1 - p = O / (1 + O), H + log p =
    W / (1 + O), so dz = (g O - others - dH W / (1 + O)) / (1 + O), without a difference of near numbers.

    Errors: of O and W as in the oracle's bounds (3 |t| + 5 + 92 roundings of a term), log1p, expm1 and the
    power 4 each, products and sums 8 more, each of its own term; bf16 results are rounded once more."""
    print_case("token_logp sure", lead=lead, n=n, dtype=dtype)
    r = np.random.default_rng(lead + n)
    z = (r.integers(-8, 9, (6, n)) / 8).astype(np.float32)
    z[:, 17] = lead
    z[:, 3] = 1.125                             # the next best
    c = Case(dtype, 6, n, 0, 0, 2, True, None, z=z, targets=[17, 17, 17, 17, -1, -1])
    dl, dh = np.array([1, -1, 1, 0.7, 0, 0], np.float32), np.array([0.5, 0.1, 0, -0.3, 0.25, 0], np.float32)
    dt = np.array([[0, 0], [0, 0], [0, 0.6], [0.9, -0.7], [0, 0], [1, 0.4]], np.float32)
    for k, a in (("dlogp", dl), ("dentropy", dh), ("dtop", dt)):
        c.d[k].copy_(torch.from_numpy(a))
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    got = c.d["dz"][:, 17].double().cpu().numpy()
    t = np.delete(z.astype(np.float64), 17, 1) - lead
    O, W = np.exp(t).sum(1), -(np.exp(t) * t).sum(1)
    ls = np.log1p(O)
    p = 1 / (1 + O)
    g = dl.astype(np.float64) * (np.arange(6) < 4) + dt[:, 0] * p
    others = dt[:, 1] * np.exp(1.125 - lead) * p
    want = p * (g * O - others - dh * W * p)
    rel = (3 * (lead + 1) + 5 + 92 + 12 + 8) * U
    lim = rel * p * (np.abs(g) * O + np.abs(others) + np.abs(dh) * (W * p + 2 * ls))
    if dtype == "bf16":
        lim = lim + L.HALF16 * (np.abs(want) + lim)
    assert np.all(np.abs(got - want) <= lim + L.TINY), (got, want, lim)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [2, 64, 1500, 70000])
def test_small_probabilities(n, dtype):
    """Probabilities of two classes t apart, t to 20 in eighths, the others ruled out: exp(z - M) / S with z - M
    exact.  The power is off by 2 U of itself, the sum by U, its own power (at most 1.4 U, and fix and its product
    1.5) and the quotient by U: 7, and 1 for what these leave out."""
    print_case("token_logp small probabilities", n=n, dtype=dtype)
    t = np.arange(161) / 8.0
    z = np.full((161, n), -np.inf, np.float32)
    z[:, n - 1], z[:, 0] = 0.5, 0.5 - t
    c = Case(dtype, 161, n, 0, 0, 2, True, None, z=z)
    c.fwd()
    torch.cuda.synchronize()
    got, x = c.d["top_values"].double().cpu().numpy(), np.exp(-t)
    want = np.stack([1 / (1 + x), x / (1 + x)], 1)
    far = np.abs(got - want) / (U * want)
    assert np.all(far <= 8), (np.argwhere(far > 8)[:4], far.max())


@pytest.mark.parametrize("n", [8, 1500, 70000])
def test_probabilities_of_special_rows(n):
    z = np.zeros((5, n), np.float32)
    z[0] = -np.inf
    z[1, 3] = np.nan
    z[2, 4] = np.inf
    z[3, 2:] = -np.inf
    z[4, 2] = -3.38e38
    c = Case("f32", 5, n, 0, 0, 8, True, None, z=z)
    c.fwd()
    torch.cuda.synchronize()
    f = L.forward(z, None, 8, True)
    got = c.d["top_values"].double().cpu().numpy()
    assert np.array_equal(c.d["top_ids"].cpu().numpy(), f["top_ids"])
    np.testing.assert_allclose(got, f["top_values"], rtol=8 * U, atol=0)
