"""AdamW's root on both sides of the eps from which a subnormal second moment counts
for nothing: the hardware's root reads it as 0."""
import numpy as np
import pytest
import torch

from oracle import adamw as A
from paper_2112_15317_amd import sb
from tests.helpers import print_case
from tests.test_gpu_adamw import B1, LR, U

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", [1, 1000])
@pytest.mark.parametrize("beta2", [0.9, 0.999, 0.999999, 1 - 1e-12])
@pytest.mark.parametrize("eps", [1e-12, 1e-11, 1e-10, 1e-9, 1e-8, 1e-5, 1e37])
def test_subnormal_second_moments_beside_eps(eps, beta2, t):
    """The move of w, lr m' / (root + eps), with the 17 half steps that its roundings
    are together, and in v' half a step of the smallest subnormal value for each of
    its three products and sums, of which the root has up to as much again."""
    print_case("adamw_eps", eps=eps, beta2=beta2, t=t)
    n = 2000
    rng = np.random.default_rng(23)
    f = np.float32
    v = (2.0 ** rng.uniform(-145, -100, n)).astype(f)
    m = (2.0 ** rng.uniform(-60, -20, n) * rng.choice([-1, 1], n)).astype(f)
    if eps > 1:
        m *= f(2.0 ** 120)
    w, g = np.zeros(n, f), np.zeros(n, f)
    d = [torch.from_numpy(x).cuda() for x in (w, g, m, v)]
    lst = sb.AdamwList([dict(w=d[0], g=d[1], m=d[2], v=d[3])])
    sb.sb_adamw_update(lst, LR, B1, beta2, eps, step=t)
    got = d[0].cpu().numpy().astype(np.float64)
    rw, _, rv = A.update(w, g, m, v, t, LR, B1, beta2, eps)
    far = np.abs(got - rw)
    # The error of v' in the denominator's terms: of the root, which is its part of it.
    root = np.sqrt(rv / (1 - beta2 ** t))
    lim = 17 * U + 3 * 2.0 ** -150 / (2 * rv) * root / (root + eps)
    assert np.all(far <= lim * np.abs(rw) + 2.0 ** -149)
