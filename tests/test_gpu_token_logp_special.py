"""GPU parity of the token log-probabilities where single numbers decide: logits and
masks of any magnitude, over whole stretches of a row and alone; NaN in a row's first
class.  The shapes reach what tests/test_gpu_token_logp.py leaves: stretches of the
longest and the shortest kind, many blocks of the joining launch."""
import numpy as np
import pytest
import torch

from oracle import token_logp as L
from tests.helpers import print_case
from tests.test_gpu_token_logp import FWD, Case

pytestmark = pytest.mark.gpu

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
