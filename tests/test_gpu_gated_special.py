"""Gated FC shard: values that its products' parts do not carry, at sizes that end
inside a tile's pieces."""
import numpy as np
import pytest
import torch

from oracle import gated as G
from paper_2112_15317_amd import sb
from tests.helpers import print_case
from tests.test_gpu_gated import Case

pytestmark = pytest.mark.gpu


def _among_nan(t, lines):
    """t's values with `lines` lines of NaN behind them in the same allocation."""
    w = torch.full((t.shape[0] + lines, t.shape[1]), float("nan"), dtype=t.dtype, device="cuda")
    w[:t.shape[0]] = t
    return w[:t.shape[0]]


# (m, k, n): rows of x that are padded to a multiple of 8 k, weights as they are (n a
# multiple of 8) or packed, one range of k and many; fewer columns than a piece.
ODD_K = [(64, 261, 192), (64, 261, 197), (300, 1859, 741), (40, 3003, 72), (12, 4001, 30), (5, 261, 4),
         (200, 9, 520)]


@pytest.mark.parametrize("what", ["inf", "tiny"])
@pytest.mark.parametrize("m,k,n", ODD_K)
def test_fp32_sums_end_with_the_weights(m, k, n, what):
    """Tiles that are formed again in fp32 take k lines of the weights: NaN in the lines
    behind them and all over the workspace reach no row but x's infinite one."""
    print_case("gated_odd_k", m=m, k=k, n=n, what=what)
    c = Case("sigmoid", "f32", m, k, n, bias=False)
    for t in ("wg", "wu"):
        c.d[t] = _among_nan(c.d[t], 8)
    if what == "inf":
        c.x[1, k // 2] = np.inf
    else:
        c.x *= np.float32(2.0 ** -60)
        c.wu *= np.float32(2.0 ** -58)
    c.d["x"].copy_(torch.from_numpy(c.x))
    c.d["wu"].copy_(torch.from_numpy(c.wu))
    # (Any workspace starts at a multiple of 16 and is whole floats.)
    c.ws[0].view(torch.float32).fill_(float("nan"))
    c.fwd()
    torch.cuda.synchronize()
    y, pre = c.get("y").astype(np.float64), c.d["pre"].cpu().numpy().astype(np.float64)
    x = c.x
    if what == "inf":
        assert not np.isfinite(pre[:, 1]).any()
        x = x.copy()
        x[1] = 0
    rows = np.delete(np.arange(m), 1) if what == "inf" else np.arange(m)
    _, a, u = G.forward("sigmoid", x, c.wg, c.wu)
    # k products and sums of them, each rounded or truncated: (k + 1) steps of the sum of
    # magnitudes, and one of the smallest subnormal value for each.
    for got, want, w in ((pre[0], a, c.wg), (pre[1], u, c.wu)):
        lim = (k + 1) * 2.0 ** -23 * (np.abs(x).astype(np.float64) @ np.abs(w).astype(np.float64)) + 2 * k * 2.0 ** -149
        assert np.all(np.abs(got - want)[rows] <= lim[rows])
    assert np.isfinite(y[rows]).all()
    c.untouched(("y", "pre"))
