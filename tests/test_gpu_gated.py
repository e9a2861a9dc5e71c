"""GPU parity of the gated FC shard (sb_gated_shard_fwd, sb_gated_shard_bwd)
against oracle/gated.py, element by element within bounds of the roundings:
one row to many, odd sizes, row strides, views off any alignment, missing
biases, accumulation, special values, captured and concurrent calls."""
import numpy as np
import pytest
import torch

from oracle import gated as G
from paper_2112_15317_amd import sb
from tests.helpers import print_case

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": sb.SB_F32, "bf16": sb.SB_BF16}
ACT = {name: i for i, name in enumerate(G.ACTS)}
# (m, k, n, extra row stride of x, of y, elements the tensors start past an allocation)
SHAPES = [(1, 1, 1, 0, 0, 0), (1, 64, 64, 0, 0, 0), (3, 5, 7, 0, 0, 0), (2, 200, 33, 3, 1, 1),
          (8, 130, 264, 6, 0, 0), (7, 513, 70, 0, 2, 1), (9, 100, 72, 4, 0, 0), (4, 1024, 1000, 0, 0, 0),
          (64, 64, 64, 0, 0, 0), (127, 66, 130, 0, 0, 0), (200, 300, 129, 4, 7, 1),
          (65, 1030, 258, 2, 2, 2), (256, 256, 256, 0, 0, 0), (333, 512, 320, 64, 64, 0),
          (129, 2048, 96, 8, 0, 8), (520, 72, 640, 0, 8, 0), (1100, 160, 200, 0, 0, 0),
          (16, 1024, 512, 0, 0, 0), (768, 264, 512, 0, 0, 4)]


class Case:
    """Inputs on the host, their device copies inside larger allocations, and
    outputs that start out as 77."""

    def __init__(self, act, dtype, m, k, n, xs=0, ys=0, shift=0, bias=True, seed=0):
        r = np.random.default_rng(seed + m + 7 * k + 31 * n)
        f = lambda *s, std=1.0: (r.normal(size=s) * std).astype(np.float32)
        self.act, self.dtype, self.m, self.k, self.n, self.shift = act, dtype, m, k, n, shift
        self.ldx, self.ldy = k + xs, n + ys
        self.x, self.dy = f(m, self.ldx), f(m, self.ldy)
        self.wg, self.wu = f(k, n, std=k ** -0.5), f(k, n, std=k ** -0.5)
        self.bg, self.bu = (f(n, std=0.3), f(n, std=0.3)) if bias else (None, None)
        if dtype == "bf16":
            for t in ("x", "dy", "wg", "wu"):
                setattr(self, t, torch.from_numpy(getattr(self, t)).bfloat16().float().numpy())
        self.desc = sb.gated_desc(m, k, n, CODE[dtype], ACT[act], self.ldx, self.ldy,
                                  unaligned=shift % 8 != 0)
        self.d = {t: self.put(getattr(self, t)) for t in ("x", "dy", "wg", "wu")}
        self.d.update({t: None if getattr(self, t) is None else self.put(getattr(self, t), "f32")
                       for t in ("bg", "bu")})
        need = [sb.sb_gated_workspace_bytes(self.desc, p) for p in (sb.SB_FC_FWD, sb.SB_FC_BWD)]
        # Workspaces of exactly the size asked for, with marked bytes behind.
        self.whole_ws = [torch.full((b + 256,), 77, dtype=torch.uint8, device="cuda") for b in need]
        self.ws = [w[:b] for w, b in zip(self.whole_ws, need)]
        self.whole = {}
        for t, shape, kind in (("y", (m, self.ldy), dtype), ("dx", (m, self.ldx), dtype),
                               ("pre", (2, m, n), "f32"), ("dwg", (k, n), "f32"),
                               ("dwu", (k, n), "f32"), ("dbg", (n,), "f32"), ("dbu", (n,), "f32")):
            size = int(np.prod(shape))
            w = torch.full((size + shift + 64,), 77.0, dtype=TYPES[kind], device="cuda")
            self.whole[t] = w
            self.d[t] = w[shift:shift + size].view(shape)

    def put(self, a, dtype=None):
        t = torch.from_numpy(np.ascontiguousarray(a)).to(TYPES[dtype or self.dtype])
        w = torch.full((t.numel() + self.shift + 64,), float("nan"), dtype=t.dtype, device="cuda")
        v = w[self.shift:self.shift + t.numel()].view(t.shape)
        v.copy_(t)
        return v

    def fwd(self, pre=True, stream=None):
        d = self.d
        sb.sb_gated_shard_fwd(self.desc, d["x"], d["wg"], d["wu"], d["bg"], d["bu"], d["y"],
                              d["pre"] if pre else None, self.ws[0], stream)

    def bwd(self, accumulate=False, dx=True, db=True, stream=None):
        d = self.d
        sb.sb_gated_shard_bwd(self.desc, d["x"], d["wg"], d["wu"], d["pre"], d["dy"],
                              d["dx"] if dx else None, d["dwg"], d["dwu"], d["dbg"] if db else None,
                              d["dbu"] if db else None, accumulate, self.ws[1], stream)

    def ref(self):
        x, dy = self.x[:, :self.k], self.dy[:, :self.n]
        y, a, u = G.forward(self.act, x, self.wg, self.wu, self.bg, self.bu)
        return dict(zip(("y", "dx", "dwg", "dwu", "dbg", "dbu"),
                        (y,) + G.backward(self.act, x, self.wg, self.wu, a, u, dy)))

    def bound(self):
        return dict(zip(("y", "dx", "dwg", "dwu", "dbg", "dbu"),
                        G.bounds(self.act, self.x[:, :self.k], self.wg, self.wu, self.bg, self.bu,
                                 self.dy[:, :self.n], self.dtype == "bf16")))

    def get(self, t):
        a = self.d[t].float().cpu().numpy()
        return a[:, :self.n] if t == "y" else a[:, :self.k] if t == "dx" else a

    def check(self, names, base=0.0):
        torch.cuda.synchronize()
        ref, bound = self.ref(), self.bound()
        for t in names:
            got = self.get(t).astype(np.float64)
            far = np.abs(got - base * (t[:2] in ("dw", "db")) - ref[t])
            lim = bound[t] + base * 2.0 ** -23 * (np.abs(ref[t]) + base)
            assert np.all(far <= lim), (t, float(np.nanmax(far / lim)), np.argwhere(~(far <= lim))[:4])

    def untouched(self, names):
        """What lies around the outputs, between their rows and behind the workspaces."""
        for t in names:
            w, n = self.whole[t], self.d[t].numel()
            assert bool((w[:self.shift] == 77).all()) and bool((w[self.shift + n:] == 77).all()), t
        for t, width in (("y", self.n), ("dx", self.k)):
            if t in names:
                assert bool((self.d[t][:, width:] == 77).all()), t
        for w, v in zip(self.whole_ws, self.ws):
            assert bool((w[len(v):] == 77).all())


ALL = ("y", "dx", "dwg", "dwu", "dbg", "dbu")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_shapes(shape, dtype):
    print_case("gated", shape=shape, dtype=dtype)
    act = G.ACTS[(shape[0] + shape[1]) % 5]
    c = Case(act, dtype, *shape)
    c.fwd()
    c.bwd()
    c.check(ALL)
    c.untouched(ALL + ("pre",))
    # Without pre (inference), and again: the same bits.
    y, grads = c.d["y"].clone(), [c.d[t].clone() for t in ALL[1:]]
    c.d["y"].fill_(0)
    c.fwd(pre=False)
    c.bwd()
    torch.cuda.synchronize()
    assert torch.equal(c.d["y"][:, :c.n], y[:, :c.n])
    for t, g in zip(ALL[1:], grads):
        assert torch.equal(c.d[t], g), t


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", G.ACTS)
@pytest.mark.parametrize("bias", [False, True])
def test_activations(act, dtype, bias):
    print_case("gated_act", act=act, dtype=dtype, bias=bias)
    c = Case(act, dtype, 96, 200, 160, bias=bias)
    c.fwd()
    c.bwd()
    c.check(ALL)
    torch.cuda.synchronize()
    a = c.d["pre"].cpu().numpy()
    _, ra, ru = G.forward(act, c.x, c.wg, c.wu, c.bg, c.bu)
    assert np.allclose(a[0], ra, atol=1e-4) and np.allclose(a[1], ru, atol=1e-4)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_accumulated_and_skipped_gradients(dtype):
    print_case("gated_accumulate", dtype=dtype)
    c = Case("silu", dtype, 150, 136, 72)
    c.fwd()
    c.bwd(dx=False, db=False)
    c.check(("y", "dwg", "dwu"))
    for t in ("dx", "dbg", "dbu"):
        assert bool((c.whole[t] == 77).all())
    for t in ("dwg", "dwu", "dbg", "dbu"):
        c.d[t].fill_(3.0)
    c.bwd(accumulate=True)
    c.check(ALL, base=3.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m", [64, 700])
def test_special_values_stay_in_their_rows_and_columns(dtype, m):
    """An infinity or NaN in row i of x reaches row i of y alone (one in column j
    of a weight, column j), and the rest is what it is without."""
    print_case("gated_special", dtype=dtype, m=m)
    c = Case("sigmoid", dtype, m, 264, 192, bias=False)
    c.x[5, 7], c.x[m - 2, 100] = np.inf, np.nan
    c.wu[11, 50] = np.inf
    c.d["x"].copy_(torch.from_numpy(c.x))
    c.d["wu"].copy_(torch.from_numpy(c.wu))
    c.fwd()
    torch.cuda.synchronize()
    with np.errstate(all="ignore"):
        ref = c.ref()["y"]
    got = c.get("y")
    assert np.isnan(got[m - 2]).all() and not np.isfinite(got[5]).any()
    rows, cols = np.delete(np.arange(m), [5, m - 2]), np.delete(np.arange(192), 50)
    assert np.array_equal(got[rows, 50], ref[rows, 50])            # infinities, by sign
    # The rest against the bounds of finite inputs.
    c.x[[5, m - 2]] = 0
    c.wu[:, 50] = 0
    ok = np.ix_(rows, cols)
    assert np.all(np.abs(got[ok] - c.ref()["y"][ok]) <= c.bound()["y"][ok])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_special_gradients(dtype):
    print_case("gated_special_bwd", dtype=dtype)
    m, k, n = 70, 136, 130
    c = Case("silu", dtype, m, k, n)
    c.fwd()
    c.dy[4, 9] = np.inf
    c.d["dy"].copy_(torch.from_numpy(c.dy))
    c.bwd()
    torch.cuda.synchronize()
    assert not np.isfinite(c.get("dx")[4]).any()
    for t in ("dwg", "dwu", "dbg", "dbu"):
        g = c.get(t)
        bad = ~np.isfinite(g)
        assert bad[..., 9].all() and not np.delete(bad, 9, axis=-1).any(), t
    # The sign of an infinite sum is the sign of the infinite term.
    with np.errstate(all="ignore"):
        ref = c.ref()
    assert np.array_equal(c.get("dwu")[:, 9], ref["dwu"][:, 9])
    assert np.isfinite(np.delete(c.get("dx"), 4, axis=0)).all()


def test_tiny_fp32_values():
    """Operands whose lower parts bf16 cannot hold: the fp32 products still can."""
    print_case("gated_tiny")
    c = Case("sigmoid", "f32", 40, 96, 64, bias=False)
    c.x *= np.float32(2.0 ** -60)
    c.wu *= np.float32(2.0 ** -58)
    c.d["x"].copy_(torch.from_numpy(c.x))
    c.d["wu"].copy_(torch.from_numpy(c.wu))
    c.fwd()
    torch.cuda.synchronize()
    ref = c.ref()["y"]
    got = c.get("y").astype(np.float64)
    assert np.all(np.abs(got - ref) <= 1e-5 * np.abs(ref) + 1e-5 * np.abs(c.x).astype(np.float64) @ np.abs(c.wu))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_captured_and_concurrent_calls(dtype):
    """A captured forward and backward replayed over new inputs, with eager work
    between the replays; two streams at once with a workspace each."""
    print_case("gated_graph", dtype=dtype)
    c, e = (Case("gelu", dtype, 300, 192, 256, seed=s) for s in (1, 1))
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.fwd()
        c.bwd()
    for step in range(4):
        for t in ("x", "dy"):
            new = torch.randn(c.d[t].shape, device="cuda").to(TYPES[dtype])
            c.d[t].copy_(new)
            e.d[t].copy_(new)
        graph.replay()
        e.fwd()
        e.bwd()
        torch.cuda.synchronize()
        for t in ALL:
            assert torch.equal(c.d[t], e.d[t]), (step, t)
    want = {t: c.d[t].clone() for t in ALL}
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for s, case in zip(streams, (c, e)):
        case.fwd(stream=s)
        case.bwd(stream=s)
    torch.cuda.synchronize()
    for case in (c, e):
        for t in ALL:
            assert torch.equal(case.d[t], want[t]), t


# Shapes whose products take the 256-row tiles, unsplit and split over the reduction,
# with tails in all three dimensions: (m, k, n), whether dx is asked for.
WIDE = [(2829, 205, 2139, True), (410, 1830, 4144, True), (314, 1173, 3339, False),
        (604, 414, 4212, False), (539, 5700, 854, True), (4010, 907, 968, True),
        (431, 1922, 2534, True), (3771, 203, 5514, True)]


@pytest.mark.parametrize("shape", WIDE, ids=lambda s: "x".join(map(str, s[:3])))
def test_wide_tiles(shape):
    print_case("gated_wide", shape=shape)
    c = Case("silu", "bf16", *shape[:3], xs=2, ys=1)
    c.fwd()
    c.bwd(dx=shape[3])
    names = ALL if shape[3] else tuple(t for t in ALL if t != "dx")
    c.check(names)
    c.untouched(names + ("pre",))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(9, 4000, 30), (300, 2000, 70), (520, 300, 40), (64, 64, 4000),
                                   (3000, 72, 72)], ids=lambda s: "x".join(map(str, s)))
def test_many_splits(shape, dtype):
    """Small outputs of long reductions: up to 63 splits, joined by four waves."""
    print_case("gated_splits", shape=shape, dtype=dtype)
    c = Case("gelu", dtype, *shape)
    c.fwd()
    c.bwd()
    c.check(ALL)
    c.bwd(dx=False)
    c.check(tuple(t for t in ALL if t != "dx"))
    c.untouched(ALL + ("pre",))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m", [1, 3, 8, 9, 100, 520])
@pytest.mark.parametrize("stride", [8, 5])
def test_what_lies_between_the_rows_is_not_read(m, stride, dtype):
    """NaN between the rows of x and dy, at strides that are taken as they are and
    at such that are laid out anew."""
    print_case("gated_between", m=m, stride=stride, dtype=dtype)
    c = Case("gelu_tanh", dtype, m, 136, 72, xs=stride, ys=stride)
    c.d["x"][:, c.k:] = float("nan")
    c.d["dy"][:, c.n:] = float("nan")
    c.fwd()
    c.bwd()
    c.check(ALL)
    c.bwd(dx=False, db=False)
    c.check(("dwg", "dwu"))
    c.untouched(ALL + ("pre",))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_special_values_of_few_rows(dtype):
    print_case("gated_special_few", dtype=dtype)
    c = Case("sigmoid", dtype, 5, 264, 100, bias=False)
    c.x[1, 7], c.x[3, 100] = np.inf, np.nan
    c.d["x"].copy_(torch.from_numpy(c.x))
    c.fwd()
    c.dy[4, 9] = np.nan
    c.d["dy"].copy_(torch.from_numpy(c.dy))
    torch.cuda.synchronize()
    got = c.get("y")
    assert np.isnan(got[3]).all() and not np.isfinite(got[1]).any()
    c.x[[1, 3]] = 0
    rest = [0, 2, 4]
    c.dy[4, 9] = 0
    assert np.all(np.abs(got[rest] - c.ref()["y"][rest]) <= c.bound()["y"][rest])
    c.d["x"].copy_(torch.from_numpy(c.x))
    c.fwd()                                                # a finite pre
    c.bwd()
    torch.cuda.synchronize()
    dx = c.get("dx")
    assert np.isnan(dx[4]).all()
    ok = slice(0, 4)
    assert np.all(np.abs(dx[ok] - c.ref()["dx"][ok]) <= c.bound()["dx"][ok])
    for t in ("dwg", "dwu", "dbg", "dbu"):
        bad = np.isnan(c.get(t))
        assert bad[..., 9].all() and not np.delete(bad, 9, axis=-1).any(), t


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_two_graphs_with_one_workspace(dtype):
    """Two captured steps that share a workspace, replayed in turn on one stream."""
    print_case("gated_two_graphs", dtype=dtype)
    cases = [Case("silu", dtype, 200, 160, 120, seed=s) for s in (1, 2)]
    cases[1].ws = cases[0].ws
    want, graphs = [], []
    for c in cases:
        c.fwd()
        c.bwd()
        torch.cuda.synchronize()
        want.append({t: c.d[t].clone() for t in ALL})
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.fwd()
            c.bwd()
        graphs.append(g)
    for _ in range(3):
        for c in cases:
            for t in ALL:
                c.d[t].fill_(5)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for c, w in zip(cases, want):
            for t, width in (("y", c.n), ("dx", c.k), ("dwg", c.n), ("dwu", c.n)):
                assert torch.equal(c.d[t][:, :width], w[t][:, :width]), t
            for t in ("dbg", "dbu"):
                assert torch.equal(c.d[t], w[t]), t


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m", [1, 2, 4, 8])
@pytest.mark.parametrize("k,n", [(8, 8), (13, 19), (15, 9), (1030, 70), (4093, 33), (2600, 260), (9, 1000)])
def test_ends_of_few_rows(m, k, n, dtype):
    """Lines and rows that end inside a piece, and infinities in the elements that the
    last two pieces share: both projections are infinite, by sign, where they are in
    float64, and NaN nowhere."""
    print_case("gated_ends", m=m, k=k, n=n, dtype=dtype)
    c = Case("relu", dtype, m, k, n, shift=1)
    c.fwd()
    c.bwd()
    c.check(ALL)
    c.untouched(ALL + ("pre",))
    x, wg = c.x.copy(), c.wg.copy()
    c.x[0, k - 2] = np.inf
    c.wg[max(k - 6, 0), n - 3] = np.inf
    c.d["x"].copy_(torch.from_numpy(c.x))
    c.d["wg"].copy_(torch.from_numpy(c.wg))
    c.fwd()
    torch.cuda.synchronize()
    with np.errstate(all="ignore"):
        _, a, u = G.forward("relu", c.x[:, :k], c.wg, c.wu, c.bg, c.bu)
    got = c.d["pre"].cpu().numpy().astype(np.float64)
    for g, r in zip(got, (a, u)):
        far = ~np.isfinite(r)
        assert far[0].all() and np.array_equal(g[far], r[far], equal_nan=True)
        # The rest: k products and sums, each rounded, of values that x and the weights bound.
        lim = (k + 2) * 2.0 ** -23 * (np.abs(x[:, :k]).astype(np.float64) @ np.maximum(np.abs(wg), np.abs(c.wu)) + 2)
        ok = np.isfinite(r)
        assert np.all(np.abs(g[ok] - r[ok]) <= lim[ok])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,k,n", [(1, 8, 140000), (3, 300, 70001), (8, 70001, 9), (5, 4100, 600)])
def test_long_sides_of_few_rows(m, k, n, dtype):
    """Accumulated gradients of many strips and of many lines a block; without dx."""
    print_case("gated_long", m=m, k=k, n=n, dtype=dtype)
    c = Case("silu", dtype, m, k, n)
    c.fwd()
    c.bwd()
    c.check(ALL)
    for t in ("dwg", "dwu", "dbg", "dbu"):
        c.d[t].fill_(3.0)
    c.d["dx"].fill_(77)
    c.bwd(accumulate=True, dx=False)
    c.check(("dwg", "dwu", "dbg", "dbu"), base=3.0)
    assert bool((c.d["dx"] == 77).all())
    c.untouched(ALL + ("pre",))
