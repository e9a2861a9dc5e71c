"""GPU parity of the token log-probabilities (sb_token_logp_fwd, sb_token_logp_bwd)
against oracle/token_logp.py: alternatives' classes to the number, the rest within
bounds of the roundings; one class to many, one row to many, odd sizes and strides,
masks that leave little or nothing, ties, special values, in place, repeated,
captured and concurrent calls."""
import numpy as np
import pytest
import torch

from oracle import token_logp as L
from paper_2112_15317_amd import sb
from tests.helpers import print_case

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": sb.SB_F32, "bf16": sb.SB_BF16}
# (rows, classes, extra row stride, elements the tensors start past an allocation, top, probabilities, logits)
SHAPES = [(1, 1, 0, 0, 1, False, "normal"), (3, 2, 1, 1, 2, True, "normal"), (70, 8, 0, 0, 8, True, "normal"),
          (33, 64, 0, 0, 8, True, "masked"), (65, 127, 1, 0, 32, False, "ties"), (40, 128, 0, 0, 0, False, "sure"),
          (29, 129, 0, 1, 5, True, "masked"), (17, 500, 12, 0, 32, True, "ties"), (9, 1024, 0, 0, 8, True, "normal"),
          (7, 1025, 0, 0, 8, False, "normal"), (5, 1100, 3, 3, 32, False, "masked"), (1, 32000, 0, 0, 5, False, "normal"),
          (3, 50001, 7, 1, 32, False, "masked"), (2, 4096, 0, 0, 20, True, "equal"), (6, 4097, 0, 0, 32, False, "ties"),
          (530, 5000, 0, 0, 3, False, "sure"), (1100, 4200, 0, 1, 0, False, "masked"), (2, 300000, 0, 0, 32, False, "ties"),
          (1, 1 << 20, 0, 0, 9, False, "normal"), (8, 2500, 0, 0, 32, False, "rising"), (4, 33000, 0, 0, 32, False, "falling"),
          (65, 128, 0, 0, 8, True, "close"), (13, 700, 3, 1, 32, False, "close"), (6, 6000, 0, 0, 20, False, "close"),
          (9, 30, 0, 0, 29, True, "close"), (4100, 1040, 8, 0, 2, True, "normal"), (1300, 9000, 0, 0, 32, False, "wide")]


def _logits(kind, r, m, n):
    z = r.normal(size=(m, n)) * 2
    if kind == "masked":                        # few classes are left, in some rows one or none
        z[r.uniform(size=(m, n)) < 0.9] = -np.inf
        z[::7] = -np.inf
        z[::14, n // 2] = 1.5
    elif kind == "ties":                        # a handful of values, both zeros among them
        z = np.round(z) * np.where(r.uniform(size=(m, n)) < 0.5, 1.0, -1.0)
    elif kind == "equal":
        z[:] = -3.25
    elif kind == "sure":
        z[np.arange(m), r.integers(0, n, m)] += 30.0
    elif kind == "rising":
        z = np.linspace(-5, 5, n) + np.zeros((m, 1))
    elif kind == "falling":
        z = np.linspace(5, -5, n) + np.zeros((m, 1))
    elif kind == "close":                       # fp32's last bits decide
        z = 1.0 + r.integers(0, 4000, (m, n)) * 2.0 ** -23
    elif kind == "wide":                        # the type's ends as masks
        z[:, ::3] = -3.38e38
        z[::5] -= 60.0
        z[1::5] += 60.0
    return z.astype(np.float32)


class Case:
    """Inputs on the host, their device copies inside larger allocations, and
    outputs that start out as 77."""

    def __init__(self, dtype, m, n, stride, shift, top, probs, kind, seed=0, z=None, targets=None):
        r = np.random.default_rng(seed + m + 7 * n)
        self.dtype, self.m, self.n, self.top, self.probs, self.shift = dtype, m, n, top, probs, shift
        self.ld = n + stride
        self.z = np.full((m, self.ld), 100.0, np.float32)
        self.z[:, :n] = _logits(kind, r, m, n) if z is None else z
        if dtype == "bf16":
            self.z = torch.from_numpy(self.z).bfloat16().float().numpy()
        self.targets = r.integers(0, n, m).astype(np.int32) if targets is None else np.asarray(targets, np.int32)
        if targets is None:
            self.targets[::2] = np.argmax(self.z[::2, :n], 1)
            self.targets[3::8] = -1
        f = lambda *s: r.normal(size=s).astype(np.float32)
        self.h = {"dlogp": f(m), "dentropy": f(m), "dtop": f(m, top)}
        self.desc = sb.token_logp_desc(m, n, top, CODE[dtype], self.ld, probs)
        self.d = {k: self.put(torch.from_numpy(a)) for k, a in self.h.items()}
        self.d["z"], self.d["targets"] = self.put(torch.from_numpy(self.z).to(TYPES[dtype])), self.put(
            torch.from_numpy(self.targets))
        self.whole = {}
        for k, s, kind in (("logp", (m,), torch.float32), ("entropy", (m,), torch.float32),
                           ("stats", (m, 2), torch.float32), ("top_ids", (m, top), torch.int32),
                           ("top_values", (m, top), torch.float32), ("dz", (m, self.ld), TYPES[dtype])):
            self.whole[k], self.d[k] = self.room(s, kind)
        need = sb.sb_token_logp_workspace_bytes(self.desc)
        self.whole_ws = torch.full((need + 256,), 77, dtype=torch.uint8, device="cuda")
        self.ws = self.whole_ws[:need]

    def room(self, shape, kind):
        size = int(np.prod(shape))
        w = torch.full((size + self.shift + 64,), 77, dtype=kind, device="cuda")
        return w, w[self.shift:self.shift + size].view(shape)

    def put(self, t):
        _, v = self.room(t.shape, t.dtype)
        v.copy_(t)
        return v

    def fwd(self, stream=None, logp=True):
        d = self.d
        t = self.top > 0
        sb.sb_token_logp_fwd(self.desc, d["z"], d["targets"] if logp else None, d["logp"] if logp else None,
                             d["entropy"] if logp else None, d["stats"], d["top_ids"] if t else None,
                             d["top_values"] if t else None, self.ws, stream)

    def bwd(self, logp=True, entropy=True, top=True, place=False, stream=None):
        d = self.d
        top = top and self.top > 0
        sb.sb_token_logp_bwd(self.desc, d["z"], d["stats"], d["targets"] if logp else None,
                             d["dlogp"] if logp else None, d["entropy"] if entropy else None,
                             d["dentropy"] if entropy else None, d["top_ids"] if top else None,
                             d["top_values"] if top else None, d["dtop"] if top else None,
                             d["z"] if place else d["dz"], stream)

    def grads(self, logp=True, entropy=True, top=True):
        h = self.h
        return dict(targets=self.targets, dlogp=h["dlogp"] if logp else None,
                    dentropy=h["dentropy"] if entropy else None,
                    dtop=h["dtop"] if top and self.top else None, probs=self.probs)

    def check(self, names, dz_from="dz", **which):
        torch.cuda.synchronize()
        z = self.z[:, :self.n]
        f = L.forward(z, self.targets, self.top, self.probs)
        g = self.grads(**which)
        lim = L.bounds(z, f, bf16=self.dtype == "bf16", **g)
        ref = dict(f, dz=L.backward(z, f, **g))
        for k in names:
            got = self.d[dz_from if k == "dz" else k].double().cpu().numpy()
            if k == "dz":
                got = got[:, :self.n]
            if k == "top_ids":
                assert np.array_equal(got, f["top_ids"]), np.argwhere(got != f["top_ids"])[:4]
                continue
            if k == "top_values" and not self.top:
                continue
            r = ref[k]
            same = (got == r) | (np.isnan(got) & np.isnan(r))
            with np.errstate(invalid="ignore"):
                ok = same | (np.abs(got - r) <= lim[k])
            assert np.all(ok), (k, np.argwhere(~ok)[:4], got[~ok][:4], r[~ok][:4], lim[k][~ok][:4])

    def untouched(self):
        for k, w in self.whole.items():
            n = self.d[k].numel()
            assert bool((w[:self.shift] == 77).all()) and bool((w[self.shift + n:] == 77).all()), k
        assert bool((self.d["dz"][:, self.n:] == 77).all())
        assert bool((self.whole_ws[len(self.ws):] == 77).all())


FWD = ("stats", "logp", "entropy", "top_values")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_shapes(shape, dtype):
    print_case("token_logp", shape=shape, dtype=dtype)
    c = Case(dtype, *shape)
    c.fwd()
    c.bwd()
    c.check(FWD + (("top_ids",) if c.top else ()) + ("dz",))
    c.untouched()


@pytest.mark.parametrize("which", [dict(logp=True, entropy=False, top=False), dict(logp=False, entropy=True, top=False),
                                   dict(logp=False, entropy=False, top=True), dict(logp=True, entropy=False, top=True),
                                   dict(logp=False, entropy=False, top=False)], ids=lambda w: str(sorted(w.items())))
@pytest.mark.parametrize("shape", [(20, 300, 0, 0, 4, True, "normal"), (20, 3001, 0, 0, 6, True, "normal"),
                                   (20, 3001, 0, 0, 6, False, "masked")], ids=lambda s: "x".join(map(str, s)))
def test_each_gradient_alone(shape, which):
    print_case("token_logp alone", shape=shape, **which)
    c = Case("f32", *shape)
    c.fwd()
    c.bwd(**which)
    if any(which.values()):
        c.check(("dz",), **which)
    else:
        torch.cuda.synchronize()
        assert float(c.d["dz"][:, :c.n].abs().max()) == 0


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", [(50, 200, 0, 0, 8, True, "normal"), (33, 9001, 5, 1, 32, True, "normal"),
                                   (600, 9001, 0, 0, 4, False, "ties")], ids=lambda s: "x".join(map(str, s)))
def test_in_place(shape, dtype):
    print_case("token_logp in place", shape=shape, dtype=dtype)
    c = Case(dtype, *shape)
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    z = c.d["z"].clone()
    c.bwd(place=True)
    torch.cuda.synchronize()
    assert torch.equal(c.d["z"][:, :c.n], c.d["dz"][:, :c.n])
    assert torch.equal(c.d["z"][:, c.n:], z[:, c.n:])


@pytest.mark.parametrize("n", [90, 1024, 1025, 20000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_special_rows(n, dtype):
    """Rows of -inf alone, with one class left, with NaN of both signs, +inf, the type's ends, targets past the classes."""
    print_case("token_logp special", n=n, dtype=dtype)
    r = np.random.default_rng(n)
    z = r.normal(size=(12, n)).astype(np.float32)
    z[0] = -np.inf
    z[1] = -np.inf
    z[1, n - 1] = 4.0
    z[2, n // 3] = np.nan
    z[3, n - 1] = -np.nan
    z[4, 5] = np.inf
    z[5, 1:] = -3.38e38
    z[6] = -3.38e38
    z[7, 3:] = 0.0
    z[7, 3::2] = -0.0
    z[8, :] = -np.inf
    z[8, 7] = np.nan
    z[9, 5] = z[9, n - 2] = np.inf
    z = np.concatenate([z, np.full((2, n), 3.38e38, np.float32)])      # all the same, and largest but one half
    z[13, ::2] = 1e30
    t = np.array([3, n - 1, 4, 5, 5, 0, 9, -1, 2, 5, n, 2 ** 31 - 1, 8, 1])
    c = Case(dtype, 14, n, 0, 0, 6, False, None, z=z, targets=t)
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    f = L.forward(c.z, t, 6)
    assert np.array_equal(c.d["top_ids"].cpu().numpy(), f["top_ids"])
    dz = L.backward(c.z, f, t, c.h["dlogp"], c.h["dentropy"], c.h["dtop"])
    for k, ref in (("logp", f["logp"]), ("entropy", f["entropy"]), ("top_values", f["top_values"]), ("dz", dz)):
        got = c.d[k].double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(ref)), (k, np.argwhere(np.isnan(got) != np.isnan(ref))[:4])
        assert np.array_equal(got == -np.inf, ref == -np.inf), k
    # What is finite in those rows is as everywhere.
    keep = [0, 1, 5, 6, 7, 12, 13]
    s = Case(dtype, 7, n, 0, 0, 6, False, None, z=z[keep], targets=t[keep])
    s.fwd()
    s.bwd()
    s.check(FWD + ("top_ids", "dz"))
    assert float(s.d["dz"][0].abs().max()) == 0


def test_sure_rows_keep_their_bits():
    """A token 30 ahead of 1999 others: log p = -1999 exp(-30), not 0; to a few steps of fp32."""
    z = np.zeros((4, 2000), np.float32)
    z[:, 17] = 30.0
    c = Case("f32", 4, 2000, 0, 0, 1, False, None, z=z, targets=[17] * 4)
    c.fwd()
    torch.cuda.synchronize()
    want = -np.log1p(1999 * np.exp(-30.0))
    # 3 * 30 + 2 + 92 roundings of a term and 4 of log1p, as in the oracle's bounds.
    assert abs(float(c.d["logp"][0]) - want) <= 200 * 2.0 ** -24 * abs(want)


@pytest.mark.parametrize("shape", [(40, 256, 0, 0, 8, True, "normal"), (300, 12000, 0, 0, 8, False, "ties")],
                         ids=["short rows", "long rows"])
def test_repeats_streams_and_graphs_agree(shape):
    outs = FWD + ("top_ids", "dz")
    c, d = Case("bf16", *shape), Case("bf16", *shape, seed=3)
    d.ws = c.ws
    want = []
    for x in (c, d):
        x.fwd()
        x.bwd()
        torch.cuda.synchronize()
        want.append([x.d[k].clone() for k in outs])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c.fwd()
        c.bwd()
    side.synchronize()
    assert all(torch.equal(c.d[k], w) for k, w in zip(outs, want[0]))
    graphs = []
    for x in (c, d):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.fwd()
            x.bwd()
        graphs.append(g)
    for turn in range(3):
        for x, g, w in zip((c, d), graphs, want):
            for k in outs:
                x.d[k].fill_(turn)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x.d[k], t) for k, t in zip(outs, w))


def test_calls_at_once_on_their_own_workspaces():
    cases = [Case("f32", 200, 6000, 0, 0, 5, False, "normal", seed=i) for i in range(3)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for c, s in zip(cases, streams):
        for _ in range(3):
            c.fwd(stream=s)
            c.bwd(stream=s)
    for c in cases:
        c.check(FWD + ("top_ids", "dz"))


def test_without_targets_and_alternatives():
    c = Case("bf16", 10, 7000, 0, 0, 0, False, "normal")
    c.fwd(logp=False)
    c.check(("stats",))
    assert bool((c.d["logp"] == 77).all()) and bool((c.d["entropy"] == 77).all())


def test_logits_past_32_bits():
    """Rows whose start lies past 2^32 elements."""
    m, n = 3, 1500
    ld = 2 ** 31 - 1
    z = torch.zeros(2 * ld + n, dtype=torch.bfloat16, device="cuda")
    for i in range(m):
        z[i * ld + 700 + i] = 9.0
    t = torch.tensor([700, 701, 702], dtype=torch.int32, device="cuda")
    d = sb.token_logp_desc(m, n, 2, sb.SB_BF16, ld)
    f32 = dict(dtype=torch.float32, device="cuda")
    logp, h, stats, top = (torch.empty(s, **f32) for s in ((m,), (m,), (m, 2), (m, 2)))
    ids = torch.empty((m, 2), dtype=torch.int32, device="cuda")
    ws = torch.empty((sb.sb_token_logp_workspace_bytes(d),), dtype=torch.uint8, device="cuda")
    sb.sb_token_logp_fwd(d, z, t, logp, h, stats, ids, top, ws)
    assert ids.tolist() == [[700, 0], [701, 0], [702, 0]]
    assert float((logp - logp[0]).abs().max()) == 0
    sb.sb_token_logp_bwd(d, z, stats, t, torch.ones(m, **f32), None, None, None, None, None, z)
    # 1 - p of the target, minus the others' probabilities, all rounded to bf16: eps / 2 of each.
    for i in range(m):
        row = z[i * ld:i * ld + n].double()
        p = float(logp[i].double().exp())
        assert abs(float(row[700 + i]) - (1 - p)) <= 2.0 ** -8 * (1 - p) * 1.01
        assert float(row[:700].max()) < 0
    assert float(z[n:ld].abs().max()) == 0
