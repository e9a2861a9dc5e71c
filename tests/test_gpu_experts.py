"""GPU parity of the expert rows (sb_expert_sort, _gather, _combine, _combine_bwd)
against oracle/experts.py: places to the number, rows within bounds of the
roundings; one token to many, one expert for all, experts of other workers, the same
expert twice, odd widths and strides, tensors off any alignment, repeated, captured
and concurrent calls."""
import numpy as np
import pytest
import torch

from oracle import experts as X
from paper_2112_15317_amd import sb
from tests.helpers import print_case

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": sb.SB_F32, "bf16": sb.SB_BF16}
# (tokens, top, experts, all workers' experts, first, width, extra strides, start past an allocation, kind)
SHAPES = [(1, 1, 1, 1, 0, 1, 0, 0, 0, "any"), (1, 2, 8, 8, 0, 1024, 0, 0, 0, "any"),
          (5, 3, 4, 9, 3, 7, 2, 1, 1, "any"), (16, 2, 8, 8, 0, 64, 0, 0, 0, "any"),
          (33, 1, 5, 5, 0, 65, 0, 0, 3, "one"), (70, 2, 3, 9, 6, 130, 4, 0, 0, "any"),
          (100, 4, 6, 12, 3, 512, 0, 8, 0, "none"), (257, 8, 300, 512, 100, 40, 0, 0, 0, "any"),
          (300, 2, 512, 512, 0, 33, 1, 2, 2, "any"), (1365, 3, 11, 22, 11, 741, 0, 0, 0, "any"),
          (2048, 3, 7, 7, 0, 16, 0, 0, 0, "twice"), (2049, 3, 8, 8, 0, 24, 0, 0, 0, "any"),
          (30000, 3, 40, 60, 0, 9, 0, 0, 1, "any"), (90000, 3, 2, 2, 0, 4, 0, 0, 0, "twice"),
          (60, 5, 6, 6, 0, 4200, 8, 0, 0, "any"), (40, 12, 16, 16, 0, 2049, 0, 0, 0, "any")]


def _ids(kind, r, n, top, whole):
    if kind == "one":
        return np.full((n, top), whole // 2)
    if kind == "none":                          # of other workers, or of none
        return r.choice([-1, -2 ** 31, 2 ** 31 - 1, 0], (n, top))
    if kind == "twice":                         # a token may choose an expert more than once
        return r.integers(0, whole, (n, top))
    return np.argsort(r.uniform(size=(n, whole)), axis=1)[:, :top]


class Case:
    def __init__(self, dtype, n, top, experts, whole, first, width, xs, rs, shift, kind, seed=0):
        r = np.random.default_rng(seed + n + 7 * top + 31 * width)
        self.dtype, self.n, self.top, self.experts, self.first, self.width = dtype, n, top, experts, first, width
        self.ldx, self.ldr, self.shift = width + xs, width + rs, shift
        f = lambda *s: r.normal(size=s).astype(np.float32)
        self.ids = _ids(kind, r, n, top, whole).astype(np.int32)
        self.h = {"x": f(n, self.ldx), "dy": f(n, self.ldx), "ys": f(n * top, self.ldr), "dxs": f(n * top, self.ldr)}
        self.weights = r.uniform(size=(n, top)).astype(np.float32)
        if dtype == "bf16":
            self.h = {k: torch.from_numpy(a).bfloat16().float().numpy() for k, a in self.h.items()}
        self.desc = sb.expert_desc(n, top, experts, width, CODE[dtype], first, self.ldx, self.ldr)
        self.d = {k: self.put(torch.from_numpy(a).to(TYPES[dtype])) for k, a in self.h.items()}
        self.d["ids"] = self.put(torch.from_numpy(self.ids))
        self.d["weights"] = self.put(torch.from_numpy(self.weights))
        self.whole = {}
        for k, shape, kind in (("place", (n, top), torch.int32), ("offsets", (experts + 1,), torch.int32),
                               ("xs", (n * top, self.ldr), TYPES[dtype]), ("y", (n, self.ldx), TYPES[dtype]),
                               ("dys", (n * top, self.ldr), TYPES[dtype]), ("dx", (n, self.ldx), TYPES[dtype]),
                               ("dweights", (n, top), torch.float32)):
            self.whole[k], self.d[k] = self.room(shape, kind)
        need = sb.sb_expert_workspace_bytes(self.desc)
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

    def run(self, stream=None, weights=True):
        d = self.d
        w = d["weights"] if weights else None
        sb.sb_expert_sort(self.desc, d["ids"], d["place"], d["offsets"], self.ws, stream)
        sb.sb_expert_gather(self.desc, d["x"], d["place"], d["xs"], stream)
        sb.sb_expert_combine(self.desc, d["ys"], d["place"], w, d["y"], stream=stream)
        sb.sb_expert_combine_bwd(self.desc, d["dy"], d["ys"], d["place"], w, d["dys"], d["dweights"], stream)
        sb.sb_expert_combine(self.desc, d["dxs"], d["place"], None, d["dx"], stream=stream)

    def get(self, k):
        return self.d[k].double().cpu().numpy()[:, :self.width]

    def check(self, weights=True):
        torch.cuda.synchronize()
        w = self.weights if weights else None
        bf16 = self.dtype == "bf16"
        place, offsets = X.sort(self.ids, self.first, self.experts)
        assert np.array_equal(self.d["place"].cpu().numpy(), place)
        assert np.array_equal(self.d["offsets"].cpu().numpy(), offsets)
        x, dy, ys, dxs = (self.h[k][:, :self.width] for k in ("x", "dy", "ys", "dxs"))
        rows = np.full((self.n * self.top, self.width), 77.0)       # behind the last one: as they were
        assert np.array_equal(self.get("xs"), X.gather(x, place, rows))
        ey, edys, edw = X.bounds(dy, ys, place, w, rows, bf16)
        dys, dw = X.combine_backward(dy, ys, place, w, rows)
        edx = X.bounds(dy, dxs, place, None, rows, bf16)[0]
        for k, ref, lim in (("y", X.combine(ys, place, w), ey), ("dys", dys, edys), ("dx", X.combine(dxs, place), edx)):
            far = np.abs(self.get(k) - ref)
            assert np.all(far <= lim), (k, np.argwhere(~(far <= lim))[:4])
        assert np.all(np.abs(self.d["dweights"].double().cpu().numpy() - dw) <= edw)

    def untouched(self):
        for k, w in self.whole.items():
            n = self.d[k].numel()
            assert bool((w[:self.shift] == 77).all()) and bool((w[self.shift + n:] == 77).all()), k
        for k in ("xs", "y", "dys", "dx"):
            assert bool((self.d[k][:, self.width:] == 77).all()), k
        assert bool((self.whole_ws[len(self.ws):] == 77).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_shapes(shape, dtype):
    print_case("experts", shape=shape, dtype=dtype)
    c = Case(dtype, *shape)
    c.run()
    c.check()
    c.untouched()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_combining_on_top_of_rows(dtype):
    c = Case(dtype, *SHAPES[5])
    c.run()
    place, _ = X.sort(c.ids, c.first, c.experts)
    add, ys = c.h["dy"][:, :c.width], c.h["ys"][:, :c.width]
    ref = X.combine(ys, place, c.weights, add)
    lim = X.bounds(add, ys, place, c.weights, ys, dtype == "bf16", add)[0]
    sb.sb_expert_combine(c.desc, c.d["ys"], c.d["place"], c.d["weights"], c.d["y"], c.d["dy"])
    assert np.all(np.abs(c.get("y") - ref) <= lim)
    c.untouched()
    there = c.d["dy"].clone()                       # in place: what lies between the rows stays
    sb.sb_expert_combine(c.desc, c.d["ys"], c.d["place"], c.d["weights"], there, there)
    assert torch.equal(there[:, :c.width], c.d["y"][:, :c.width])
    assert torch.equal(there[:, c.width:], c.d["dy"][:, c.width:])


def test_without_weights_and_without_their_gradient():
    c = Case("bf16", *SHAPES[5])
    c.run(weights=False)
    c.check(weights=False)
    c.d["dys"].fill_(77)
    dys = c.d["dys"].clone()
    sb.sb_expert_combine_bwd(c.desc, c.d["dy"], None, c.d["place"], c.d["weights"], c.d["dys"], None)
    sb.sb_expert_combine_bwd(c.desc, c.d["dy"], c.d["ys"], c.d["place"], c.d["weights"], dys, c.d["dweights"])
    assert torch.equal(c.d["dys"], dys)


def test_a_batch_without_tokens_has_no_rows():
    d = sb.expert_desc(0, 2, 6, 8)
    offsets = torch.full((8,), 77, dtype=torch.int32, device="cuda")
    sb.sb_expert_sort(d, None, None, offsets[:7])
    assert offsets.tolist() == [0] * 7 + [77]


def test_places_out_of_range_are_none():
    """Whatever stands in `place`, no row outside the buffers is touched."""
    c = Case("f32", 20, 2, 4, 4, 0, 10, 0, 0, 0, "any")
    c.run()
    place = c.d["place"]
    place[3, 0], place[5, 1], place[7, 0] = 40, -2 ** 31, 2 ** 31 - 1
    kept = place.cpu().numpy().copy()
    kept[(kept < 0) | (kept >= 40)] = -1
    sb.sb_expert_combine(c.desc, c.d["ys"], place, c.d["weights"], c.d["y"])
    sb.sb_expert_gather(c.desc, c.d["x"], place, c.d["xs"])
    sb.sb_expert_combine_bwd(c.desc, c.d["dy"], c.d["ys"], place, c.d["weights"], c.d["dys"], c.d["dweights"])
    ey = X.bounds(c.h["dy"], c.h["ys"], kept, c.weights, c.h["ys"], False)[0]
    assert np.all(np.abs(c.get("y") - X.combine(c.h["ys"], kept, c.weights)) <= ey)
    assert float(c.d["dweights"][3, 0]) == 0 and float(c.d["dweights"][7, 0]) == 0
    c.untouched()


def test_special_values_stay_with_their_token():
    c = Case("bf16", 50, 2, 5, 5, 0, 66, 0, 0, 0, "any")
    place, _ = X.sort(c.ids, 0, 5)
    c.d["ys"][place[7, 1], 3] = float("nan")
    c.d["ys"][place[9, 0], 65] = float("inf")
    c.run()
    bad = ~torch.isfinite(c.d["y"].float())
    assert bool(bad[7, 3]) and bool(bad[9, 65]) and int(bad.sum()) == 2
    badw = ~torch.isfinite(c.d["dweights"])
    assert bool(badw[7, 1]) and bool(badw[9, 0]) and int(badw.sum()) == 2


@pytest.mark.parametrize("shape", [SHAPES[9], SHAPES[12]], ids=["one launch", "many tiles"])
def test_repeats_streams_and_graphs_agree(shape):
    outs = ("place", "offsets", "xs", "y", "dys", "dx", "dweights")
    c, d = Case("bf16", *shape), Case("bf16", *shape, seed=5)
    d.ws = c.ws
    want = []
    for x in (c, d):
        x.run()
        torch.cuda.synchronize()
        want.append([x.d[k].clone() for k in outs])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c.run()
    side.synchronize()
    assert all(torch.equal(c.d[k], w) for k, w in zip(outs, want[0]))
    graphs = []
    for x in (c, d):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.run()
        graphs.append(g)
    for turn in range(3):
        for x, g, w in zip((c, d), graphs, want):
            for k in outs:
                if k not in ("xs", "dys"):
                    x.d[k].fill_(turn)
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x.d[k], t) for k, t in zip(outs, w))
    c.d["ids"].copy_(d.d["ids"])
    c.d["xs"].fill_(77)
    c.d["dys"].fill_(77)
    c.ids = d.ids
    graphs[0].replay()
    c.check()


def test_calls_at_once_on_their_own_workspaces():
    cases = [Case("f32", 9000, 2, 16, 16, 0, 32, 0, 0, 0, "any", seed=i) for i in range(3)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for c, s in zip(cases, streams):
        for _ in range(3):
            c.run(stream=s)
    for c in cases:
        c.check()


def test_rows_past_32_bits():
    """Sorted rows beyond 2^32 elements of the buffer."""
    n, width = 3, 16
    d = sb.expert_desc(n, 1, 2, width, sb.SB_BF16, ldr=2 ** 31 - 1)
    rows = torch.zeros(2 * (2 ** 31 - 1) + width, dtype=torch.bfloat16, device="cuda")
    x = torch.arange(n * width, device="cuda").view(n, width).to(torch.bfloat16)
    ids = torch.tensor([[1], [0], [1]], dtype=torch.int32, device="cuda")
    place, offsets = torch.empty_like(ids), torch.empty(3, dtype=torch.int32, device="cuda")
    sb.sb_expert_sort(d, ids, place, offsets)
    assert place.flatten().tolist() == [1, 0, 2] and offsets.tolist() == [0, 1, 3]
    sb.sb_expert_gather(d, x, place, rows)
    y = torch.empty_like(x)
    sb.sb_expert_combine(d, rows, place, None, y)
    assert torch.equal(x, y) and torch.equal(rows[-width:], x[2])
