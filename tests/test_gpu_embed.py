"""GPU parity of the embedding shard (sb_embed_fwd, sb_embed_bwd) against
oracle/embed.py within bounds of the roundings: from no token to many, ids that all
agree, are all unlike or lie outside, odd widths, row strides, tensors off any
alignment, accumulation, repeated, captured and concurrent calls."""
import numpy as np
import pytest
import torch

from oracle import embed as E
from paper_2112_15317_amd import sb
from tests.helpers import print_case

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CODE = {"f32": sb.SB_F32, "bf16": sb.SB_BF16}
# (tokens, vocab, width, extra row stride, elements the tensors start past an allocation, kind of ids)
SHAPES = [(0, 7, 5, 0, 0, "any"), (1, 1, 1, 0, 0, "any"), (1, 300, 64, 0, 0, "any"), (3, 5, 7, 2, 1, "any"),
          (8, 1000, 1024, 0, 0, "any"), (9, 4, 129, 3, 3, "one"), (64, 33, 8, 0, 0, "one"), (65, 33, 9, 0, 1, "pad"),
          (128, 700, 65, 0, 1, "zipf"), (129, 700, 65, 0, 0, "zipf"), (128, 9, 2100, 0, 0, "one"),
          (100, 64, 130, 0, 3, "out"), (5000, 30000, 300, 0, 0, "zipf"), (6000, 8000, 1030, 0, 0, "far"),
          (16384, 700, 33, 0, 0, "zipf"), (16385, 700, 33, 0, 0, "zipf"),
          (300, 50, 520, 8, 0, "out"), (511, 2000, 100, 0, 0, "zipf"), (1000, 3, 260, 0, 2, "zipf"),
          (2047, 1025, 65, 1, 0, "far"), (8192, 700, 33, 0, 0, "zipf"), (8193, 700, 33, 0, 0, "zipf"),
          (20000, 1023, 24, 0, 1, "one"), (33000, 5000, 17, 0, 0, "far"), (270000, 2100, 4, 0, 0, "zipf"),
          (4100, 70000, 3, 0, 0, "far"), (256, 700, 741, 0, 0, "zipf"), (256, 33, 129, 3, 1, "one"),
          (257, 33, 741, 0, 0, "one"), (200, 12, 12, 0, 1, "pad"),
          (9000, 1 << 21, 1, 0, 0, "far"), (600, 40, 2300, 0, 0, "zipf")]


def _ids(kind, r, n, vocab, first):
    if kind == "one":                           # every token the same
        return np.full(n, first + vocab // 2)
    if kind == "out":                           # none of the shard's
        return r.choice([-1, -2 ** 31, first - 1, first + vocab, 2 ** 31 - 1], n)
    if kind == "zipf":
        return first + np.minimum(r.zipf(1.3, n) - 1, vocab - 1)
    ids = first + r.integers(-vocab // 4, vocab + vocab // 4 + 1, n)
    if kind == "pad":
        ids[n - n // 3:] = -1
    return ids


class Case:
    """Inputs on the host, their device copies inside larger allocations, and
    outputs that start out as 77."""

    def __init__(self, dtype, n, vocab, width, stride, shift, kind, scale=0.3, first=11, seed=0):
        r = np.random.default_rng(seed + n + 7 * vocab + 31 * width)
        f = lambda *s: r.normal(size=s).astype(np.float32)
        self.dtype, self.n, self.vocab, self.width, self.first = dtype, n, vocab, width, first
        self.scale, self.ld, self.shift = float(np.float32(scale)), width + stride, shift
        self.ids = _ids(kind, r, n, vocab, first).astype(np.int32)
        self.table, self.dy, self.old = f(vocab, width), f(n, self.ld), f(vocab, width)
        if dtype == "bf16":
            self.table, self.dy = (torch.from_numpy(a).bfloat16().float().numpy() for a in (self.table, self.dy))
        self.desc = sb.embed_desc(n, vocab, width, CODE[dtype], first, self.ld, self.scale)
        t = lambda a, kind: torch.from_numpy(np.ascontiguousarray(a)).to(TYPES.get(kind, torch.int32))
        self.d_table, self.d_dy = self.put(t(self.table, dtype)), self.put(t(self.dy, dtype))
        self.d_ids = self.put(t(self.ids, "i32"))
        self.whole_y, self.y = self.room((n, self.ld), TYPES[dtype])
        self.whole_d, self.dtable = self.room((vocab, width), torch.float32)
        need = sb.sb_embed_workspace_bytes(self.desc)
        self.whole_ws = torch.full((need + 256,), 77, dtype=torch.uint8, device="cuda")
        self.ws = self.whole_ws[:need]

    def room(self, shape, kind):
        size = int(np.prod(shape))
        w = torch.full((size + self.shift + 64,), 77, dtype=kind, device="cuda")
        return w, w[self.shift:self.shift + size].view(shape)

    def put(self, t):
        w, v = self.room(t.shape, t.dtype)
        v.copy_(t)
        return v

    def fwd(self, stream=None):
        sb.sb_embed_fwd(self.desc, self.d_table, self.d_ids, self.y, stream)

    def bwd(self, accumulate=False, stream=None):
        sb.sb_embed_bwd(self.desc, self.d_ids, self.d_dy, self.dtable, accumulate, self.ws, stream)

    def check_fwd(self):
        ref = E.forward(self.table, self.ids, self.first, self.scale)
        far = np.abs(self.y.double().cpu().numpy()[:, :self.width] - ref)
        assert np.all(far <= E.forward_bound(ref, self.scale, self.dtype == "bf16"))

    def check_bwd(self, old=None):
        dy = self.dy[:, :self.width]
        ref = E.backward(dy, self.ids, self.first, self.vocab, self.scale, old)
        lim = E.backward_bound(dy, self.ids, self.first, self.vocab, self.scale, old)
        far = np.abs(self.dtable.double().cpu().numpy() - ref)
        assert np.all(far <= lim), (np.argwhere(~(far <= lim))[:4], float(np.nanmax(far)))

    def untouched(self):
        for w, v in ((self.whole_y, self.y), (self.whole_d, self.dtable)):
            n = v.numel()
            assert bool((w[:self.shift] == 77).all()) and bool((w[self.shift + n:] == 77).all())
        assert bool((self.y[:, self.width:] == 77).all())
        assert bool((self.whole_ws[len(self.ws):] == 77).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_shapes(shape, dtype):
    print_case("embed", shape=shape, dtype=dtype)
    c = Case(dtype, *shape)
    c.fwd()
    c.bwd()
    torch.cuda.synchronize()
    c.check_fwd()
    c.check_bwd()
    c.untouched()
    # On top of what is there; rows without a token stay as they are, to the bit.
    c.dtable.copy_(torch.from_numpy(c.old))
    c.bwd(True)
    torch.cuda.synchronize()
    c.check_bwd(c.old)
    c.untouched()


def test_scale_of_one_keeps_rows_to_the_bit():
    for dtype, bits in (("f32", torch.int32), ("bf16", torch.int16)):
        c = Case(dtype, 50, 9, 40, 0, 0, "any", scale=1.0)
        c.d_table[3] = float("inf")
        c.d_table[4] = float("nan")
        c.d_table[5] = -0.0
        c.d_table.view(bits)[6] = 1                 # the smallest subnormal
        c.fwd()
        at = torch.from_numpy(c.ids).long().cuda() - c.first
        inside = (at >= 0) & (at < 9)
        want = torch.where(inside[:, None], c.d_table.view(bits)[at.clamp(0, 8)], 0)
        assert torch.equal(c.y.view(bits), want)


def test_special_gradients_stay_in_their_row():
    c = Case("f32", 700, 40, 70, 0, 0, "zipf")
    hit = int(np.argmax(c.ids == c.first + 1))
    c.d_dy[hit, 5] = float("nan")
    c.d_dy[int(np.argmax(c.ids == c.first)), 6] = float("inf")
    c.bwd()
    bad = ~torch.isfinite(c.dtable)
    assert bool(bad[1, 5]) and bool(bad[0, 6]) and int(bad.sum()) == 2


def test_long_sums_of_one_sign_do_not_drift():
    """A token that fills the batch: 40000 ones are summed exactly (whole numbers below 2^24)."""
    c = Case("f32", 40000, 5, 130, 0, 0, "one", scale=1.0)
    c.d_dy.fill_(1.0)
    c.bwd()
    want = torch.zeros_like(c.dtable)
    want[2] = 40000.0
    assert torch.equal(c.dtable, want)


@pytest.mark.parametrize("shape", [(5000, 900, 129, 0, 0, "zipf"), (20000, 3000, 40, 0, 0, "zipf"),
                                   (200, 90, 129, 0, 0, "zipf")])
def test_repeats_streams_and_graphs_agree(shape):
    print_case("embed repeats", shape=shape)
    c = Case("bf16", *shape)
    c.bwd()
    torch.cuda.synchronize()
    first = c.dtable.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        c.dtable.fill_(5)
        c.bwd()
        c.fwd()
    side.synchronize()
    assert torch.equal(c.dtable, first)
    y = c.y.clone()
    # Two graphs on one workspace, replayed in turn with eager work between them.
    d = Case("bf16", *shape, seed=9)
    d.ws = c.ws
    d.bwd()
    torch.cuda.synchronize()
    other = d.dtable.clone()
    graphs = []
    for x in (c, d):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.fwd()
            x.bwd()
        graphs.append(g)
    for turn in range(3):
        for x, g, want in ((c, graphs[0], first), (d, graphs[1], other)):
            x.dtable.fill_(turn)
            x.y.fill_(turn)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(x.dtable, want)
        assert torch.equal(c.y, y)
    # New ids in the same buffer: the graph reads them.
    c.d_ids.copy_(d.d_ids)
    c.ids = d.ids
    graphs[0].replay()
    torch.cuda.synchronize()
    c.check_bwd()


def test_calls_at_once_on_their_own_workspaces():
    cases = [Case("f32", 9000 + 100 * i, 500, 64, 0, 0, "zipf", seed=i) for i in range(3)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for c, s in zip(cases, streams):
        for _ in range(3):
            c.bwd(stream=s)
    torch.cuda.synchronize()
    for c in cases:
        c.check_bwd()


def test_tables_past_32_bits():
    """A table of more than 2^32 elements and a gradient row at its end."""
    vocab, width = (1 << 21) + 5, 2050
    table = torch.empty((vocab, width), dtype=torch.bfloat16, device="cuda")
    table[-1] = 3.0
    table[-2] = 2.0
    ids = torch.tensor([vocab - 1, vocab - 2, vocab - 1], dtype=torch.int32, device="cuda")
    y = torch.empty((3, width), dtype=torch.bfloat16, device="cuda")
    d = sb.embed_desc(3, vocab, width, sb.SB_BF16)
    sb.sb_embed_fwd(d, table, ids, y)
    assert bool((y[0] == 3).all()) and bool((y[1] == 2).all()) and bool((y[2] == 3).all())
    del table
    dtable = torch.full((vocab, width), 7.0, device="cuda")
    ws = torch.empty((sb.sb_embed_workspace_bytes(d),), dtype=torch.uint8, device="cuda")
    sb.sb_embed_bwd(d, ids, y, dtable, False, ws)
    assert bool((dtable[-1] == 6).all()) and bool((dtable[-2] == 2).all())
    assert float(dtable[:-2].abs().max()) == 0.0
