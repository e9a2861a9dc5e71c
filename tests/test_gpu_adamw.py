"""GPU parity of the AdamW step (sb_adamw_update, sb_adamw_advance,
sb_adamw_unpack) against oracle/adamw.py: fp32 moments within bounds of their
roundings, moments in bytes bit for bit over several steps; odd sizes, views off
any alignment, more tensors than a launch takes, special values, a captured
step, another stream."""
import numpy as np
import pytest
import torch

from oracle import adamw as A
from paper_2112_15317_amd import sb
from tests.helpers import print_case

pytestmark = pytest.mark.gpu

B1, B2, EPS, LR = 0.9, 0.999, 1e-8, 1e-3
U = 2.0 ** -24                    # half a step of fp32
SIZES = {"one": [1], "odd": [5, 1024, 4099, 0, 17, 256, 257, 4096, 12289], "many": [300 + 7 * i for i in range(95)],
         "large": [3 << 20, 3, 4097]}


def _inputs(n, seed):
    rng = np.random.default_rng(seed)
    f = np.float32
    octave = 2.0 ** rng.integers(-6, 3, n)
    return ((rng.normal(size=n) * 0.02).astype(f), (rng.normal(size=n) * 1e-3 * octave).astype(f),
            (rng.normal(size=n) * 1e-3 * octave).astype(f),
            (rng.normal(size=n) ** 2 * 1e-6 * octave ** 2).astype(f))


def _dev(a, shift=0):
    """A device copy whose data start `shift` elements into an allocation, with
    16 elements behind it; the whole allocation and the view."""
    t = torch.from_numpy(np.ascontiguousarray(a))
    whole = torch.full((len(t) + shift + 16,), 77, dtype=t.dtype, device="cuda")
    whole[shift:shift + len(t)] = t.cuda()
    return whole, whole[shift:shift + len(t)]


def _untouched(whole, shift, n):
    w = whole.cpu()
    return bool((w[:shift] == 77).all()) and bool((w[shift + n:] == 77).all())


def _check_w(got, w, g, m, v, t, scale, decay):
    """w' = keep w - rate (m' / den).  Roundings: keep and its product and the
    difference, 3 of |w|, and one of the result; m' 4 of its two terms (constant,
    scale, product, sum), v' 5 (2 and more of g^2) that the root halves, rate,
    root, bias factor and its product, eps and the sum with it, quotient and product:
    under 16 of the update's terms."""
    rw, rm, rv = A.update(w, g, m, v, t, LR, B1, B2, EPS, scale, decay)
    terms = np.abs(B1 * m.astype(np.float64)) + np.abs((1 - B1) * scale * g.astype(np.float64))
    den = np.sqrt(rv / (1 - B2 ** t)) + EPS
    upd = LR / (1 - B1 ** t) * terms / den
    assert np.all(np.abs(got - rw) <= U * (3 * np.abs(w) + 16 * upd + np.abs(rw)))
    return rw, rm, rv, terms


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("sizes", SIZES)
def test_fp32_moments(sizes, shift):
    print_case("adamw32", sizes=sizes, shift=shift)
    items, host, keep = [], [], []
    for i, n in enumerate(SIZES[sizes]):
        w, g, m, v = _inputs(n, i)
        bufs = [_dev(a, shift) for a in (w, g, m, v)]
        copy = torch.full((n + shift + 16,), 77, dtype=torch.bfloat16, device="cuda")
        scale, decay = (1.0, 0.1) if i % 2 == 0 else (0.25, 0.0)
        items.append(dict(w=bufs[0][1], g=bufs[1][1], m=bufs[2][1], v=bufs[3][1], scale=scale,
                          decay=decay, copy=copy[shift:shift + n] if i % 3 == 0 else None))
        host.append((w, g, m, v, scale, decay))
        keep.append(bufs + [(copy, None)])
    sb.sb_adamw_update(sb.AdamwList(items), LR, B1, B2, EPS, step=3)
    torch.cuda.synchronize()
    for (w, g, m, v, scale, decay), it, bufs in zip(host, items, keep):
        n = len(w)
        got = it["w"].cpu().numpy()
        rw, rm, rv, terms = _check_w(got, w, g, m, v, 3, scale, decay)
        assert np.all(np.abs(it["m"].cpu().numpy() - rm) <= 4 * U * terms)
        assert np.all(np.abs(it["v"].cpu().numpy() - rv) <= 6 * U * rv)
        assert np.array_equal(it["g"].cpu().numpy(), g)
        for whole, _ in bufs[:4]:
            assert _untouched(whole, shift, n)
        if it["copy"] is not None:
            assert torch.equal(it["copy"].cpu(), it["w"].cpu().to(torch.bfloat16))
            assert _untouched(bufs[4][0], shift, n)


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("sizes", SIZES)
def test_moments_in_bytes_over_steps(sizes, shift):
    print_case("adamw8", sizes=sizes, shift=shift)
    seed, items, state, keep, first = 99, [], [], [], 0
    for i, n in enumerate(SIZES[sizes]):
        w, _, _, _ = _inputs(n, i)
        tops = -(-n // 256)
        bufs = [_dev(a, shift) for a in (w, np.zeros(n, np.float32), np.zeros(n, np.uint8),
                                         np.zeros(n, np.uint8), np.zeros(tops, np.int16),
                                         np.zeros(tops, np.int16))]
        scale, decay = (1.0, 0.1) if i % 2 == 0 else (0.25, 0.0)
        it = dict(zip(("w", "g", "m", "v", "m_top", "v_top"), (b[1] for b in bufs)))
        it.update(scale=scale, decay=decay)
        if i == 2:
            it["first"] = (1 << 32) - 700           # numbers that pass 32 bits
        first = it.get("first", first)
        items.append(it)
        keep.append(bufs)
        state.append([first, np.zeros(n, np.uint8), np.zeros(tops, np.int16),
                      np.zeros(n, np.uint8), np.zeros(tops, np.int16)])
        first += n
    lst = sb.AdamwList(items)
    for t in range(1, 5):
        before = [it["w"].cpu().numpy() for it in items]
        grads = [_inputs(len(b), 1000 * t + i)[1] for i, b in enumerate(before)]
        for it, g in zip(items, grads):
            it["g"].copy_(torch.from_numpy(g))
        sb.sb_adamw_update(lst, LR, B1, B2, EPS, step=t, seed=seed)
        torch.cuda.synchronize()
        for it, w, g, s in zip(items, before, grads, state):
            m, v = A.unpack(*s[1:])
            nm, nv = A.moments(g, m, v, B1, B2, it["scale"])
            s[1:] = A.pack(nm, nv, A.noise(len(g), s[0], t, seed))
            for name, ref in zip(("m", "m_top", "v", "v_top"), s[1:]):
                np.testing.assert_array_equal(it[name].cpu().numpy(), ref, err_msg="%s %d" % (name, t))
            _check_w(it["w"].cpu().numpy(), w, g, m, v, t, it["scale"], it["decay"])
    for it, bufs, s in zip(items, keep, state):
        n = len(s[1])
        for (whole, view) in bufs:
            assert _untouched(whole, shift, len(view))
        out = [torch.full((n + 1 + 16,), 77.0, device="cuda") for _ in range(2)]
        sb.sb_adamw_unpack(n, it["m"], it["m_top"], it["v"], it["v_top"], out[0][shift:], out[1][shift:])
        for o, ref in zip(out, A.unpack(*s[1:])):
            assert np.array_equal(o[shift:shift + n].cpu().numpy(), ref)
            assert _untouched(o, shift, n)


def test_special_values_and_zero_gradients():
    print_case("adamw_special")
    n = 600
    w, g, _, _ = _inputs(n, 5)
    g[:256] = 0.0
    g[300], g[301], g[520] = np.inf, np.nan, 1e30          # 1e60 is past fp32
    st = sb.adamw_moments(torch.zeros(n, device="cuda"), 8)
    wd, gd = torch.from_numpy(w).cuda(), torch.from_numpy(g).cuda()
    sb.sb_adamw_update(sb.AdamwList([dict(w=wd, g=gd, **st)]), LR, B1, B2, EPS, step=1, seed=4)
    nm, nv = A.moments(g, np.zeros(n), np.zeros(n), B1, B2)
    ref = A.pack(nm, nv, A.noise(n, 0, 1, 4))
    for name, r in zip(("m", "m_top", "v", "v_top"), ref):
        assert np.array_equal(st[name].cpu().numpy(), r), name
    got = wd.cpu().numpy()
    assert np.array_equal(got[:256], w[:256])              # no gradient yet: nothing moves
    assert np.isnan(got[[300, 301]]).all() and np.isfinite(np.delete(got, [300, 301])).all()
    # One pair of moments alone.
    out = torch.empty(n, device="cuda")
    sb.sb_adamw_unpack(n, None, None, st["v"], st["v_top"], None, out)
    assert np.array_equal(out.cpu().numpy(), A.unpack(*ref)[1], equal_nan=True)


@pytest.mark.parametrize("bits", [8, 32])
def test_captured_step_with_a_counter(bits):
    """Every replay of a captured update and advance equals an eager update of
    the same number, bit for bit."""
    print_case("adamw_graph", bits=bits)
    n = 5000
    w, _, _, _ = _inputs(n, 8)
    a, b = torch.from_numpy(w).cuda(), torch.from_numpy(w).cuda()
    g = torch.zeros(n, device="cuda")
    sa, sb_ = sb.adamw_moments(a, bits), sb.adamw_moments(b, bits)
    la, lb = sb.AdamwList([dict(w=a, g=g, **sa)]), sb.AdamwList([dict(w=b, g=g, **sb_)])
    count = torch.zeros(1, dtype=torch.int32, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sb.sb_adamw_update(la, LR, B1, B2, EPS, step=1, seed=5, steps_done=count)
        sb.sb_adamw_advance(count)
    for t in range(1, 6):
        g.copy_(torch.from_numpy(_inputs(n, 50 + t)[1]))
        graph.replay()
        torch.cuda.synchronize()
        assert int(count.item()) == t
        # The counter's factors are formed on the device: held to an eager call
        # with a counter, and that one's moments to the call without.
        eager = torch.full((1,), t - 1, dtype=torch.int32, device="cuda")
        sb.sb_adamw_update(lb, LR, B1, B2, EPS, step=1, seed=5, steps_done=eager)
        assert torch.equal(a, b)
        for k in sa:
            assert torch.equal(sa[k], sb_[k]), (t, k)


def test_counter_and_number_agree():
    print_case("adamw_counter")
    n = 3000
    w, g, m, v = _inputs(n, 9)
    out = []
    for counter in (False, True):
        t = [torch.from_numpy(x).cuda() for x in (w, g, m, v)]
        lst = sb.AdamwList([dict(w=t[0], g=t[1], m=t[2], v=t[3])])
        done = torch.full((1,), 40, dtype=torch.int32, device="cuda") if counter else None
        sb.sb_adamw_update(lst, LR, B1, B2, EPS, step=1 if counter else 41, steps_done=done)
        out.append([x.cpu().numpy() for x in t])
    for x, y in zip(out[0][1:], out[1][1:]):
        assert np.array_equal(x, y)
    # The two factors from powers formed another way: a rounding of each.
    upd = np.abs(out[0][0] - w)
    assert np.all(np.abs(out[0][0] - out[1][0]) <= U * (4 * upd + 2 * np.abs(w)))


def test_on_another_stream():
    print_case("adamw_stream")
    n = 1 << 20
    w, g, m, v = _inputs(n, 10)
    t = [torch.from_numpy(x).cuda() for x in (w, g, m, v)]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    lst = sb.AdamwList([dict(w=t[0], g=t[1], m=t[2], v=t[3])])
    sb.sb_adamw_update(lst, LR, B1, B2, EPS, step=2, stream=s)
    s.synchronize()
    _check_w(t[0].cpu().numpy(), w, g, m, v, 2, 1.0, 0.0)


@pytest.mark.parametrize("bits", [8, 32])
def test_as_many_tensors_as_a_plan_takes(bits):
    """512 tensors, some of no elements, in one update: as 512 updates of one."""
    print_case("adamw_512", bits=bits)
    sizes = [(37 * i) % 700 if i % 50 else 0 for i in range(sb.SB_ADAMW_MAX_TENSORS)]
    first = np.concatenate([[0], np.cumsum(sizes)])
    w, g, _, _ = (torch.from_numpy(a).cuda() for a in _inputs(int(first[-1]), 3))
    out = []
    for one in (False, True):
        ws = [w[a:b].clone() for a, b in zip(first, first[1:])]
        items = [dict(w=x, g=g[a:a + x.numel()], first=int(a), decay=0.1, **sb.adamw_moments(x, bits))
                 for x, a in zip(ws, first)]
        lists = [sb.AdamwList([it]) for it in items] if one else [sb.AdamwList(items)]
        for t in (1, 2):
            for lst in lists:
                sb.sb_adamw_update(lst, LR, B1, B2, EPS, step=t, seed=7)
        torch.cuda.synchronize()
        out.append(items)
    for a, b in zip(*out):
        for key in ("w", "m", "v"):
            assert torch.equal(a[key], b[key]), key
    assert not torch.equal(torch.cat([it["w"] for it in out[0]]), w)


@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-8])
def test_small_second_moments(eps):
    """Roots of values down to fp32's subnormal ones, with an eps that hides them and
    without: a move of lr m' / (root + eps), roundings as in _check_w, and in v' half
    a step of the smallest subnormal value for each of its three products and sums."""
    print_case("adamw_small_v", eps=eps)
    n = 1000
    rng = np.random.default_rng(17)
    f = np.float32
    v = (2.0 ** rng.uniform(-140, -20, n)).astype(f)
    m = (np.sqrt(v.astype(np.float64)) * rng.normal(size=n)).astype(f)
    w, g = np.zeros(n, f), np.zeros(n, f)
    t = [torch.from_numpy(x).cuda() for x in (w, g, m, v)]
    lst = sb.AdamwList([dict(w=t[0], g=t[1], m=t[2], v=t[3])])
    sb.sb_adamw_update(lst, LR, B1, B2, eps, step=5)
    rw, _, rv = A.update(w, g, m, v, 5, LR, B1, B2, eps)
    got = t[0].cpu().numpy()
    assert np.isfinite(got).all()
    # An error d of v' moves its root by d / (2 root), so the quotient by d / (2 v').
    far = np.abs(got - rw) / np.abs(rw)
    assert np.all(far <= 17 * U + 3 * 2.0 ** -150 / (2 * rv))


def test_lists_of_a_plan_used_on_several_streams():
    """A list is ready for any stream when it is made; two lists, a stream each."""
    print_case("adamw_streams")
    n = 40000
    made = []
    for i in range(2):
        w, g, m, v = _inputs(n, 60 + i)
        t = [torch.from_numpy(x).cuda() for x in (w, g, m, v)]
        made.append((t, [x.clone() for x in t]))
    streams = [torch.cuda.Stream() for _ in range(2)]
    lists = [sb.AdamwList([dict(zip("wgmv", t))]) for t, _ in made]
    for step in (1, 2, 3):
        for lst, s in zip(lists, streams):
            sb.sb_adamw_update(lst, LR, B1, B2, EPS, step=step, stream=s)
    torch.cuda.synchronize()
    for t, u in made:
        lst = sb.AdamwList([dict(zip("wgmv", u))])
        for step in (1, 2, 3):
            sb.sb_adamw_update(lst, LR, B1, B2, EPS, step=step)
        torch.cuda.synchronize()
        for a, b in zip(t, u):
            assert torch.equal(a, b)


def test_moments_in_bytes_of_very_many_elements():
    """As many elements as take two groups a lane: the same bits as in pieces that do not."""
    print_case("adamw_very_many")
    n = (24 << 20) + 4099
    g = torch.Generator(device="cuda").manual_seed(2)
    w, grad = (torch.randn(n, generator=g, device="cuda") * s for s in (0.02, 1e-3))
    out = []
    for pieces in (1, 4):
        x, st = w.clone(), sb.adamw_moments(w, 8)
        size = -(-n // pieces) // 256 * 256 + 256
        lists = []
        for a in range(0, n, size):
            b = min(n, a + size)
            tops = slice(a // 256, -(-b // 256))
            lists.append(sb.AdamwList([dict(w=x[a:b], g=grad[a:b], m=st["m"][a:b], v=st["v"][a:b],
                                            m_top=st["m_top"][tops], v_top=st["v_top"][tops], first=a)]))
        for t in (1, 2):
            for lst in lists:
                sb.sb_adamw_update(lst, LR, B1, B2, EPS, step=t, seed=7)
        torch.cuda.synchronize()
        out.append((x, st, len(lists), lists[0].info.groups))
    assert (out[0][2:], out[1][2:]) == ((1, 2), (4, 1))
    assert torch.equal(out[0][0], out[1][0])
    for key in out[0][1]:
        assert torch.equal(out[0][1][key], out[1][1][key]), key
