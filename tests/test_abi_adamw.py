"""Refusals of the AdamW calls on the host: each call fails its checks, so no
kernel is launched and the addresses are never used."""
import ctypes

import pytest

from paper_2112_15317_amd import sb

P = 0x10000000


def _call(desc=None, tensors=None, count=None, counter=None):
    d = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, moments=32, seed=0)
    d.update(desc or {})
    tensors = [{}] if tensors is None else tensors
    ts = (sb.sb_adamw_tensor * max(1, len(tensors)))()
    for i, (t, over) in enumerate(zip(ts, tensors)):
        at = P + i * 0x1000000
        v = dict(w=at, copy=None, g=at + 0x100000, m=at + 0x200000, v=at + 0x300000,
                 m_top=at + 0x400000, v_top=at + 0x500000, first=0, n=1000, grad_scale=1.0, decay=0.0)
        v.update(over)
        for k, x in v.items():
            setattr(t, k, x)
    return sb.load().sb_adamw_update(
        ctypes.byref(sb.sb_adamw_desc(**d)), len(tensors) if count is None else count, ts, counter, None)


BAD = sb.SB_ERR_INVALID_ARG


@pytest.mark.parametrize("desc", [
    dict(step=0), dict(step=-3), dict(moments=16), dict(beta1=1.0), dict(beta1=-0.1),
    dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=-1e-8), dict(eps=float("inf")),
    dict(lr=float("nan")), dict(lr=1e300), dict(lr=float("inf"))])
def test_bad_numbers_are_refused(desc):
    assert _call(desc) == BAD


@pytest.mark.parametrize("over", [
    dict(w=None), dict(g=None), dict(m=None), dict(v=None), dict(w=P + 2), dict(g=P + 0x100002),
    dict(m=P + 0x200001), dict(copy=P + 0x600001), dict(n=1 << 40), dict(grad_scale=float("nan")),
    dict(decay=float("inf"))])
def test_bad_tensors_are_refused(over):
    assert _call(tensors=[over]) == BAD
    assert _call(tensors=[dict(n=0), over]) == BAD


@pytest.mark.parametrize("over", [dict(m_top=None), dict(v_top=None), dict(m_top=P + 0x400001)])
def test_references_are_checked_with_bytes(over):
    assert _call(dict(moments=8), [over]) == BAD


@pytest.mark.parametrize("over", [
    dict(g=P), dict(g=P + 3996), dict(m=P + 3996), dict(v=P + 0x200000), dict(copy=P + 2000),
    dict(copy=P + 0x100000), dict(m_top=P + 0x500000), dict(v_top=P + 0x300002), dict(m=P + 0x100004)])
def test_overlaps_are_refused(over):
    assert _call(dict(moments=8 if "m_top" in over or "v_top" in over else 32), [over]) == BAD


def test_overlaps_between_tensors_and_with_the_counter():
    second = P + 0x1000000
    assert _call(tensors=[{}, dict(w=P + 400)]) == BAD
    assert _call(tensors=[{}, dict(g=P + 400)]) == BAD
    assert _call(tensors=[dict(copy=second + 0x200000), {}]) == BAD
    assert _call(counter=P + 8) == BAD
    assert _call(counter=P + 0x700002) == BAD


def test_counts_and_null_arrays():
    lib = sb.load()
    assert _call(count=0) == BAD and _call(count=-1) == BAD
    assert _call(count=sb.SB_ADAMW_MAX_TENSORS + 1) == BAD
    ts = (sb.sb_adamw_tensor * 1)()
    d = sb.sb_adamw_desc(1e-3, 0.9, 0.999, 1e-8, 1, 32, 0)
    assert lib.sb_adamw_update(None, 1, ts, None, None) == BAD
    assert lib.sb_adamw_update(ctypes.byref(d), 1, None, None, None) == BAD
    assert lib.sb_adamw_update(ctypes.byref(d), 1, ts, None, None) == sb.SB_OK    # n = 0: nothing to do
    assert lib.sb_adamw_advance(None, None) == BAD and lib.sb_adamw_advance(P + 2, None) == BAD


@pytest.mark.parametrize("args", [
    (None, P, P + 0x10000, P + 0x20000, P + 0x30000, P + 0x40000),
    (P, None, P + 0x10000, P + 0x20000, P + 0x30000, P + 0x40000),
    (P, P + 0x8000, None, P + 0x20000, P + 0x30000, P + 0x40000),
    (P, P + 0x8000, P + 0x10000, None, P + 0x30000, P + 0x40000),
    (P, P + 0x8000, P + 0x10000, P + 0x20000, P + 0x30002, P + 0x40000),
    (P, P + 0x8000, P + 0x10000, P + 0x20000, P + 0x30000, P + 0x30100),
    (P, P + 0x8000, P + 0x10000, P + 0x20000, P, P + 0x40000),
    (P, P + 0x8000, P + 0x10000, P + 0x20000, P + 0x30000, P + 0xffc0)])
def test_unpack_refusals(args):
    assert sb.load().sb_adamw_unpack(1000, *args, None) == BAD


def test_unpack_of_nothing():
    assert sb.load().sb_adamw_unpack(0, None, None, None, None, None, None, None) == sb.SB_OK
    assert sb.load().sb_adamw_unpack(1 << 40, P, P, P, P, P, P, None) == BAD


def test_lists_are_checked():
    torch = pytest.importorskip("torch")
    w = torch.zeros(300)
    with pytest.raises(ValueError):
        sb.AdamwList([])
    with pytest.raises(ValueError):
        sb.AdamwList([dict(w=w, g=w[:-1], m=w, v=w)])
    with pytest.raises(ValueError):
        sb.AdamwList([dict(w=w, g=w.double(), m=w, v=w)])
    b, top = w.to(torch.uint8), torch.zeros(1, dtype=torch.int16)
    with pytest.raises(ValueError):
        sb.AdamwList([dict(w=w, g=w, m=b, v=b, m_top=top, v_top=top)])
    with pytest.raises(ValueError):
        sb.AdamwList([dict(w=w, g=w, m=w, v=w, copy=w)])
    with pytest.raises(ValueError):
        sb.adamw_moments(w, 16)
    assert {k: tuple(t.shape) for k, t in sb.adamw_moments(w, 8).items()} == {
        "m": (300,), "v": (300,), "m_top": (2,), "v_top": (2,)}
