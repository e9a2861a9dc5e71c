"""Refusals of the AdamW calls on the host: each call fails its checks, so no
kernel is launched and the addresses are never used."""
import ctypes

import pytest

from paper_2112_15317_amd import sb

P = 0x10000000


PLAN = P + 0x70000000


def _plan(tensors=None, moments=32, count=None, plan=PLAN, short=0, info=True):
    tensors = [{}] if tensors is None else tensors
    ts = (sb.sb_adamw_tensor * max(1, len(tensors)))()
    for i, (t, over) in enumerate(zip(ts, tensors)):
        at = P + i * 0x1000000
        v = dict(w=at, copy=None, g=at + 0x100000, m=at + 0x200000, v=at + 0x300000,
                 m_top=at + 0x400000, v_top=at + 0x500000, first=0, n=1000, grad_scale=1.0, decay=0.0)
        v.update(over)
        for k, x in v.items():
            setattr(t, k, x)
    count = len(tensors) if count is None else count
    need = max(0, sb.load().sb_adamw_plan_bytes(len(tensors)) - short)
    out = sb.sb_adamw_plan()
    return sb.load().sb_adamw_make_plan(moments, count, ts, plan, need,
                                        ctypes.byref(out) if info else None, None)


def _update(plan=PLAN, info=(1, 32, 1, 1), counter=None, **over):
    d = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1, seed=0)
    d.update(over)
    return sb.load().sb_adamw_update(ctypes.byref(sb.sb_adamw_desc(**d)),
                                     ctypes.byref(sb.sb_adamw_plan(*info)), plan, counter, None)


BAD = sb.SB_ERR_INVALID_ARG


@pytest.mark.parametrize("over", [
    dict(step=0), dict(step=-3), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0),
    dict(beta2=float("nan")), dict(eps=-1e-8), dict(eps=float("inf")), dict(lr=float("nan")),
    dict(lr=1e300), dict(lr=float("inf")), dict(counter=P + 2), dict(plan=None), dict(plan=PLAN + 8),
    dict(info=(1, 16, 1, 1)), dict(info=(-1, 32, 1, 1)), dict(info=(513, 32, 1, 600)),
    dict(info=(2, 32, 1, 1)), dict(info=(0, 32, 1, 1)), dict(info=(1, 8, 1, -1)),
    dict(info=(1, 32, 2, 1)), dict(info=(1, 8, 4, 1)), dict(info=(1, 8, 0, 1))])
def test_bad_updates_are_refused(over):
    assert _update(**over) == BAD


def test_an_empty_plan_has_nothing_to_do():
    assert _update(info=(0, 32, 1, 0)) == sb.SB_OK
    assert sb.load().sb_adamw_update(None, None, None, None, None) == BAD


@pytest.mark.parametrize("over", [
    dict(w=None), dict(g=None), dict(m=None), dict(v=None), dict(w=P + 2), dict(g=P + 0x100002),
    dict(m=P + 0x200001), dict(copy=P + 0x600001), dict(n=1 << 40), dict(grad_scale=float("nan")),
    dict(decay=float("inf"))])
def test_bad_tensors_are_refused(over):
    assert _plan([over]) == BAD
    assert _plan([dict(n=0), over]) == BAD


@pytest.mark.parametrize("over", [dict(m_top=None), dict(v_top=None), dict(m_top=P + 0x400001)])
def test_references_are_checked_with_bytes(over):
    assert _plan([over], 8) == BAD


@pytest.mark.parametrize("over", [
    dict(g=P), dict(g=P + 3996), dict(m=P + 3996), dict(v=P + 0x200000), dict(copy=P + 2000),
    dict(copy=P + 0x100000), dict(m_top=P + 0x500000), dict(v_top=P + 0x300002), dict(m=P + 0x100004),
    dict(w=PLAN), dict(g=PLAN + 4)])
def test_overlaps_are_refused(over):
    assert _plan([over], 8 if "m_top" in over or "v_top" in over else 32) == BAD


def test_overlaps_between_tensors():
    second = P + 0x1000000
    assert _plan([{}, dict(w=P + 400)]) == BAD
    assert _plan([{}, dict(g=P + 400)]) == BAD
    assert _plan([dict(copy=second + 0x200000), {}]) == BAD


def test_counts_null_arrays_and_short_plans():
    lib = sb.load()
    top = sb.SB_ADAMW_MAX_TENSORS
    assert _plan(count=0) == BAD and _plan(count=-1) == BAD and _plan(count=top + 1) == BAD
    assert _plan(moments=16) == BAD and _plan(plan=None) == BAD and _plan(plan=PLAN + 8) == BAD
    assert _plan(info=False) == BAD
    assert lib.sb_adamw_make_plan(32, 1, None, PLAN, 1 << 20, ctypes.byref(sb.sb_adamw_plan()), None) == BAD
    assert _plan(short=1) == sb.SB_ERR_WORKSPACE
    assert lib.sb_adamw_plan_bytes(0) == 0 and lib.sb_adamw_plan_bytes(top + 1) == 0
    assert _plan([dict(n=0)]) == sb.SB_OK                  # no tensor with elements: nothing to write
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


def test_more_elements_than_a_launch_has_lanes_for():
    assert _plan([dict(n=1 << 33)]) == sb.SB_ERR_UNSUPPORTED
    assert sb.load().sb_adamw_unpack(1 << 34, P, P, P, P, P, P, None) == sb.SB_ERR_UNSUPPORTED


def test_none_is_refused_by_the_library():
    with pytest.raises(RuntimeError):
        sb.sb_adamw_advance(None, stream=0)


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
