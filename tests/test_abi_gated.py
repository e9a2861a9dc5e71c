"""Refusals of the gated shard's calls on the host: each call fails its checks,
so no kernel is launched and the addresses are never used."""
import ctypes

import pytest

from paper_2112_15317_amd import sb

P = 0x10000000
M, K, N = 100, 64, 48
GAP = 1 << 24
ORDER_F = ("x", "w_gate", "w_up", "b_gate", "b_up", "y", "pre")
ORDER_B = ("x", "w_gate", "w_up", "pre", "dy", "dx", "dw_gate", "dw_up", "db_gate", "db_up")
BAD, NO = sb.SB_ERR_INVALID_ARG, sb.SB_ERR_UNSUPPORTED
SIZE_MAX = sb.SIZE_MAX


def _desc(**over):
    d = dict(m=M, k_in=K, n_shard=N, dtype=sb.SB_BF16, act=sb.SB_ACT_SILU)
    d.update(over)
    return sb.gated_desc(**d)


def _fwd(desc=None, ws=P + 20 * GAP, short=0, **over):
    d = desc or _desc()
    at = {t: P + i * GAP for i, t in enumerate(ORDER_F)}
    at.update(over)
    need = sb.sb_gated_workspace_bytes(_desc(), sb.SB_FC_FWD)
    return sb.load().sb_gated_shard_fwd(ctypes.byref(d), *[at[t] for t in ORDER_F], ws,
                                        max(0, need - short), None)


def _bwd(desc=None, ws=P + 20 * GAP, short=0, accumulate=0, **over):
    d = desc or _desc()
    at = {t: P + i * GAP for i, t in enumerate(ORDER_B)}
    at.update(over)
    need = sb.sb_gated_workspace_bytes(_desc(), sb.SB_FC_BWD)
    return sb.load().sb_gated_shard_bwd(ctypes.byref(d), *[at[t] for t in ORDER_B], accumulate, ws,
                                        max(0, need - short), None)


@pytest.mark.parametrize("over", [
    dict(m=0), dict(m=-1), dict(k_in=0), dict(n_shard=0), dict(dtype=2), dict(act=-1), dict(act=5),
    dict(ldx=K - 1), dict(ldy=N - 1)])
def test_bad_descriptors(over):
    d = _desc(**over)
    assert _fwd(d) == BAD and _bwd(d) == BAD
    for p in (sb.SB_FC_FWD, sb.SB_FC_BWD):
        assert sb.sb_gated_workspace_bytes(d, p) == SIZE_MAX


def test_null_descriptor_and_pass():
    lib = sb.load()
    assert lib.sb_gated_workspace_bytes(None, 0) == SIZE_MAX
    assert sb.sb_gated_workspace_bytes(_desc(), 2) == SIZE_MAX
    assert lib.sb_gated_shard_fwd(None, P, P, P, None, None, P, None, None, 0, None) == BAD
    assert lib.sb_gated_shard_bwd(None, P, P, P, P, P, P, P, P, None, None, 0, None, 0, None) == BAD


@pytest.mark.parametrize("over", [
    dict(m=1 << 20, ldx=1025), dict(m=1 << 20, ldy=1025), dict(k_in=1 << 20, n_shard=1 << 10),
    dict(m=1 << 30), dict(m=1 << 20, ldx=513, dtype=sb.SB_F32)])
def test_tensors_past_the_index_range(over):
    d = _desc(**over)
    assert _fwd(d) == NO and _bwd(d) == NO
    assert sb.sb_gated_workspace_bytes(d, sb.SB_FC_BWD) == SIZE_MAX


@pytest.mark.parametrize("t", ["x", "w_gate", "w_up", "y"])
def test_null_tensors_forward(t):
    assert _fwd(**{t: None}) == BAD


@pytest.mark.parametrize("t", ["x", "w_gate", "w_up", "pre", "dy", "dw_gate", "dw_up"])
def test_null_tensors_backward(t):
    assert _bwd(**{t: None}) == BAD


def test_accumulate_is_a_truth_value():
    assert _bwd(accumulate=2) == BAD and _bwd(accumulate=-1) == BAD


@pytest.mark.parametrize("a,b", [("y", "x"), ("y", "w_gate"), ("y", "w_up"), ("y", "b_gate"),
                                 ("y", "b_up"), ("pre", "x"), ("pre", "b_up"), ("pre", "y")])
def test_overlaps_forward(a, b):
    at = P + ORDER_F.index(b) * GAP
    assert _fwd(**{a: at}) == BAD
    assert _fwd(**{a: at + 64}) == BAD


OUTS = ORDER_B[5:]


@pytest.mark.parametrize("a", OUTS)
@pytest.mark.parametrize("b", ORDER_B)
def test_overlaps_backward(a, b):
    if a != b:
        assert _bwd(**{a: P + ORDER_B.index(b) * GAP + 64}) == BAD


@pytest.mark.parametrize("t", ORDER_B)
def test_workspace_overlaps_backward(t):
    assert _bwd(ws=P + ORDER_B.index(t) * GAP) == BAD


def test_short_missing_and_unaligned_workspaces():
    assert _bwd(short=1) == sb.SB_ERR_WORKSPACE
    assert _bwd(ws=None) == sb.SB_ERR_WORKSPACE
    assert _bwd(ws=P + 20 * GAP + 8) == BAD


def test_operands_off_16_bytes_ask_for_room():
    """The size asked for without SB_UNALIGNED does not cover them."""
    for p in (sb.SB_FC_FWD, sb.SB_FC_BWD):
        assert sb.sb_gated_workspace_bytes(_desc(unaligned=True), p) > sb.sb_gated_workspace_bytes(
            _desc(), p)
    assert _fwd(x=P + 2) == sb.SB_ERR_WORKSPACE
    assert _bwd(w_up=P + 2 * GAP + 8) == sb.SB_ERR_WORKSPACE
    d = _desc()
    d.flags = 8
    assert _fwd(d) == BAD and _bwd(d) == BAD
