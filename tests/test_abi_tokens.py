"""Refusals of the embedding's, the expert rows' and the token log-probabilities'
calls on the host: each call fails its checks, so no kernel is launched and the
addresses are never used."""
import ctypes

import pytest

from paper_2112_15317_amd import sb

P = 0x10000000
GAP = 1 << 26
BAD, NO, ROOM = sb.SB_ERR_INVALID_ARG, sb.SB_ERR_UNSUPPORTED, sb.SB_ERR_WORKSPACE
WS = P + 30 * GAP

# name: (descriptor, its sizes, tensors in the order of the call, outputs among them,
#        tensors that may be NULL, whether `accumulate` follows, the workspace's size or None)
EMBED = (sb.embed_desc, dict(tokens=9000, vocab=50, width=24, first=10, ldy=32))
EXPERT = (sb.expert_desc, dict(tokens=9000, top=2, experts=6, width=24, first=3, ldx=32, ldr=40))
LOGP = (sb.token_logp_desc, dict(m=5, classes=300000, top=4, ldz=300032, probs=True))
CALLS = {
    "sb_embed_fwd": (EMBED, ("table", "ids", "y"), ("y",), (), False, None),
    "sb_embed_bwd": (EMBED, ("ids", "dy", "dtable"), ("dtable",), (), True, sb.sb_embed_workspace_bytes),
    "sb_expert_sort": (EXPERT, ("ids", "place", "offsets"), ("place", "offsets"), (), False,
                       sb.sb_expert_workspace_bytes),
    "sb_expert_gather": (EXPERT, ("x", "place", "xs"), ("xs",), (), False, None),
    "sb_expert_combine": (EXPERT, ("ys", "place", "weights", "add", "y"), ("y",), ("weights", "add"), False, None),
    "sb_expert_combine_bwd": (EXPERT, ("dy", "ys", "place", "weights", "dys", "dweights"), ("dys", "dweights"),
                              ("weights", "dweights"), False, None),
    "sb_token_logp_fwd": (LOGP, ("z", "targets", "logp", "entropy", "stats", "top_ids", "top_values"),
                          ("logp", "entropy", "stats", "top_ids", "top_values"), ("logp", "entropy"), False,
                          sb.sb_token_logp_workspace_bytes),
    "sb_token_logp_bwd": (LOGP, ("z", "stats", "targets", "dlogp", "entropy", "dentropy", "top_ids", "top_values",
                                 "dtop", "dz"), ("dz",), ("dlogp", "dentropy", "dtop"), False, None),
}
NAMES = sorted(CALLS)
WITH_WS = [n for n in NAMES if CALLS[n][5]]


def _desc(name, **over):
    make, sizes = CALLS[name][0]
    over = {k: v for k, v in over.items()}
    raw = {k: over.pop(k) for k in list(over) if k in ("flags",)}
    d = make(**{**sizes, "dtype": sb.SB_BF16, **over})
    for k, v in raw.items():
        setattr(d, k, v)
    return d


def _call(name, desc=None, ws=WS, short=0, accumulate=0, **over):
    _, order, _, _, acc, size = CALLS[name]
    d = desc if desc is not None else _desc(name)
    args = [over.get(t, P + i * GAP) for i, t in enumerate(order)]
    if acc:
        args.append(accumulate)
    if size:
        args += [ws, size(_desc(name)) - short]
    return getattr(sb.load(), name)(ctypes.byref(d), *args, None)


BAD_DESCS = (
    [(n, o) for n in NAMES if "embed" in n for o in (
        dict(tokens=-1), dict(vocab=0), dict(width=0), dict(first=-1), dict(dtype=2), dict(ldy=23),
        dict(scale=float("nan")), dict(scale=float("inf")), dict(first=2 ** 31 - 50))] +
    [(n, o) for n in NAMES if "expert" in n for o in (
        dict(tokens=-1), dict(top=0), dict(experts=0), dict(experts=513), dict(width=0), dict(first=-1),
        dict(dtype=-1), dict(ldx=23), dict(ldr=23), dict(first=2 ** 31 - 6))] +
    [(n, o) for n in NAMES if "logp" in n for o in (
        dict(m=-1), dict(classes=0), dict(ldz=299999), dict(top=-1), dict(top=33), dict(classes=3), dict(dtype=2),
        dict(flags=1))])


@pytest.mark.parametrize("name,over", BAD_DESCS, ids=lambda v: str(v))
def test_bad_descriptors(name, over):
    d = _desc(name, **over)
    assert _call(name, d) == BAD
    if CALLS[name][5]:
        assert CALLS[name][5](d) == sb.SIZE_MAX


@pytest.mark.parametrize("name,over", [
    ("sb_embed_fwd", dict(tokens=1 << 30)), ("sb_embed_bwd", dict(width=1 << 23, ldy=1 << 23)),
    ("sb_expert_sort", dict(tokens=1 << 29)), ("sb_expert_gather", dict(width=1 << 24, ldx=1 << 24, ldr=1 << 24)),
    ("sb_token_logp_fwd", dict(classes=(1 << 20) + 1, ldz=1 << 21)), ("sb_token_logp_bwd", dict(m=1 << 30))])
def test_sizes_past_what_is_provided(name, over):
    d = _desc(name, **over)
    assert _call(name, d) == NO
    if CALLS[name][5]:
        assert CALLS[name][5](d) == sb.SIZE_MAX


# A launch has fewer than 2^32 lanes: 8 at least for a row, one for 16 of its bytes or more.
@pytest.mark.parametrize("name,over", [
    ("sb_embed_fwd", dict(tokens=1 << 29)), ("sb_embed_fwd", dict(tokens=1 << 26, width=512, ldy=512)),
    ("sb_embed_bwd", dict(vocab=1 << 29)), ("sb_embed_bwd", dict(tokens=1 << 29)),
    ("sb_expert_gather", dict(tokens=1 << 29, top=1)), ("sb_expert_combine", dict(tokens=1 << 29, top=1)),
    ("sb_expert_combine_bwd", dict(tokens=1 << 26, top=2, width=512, ldx=512, ldr=512)),
    ("sb_token_logp_fwd", dict(m=1 << 29, classes=8, ldz=8)), ("sb_token_logp_bwd", dict(m=1 << 29, classes=8, ldz=8)),
    ("sb_token_logp_fwd", dict(m=1 << 26, classes=1025)), ("sb_token_logp_bwd", dict(m=1 << 26, classes=1025)),
    ("sb_token_logp_fwd", dict(m=1 << 26, classes=1000)), ("sb_token_logp_bwd", dict(m=1 << 23, classes=1 << 15))])
def test_rows_past_the_lanes_of_a_launch(name, over):
    d = _desc(name, **over)
    assert _call(name, d) == NO
    if CALLS[name][5]:
        assert CALLS[name][5](d) == sb.SIZE_MAX


@pytest.mark.parametrize("name,over", [
    ("sb_embed_bwd", dict(tokens=(1 << 29) - 64)), ("sb_embed_bwd", dict(vocab=(1 << 29) - 1)),
    ("sb_expert_sort", dict(tokens=(1 << 29) - 64, top=1)), ("sb_token_logp_fwd", dict(m=(1 << 29) - 64, classes=8, ldz=8)),
    ("sb_token_logp_fwd", dict(m=(1 << 26) - 64, classes=1025))])
def test_rows_up_to_the_lanes_of_a_launch(name, over):
    assert CALLS[name][5](_desc(name, **over)) != sb.SIZE_MAX


@pytest.mark.parametrize("name", NAMES)
def test_null_descriptor(name):
    _, order, _, _, acc, size = CALLS[name]
    args = [P + i * GAP for i in range(len(order))] + ([0] if acc else []) + ([WS, 1 << 40] if size else [])
    assert getattr(sb.load(), name)(None, *args, None) == BAD


@pytest.mark.parametrize("name,t", [(n, t) for n in NAMES for t in CALLS[n][1] if t not in CALLS[n][3]])
def test_null_tensors(name, t):
    assert _call(name, **{t: None}) == BAD


@pytest.mark.parametrize("name,t", [(n, t) for n in NAMES for t in CALLS[n][1]])
def test_addresses_off_their_elements(name, t):
    at = P + CALLS[name][1].index(t) * GAP
    assert _call(name, **{t: at + 1}) == BAD


@pytest.mark.parametrize("name,a,b", [(n, a, b) for n in NAMES for a in CALLS[n][2] for b in CALLS[n][1] if a != b])
def test_overlaps(name, a, b):
    at = P + CALLS[name][1].index(b) * GAP
    assert _call(name, **{a: at + 16}) == BAD
    if (name, a, b) not in (("sb_token_logp_bwd", "dz", "z"), ("sb_expert_combine", "y", "add")):   # in place
        assert _call(name, **{a: at}) == BAD


@pytest.mark.parametrize("name,t", [(n, t) for n in WITH_WS for t in CALLS[n][1]])
def test_workspace_overlaps(name, t):
    assert _call(name, ws=P + CALLS[name][1].index(t) * GAP) == BAD


@pytest.mark.parametrize("name", WITH_WS)
def test_short_missing_and_unaligned_workspaces(name):
    assert CALLS[name][5](_desc(name)) > 0
    assert _call(name, short=1) == ROOM
    assert _call(name, ws=None) == ROOM
    assert _call(name, ws=WS + 8) == BAD


def test_accumulate_is_a_truth_value():
    assert _call("sb_embed_bwd", accumulate=2) == BAD and _call("sb_embed_bwd", accumulate=-1) == BAD


def test_empty_batches_need_no_tensors():
    lib = sb.load()
    e, x, z = _desc("sb_embed_fwd", tokens=0), _desc("sb_expert_sort", tokens=0), _desc("sb_token_logp_fwd", m=0)
    assert lib.sb_embed_fwd(ctypes.byref(e), None, None, None, None) == sb.SB_OK
    assert lib.sb_embed_bwd(ctypes.byref(e), None, None, P, 1, None, 0, None) == sb.SB_OK
    assert lib.sb_expert_gather(ctypes.byref(x), None, None, None, None) == sb.SB_OK
    assert lib.sb_expert_combine(ctypes.byref(x), None, None, None, None, None, None) == sb.SB_OK
    assert lib.sb_expert_combine_bwd(ctypes.byref(x), None, None, None, None, None, None, None) == sb.SB_OK
    assert lib.sb_token_logp_fwd(ctypes.byref(z), *[None] * 7, None, 0, None) == sb.SB_OK
    assert lib.sb_token_logp_bwd(ctypes.byref(z), *[None] * 11) == sb.SB_OK
    assert sb.sb_token_logp_workspace_bytes(z) == 0


def test_what_goes_together():
    """Targets with their log-probabilities' gradient, entropies with theirs, probabilities with theirs."""
    assert _call("sb_token_logp_fwd", targets=None) == BAD
    for t in ("targets", "entropy", "top_ids", "top_values"):
        assert _call("sb_token_logp_bwd", **{t: None}) == BAD
    assert _call("sb_token_logp_bwd", _desc("sb_token_logp_bwd", top=0)) == BAD
    assert _call("sb_expert_combine_bwd", ys=None) == BAD


def test_bindings_refuse_other_types():
    import torch
    f, h, i = torch.zeros(4), torch.zeros(4).bfloat16(), torch.zeros(4, dtype=torch.int64)
    d, e, z = sb.embed_desc(1, 1, 4), sb.expert_desc(1, 1, 1, 4), sb.token_logp_desc(1, 4)
    for call in (lambda: sb.sb_embed_fwd(d, h, None, f), lambda: sb.sb_embed_fwd(d, f, i, f),
                 lambda: sb.sb_embed_bwd(d, i, f, f), lambda: sb.sb_embed_bwd(d, None, f, h),
                 lambda: sb.sb_expert_sort(e, i, i, i), lambda: sb.sb_expert_gather(e, h, None, f),
                 lambda: sb.sb_expert_combine(e, f, None, h, f),
                 lambda: sb.sb_expert_combine_bwd(e, f, f, None, None, f, h),
                 lambda: sb.sb_token_logp_fwd(z, h, None, None, None, f),
                 lambda: sb.sb_token_logp_bwd(z, f, f, i, f, None, None, None, None, None, f)):
        with pytest.raises(ValueError):
            call()
