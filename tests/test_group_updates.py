"""The updates that a training step of an MP group (stack.GroupTrainStep) enqueues,
from its recorded calls on host tensors: nothing is launched."""
import pytest

from paper_2112_15317_amd import configs, partition as P, sb
from paper_2112_15317_amd.stack import AdamW, AveragedGroups, GroupTrainStep

CONV = configs.PAPER_VARIANT_CONV


@pytest.fixture
def host_tensors(monkeypatch):
    monkeypatch.setattr(sb, "_ptr", lambda t: t if t is None or isinstance(t, int) else t.data_ptr())


def _step(**kw):
    plan = P.fc_plan(P.partition(P.vgg_net(CONV, 3, 32, [(4096, 64), (64, 10)]), 2))
    return GroupTrainStep(CONV, 4, 3, 32, plan, device="cpu", **kw)


def _updates(gs):
    return [(key[0], args) for key, fn, args in gs.step_calls() if fn is sb.sb_sgd_update]


def test_the_rate_is_read_at_every_update(host_tensors):
    gs = _step(lr=0.5)
    for lr in (0.5, 0.25, 0.125):
        gs.lr = lr
        got = _updates(gs)
        assert [name for name, _ in got] == ["sgd_fc", "sgd_fc", "sgd_conv"]
        assert [args[1] for _, args in got] == [lr] * 3


def test_the_lists_of_the_updates_are_attributes(host_tensors):
    gs = _step()
    lists = [args[0] for _, args in _updates(gs)]
    assert lists == [gs.sgd_fc, gs.sgd_fc, gs.sgd_conv]
    assert gs.sgd_fc.count == 4 and gs.sgd_conv.count == 2 * len(gs.conv.layers)


def test_every_parameter_has_random_numbers_of_its_own(host_tensors, monkeypatch):
    """FC shards, conv layers and the groups that are averaged: no two of their
    elements share a number, so no two moments are rounded by the same bits."""
    made = []

    class List:
        def __init__(self, items):
            made.append(items)
    monkeypatch.setattr(sb, "AdamwList", List)
    plan = P.fc_plan(P.partition(P.vgg_net(CONV, 3, 32, [(4096, 64), (64, 10)], gate="silu"), 2))
    ag = AveragedGroups(CONV, 4, 3, 32, plan, 3, 1, device="cpu", adamw=AdamW(moments=8))
    assert len(made) == 6                                # two updates a group
    at = 0
    for it in (it for items in made for it in items):
        assert it["first"] == at
        at += it["w"].numel()
    assert [gs.end for gs in ag.groups] == [at // 3, 2 * at // 3, at]
