"""AveragedGroups with AdamW on unlike data: what the averages give, and that each
group's moments stay its own."""
import pytest
import torch

from paper_2112_15317_amd.stack import AdamW, AveragedGroups, GroupTrainStep
from tests.helpers import print_case
from tests.test_gpu_gated_group import CONV, OPT, _inputs, _plan

pytestmark = pytest.mark.gpu


def _params(gs):
    return list(gs.conv.W) + list(gs.conv.b) + list(gs.W) + list(gs.b)


def _moments(gs):
    return [m[key] for u in (gs.update_fc, gs.update_conv) for m in u.moments for key in sorted(m)]


@pytest.mark.parametrize("moments", [32, 8])
def test_groups_on_unlike_data_are_averaged(moments):
    K, n, fc = 2, 4, [(4096, 64), (64, 10)]
    print_case("gated_averaged_unlike", moments=moments)
    opt = AdamW(moments=moments, seed=9, **OPT)
    _, x, cw, cb, fw, fb, _, remote, labels = _inputs(K, n, fc, "silu", 6)
    _, x2, _, _, _, _, _, remote2, labels2 = _inputs(K, n, fc, "silu", 7)
    data = [(x, remote, labels), (x2, remote2, labels2)]
    ag = AveragedGroups(CONV, n, 3, 32, _plan(fc, K, "silu"), 2, 2, adamw=opt)
    ag.load_inputs(data, cw, cb, fw, fb)
    own = []
    for d, gs in zip(data, ag.groups):
        first = own[-1].end if own else 0
        own.append(GroupTrainStep(CONV, n, 3, 32, _plan(fc, K, "silu"), adamw=opt, first=first))
        own[-1].load_inputs(d[0], cw, cb, fw, fb, d[1], d[2])
    # A step without averaging: each group as by itself, and unlike the other.
    ag.step()
    for gs in own:
        gs.step()
    torch.cuda.synchronize()
    for gs, one in zip(ag.groups, own):
        for a, b in zip(_params(gs) + _moments(gs), _params(one) + _moments(one)):
            assert torch.equal(a, b)
    assert all(not torch.equal(a, b) for a, b in zip(_params(ag.groups[0]), _params(ag.groups[1])))
    # The second one averages: the mean of the two, the moments as without it.
    ag.step()
    for gs in own:
        gs.step()
    torch.cuda.synchronize()
    for a, b, p, q in zip(_params(ag.groups[0]), _params(ag.groups[1]), _params(own[0]), _params(own[1])):
        assert torch.equal(a, b)
        mean = (p.double() + q.double()) / 2
        # A sum and a product in fp32, half a step each.
        lim = 2.0 ** -24 * (p.double() + q.double()).abs() + 2.0 ** -24 * mean.abs()
        assert bool(((a.double() - mean).abs() <= lim).all())
        assert not torch.equal(p, q)
    for gs, one in zip(ag.groups, own):
        for a, b in zip(_moments(gs), _moments(one)):
            assert torch.equal(a, b)
    assert any(not torch.equal(a, b) for a, b in zip(_moments(ag.groups[0]), _moments(ag.groups[1])))
