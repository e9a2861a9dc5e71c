"""sb.AdamwList with its plan on another stream than the current one."""
import numpy as np
import pytest
import torch

from paper_2112_15317_amd import sb
from tests.helpers import print_case
from tests.test_gpu_adamw import B1, B2, EPS, LR, _check_w, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("number", [False, True])
def test_work_that_still_runs_does_not_reach_the_plan(number):
    """Memory of a plan's size is freed with work on it still to come on the current
    stream, and the list is made on another stream: its plan is not that memory."""
    print_case("adamw_plan_stream", number=number)
    n = 5000
    w, g, m, v = _inputs(n, 3)
    t = [torch.from_numpy(x).cuda() for x in (w, g, m, v)]
    s = torch.cuda.Stream()
    need = sb.load().sb_adamw_plan_bytes(1)
    torch.cuda.synchronize()
    busy = torch.ones(4096, 4096, device="cuda")
    old = torch.empty((need,), dtype=torch.uint8, device="cuda")
    for _ in range(20):
        busy = busy @ busy * 1e-4
    old.fill_(255)
    at = old.data_ptr()
    del old
    lst = sb.AdamwList([dict(zip("wgmv", t))], stream=s.cuda_stream if number else s)
    assert lst.plan.data_ptr() != at
    before = lst.plan.cpu()
    torch.cuda.synchronize()
    assert torch.equal(lst.plan.cpu(), before) and not bool((before == 255).all())
    for stream in (s, None):
        for a, b in zip(t, (w, g, m, v)):
            a.copy_(torch.from_numpy(b))
        torch.cuda.synchronize()
        sb.sb_adamw_update(lst, LR, B1, B2, EPS, step=2, stream=stream)
        torch.cuda.synchronize()
        _check_w(t[0].cpu().numpy(), w, g, m, v, 2, 1.0, 0.0)


def test_a_list_made_inside_a_capture():
    """On the captured stream; a stream outside the capture is refused, which leaves
    the capture as it was."""
    print_case("adamw_plan_capture")
    n = 3000
    w, g, m, v = _inputs(n, 4)
    t = [torch.from_numpy(x).cuda() for x in (w, g, m, v)]
    other = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        with pytest.raises(ValueError):
            sb.AdamwList([dict(zip("wgmv", t))], stream=other)
        lst = sb.AdamwList([dict(zip("wgmv", t))])
        sb.sb_adamw_update(lst, LR, B1, B2, EPS, step=2)
    for _ in range(3):
        for a, b in zip(t, (w, g, m, v)):
            a.copy_(torch.from_numpy(b))
        graph.replay()
        torch.cuda.synchronize()
        _check_w(t[0].cpu().numpy(), w, g, m, v, 2, 1.0, 0.0)
        assert np.array_equal(t[1].cpu().numpy(), g)
