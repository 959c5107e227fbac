"""AdamW.step() in a captured graph is refused, and the capture goes on without it."""
import pytest
import torch

from paper_2511_12653_amd import AdamW

pytestmark = pytest.mark.gpu


def test_a_step_is_not_captured():
    p = torch.nn.Parameter(torch.ones(300, device="cuda"))
    opt = AdamW([p], lr=1e-2)
    p.grad = torch.ones(300, device="cuda")
    opt.step()                                       # (the plan is there)
    before, x = p.detach().clone(), torch.ones(300, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = x * 2
        with pytest.raises(RuntimeError, match="captur"):
            opt.step()
    for turn in range(3):
        x.fill_(turn)
        graph.replay()
        torch.cuda.synchronize()
        assert bool((y == 2 * turn).all()) and torch.equal(p.detach(), before)
    assert opt.param_groups[0]["step"] == 1
    opt.step()
    assert opt.param_groups[0]["step"] == 2 and not torch.equal(p.detach(), before)
