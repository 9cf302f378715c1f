"""A step's number and seed are arguments: recorded into a graph, every replay would be the same step."""
import pytest
import torch

import paper_2202_00774_amd as sdgp
from paper_2202_00774_amd.optim import AdamW

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 32])
def test_a_step_is_not_recorded_into_a_graph(bits):
    p, x = torch.zeros(700, device="cuda"), torch.ones(700, device="cuda")
    g = torch.ones(700, device="cuda")
    opt = AdamW([p], state_bits=bits, lr=0.5, weight_decay=0.0)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        y = x * 2
        with pytest.raises(sdgp.SdgpError, match="captured") as e:
            opt.step([g])
    assert e.value.status == -8 and opt.steps == 0
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    assert (y == 2).all() and (p == 0).all() and all((t.float() == 0).all() for t in opt.state()["exp_avg"])
    opt.step([g])                                # the optimizer goes on beside the graph
    assert opt.steps == 1 and ((p + 0.5).abs() <= 1e-6).all()
