"""Which parameters OrthogonalMomentum takes: matrices and stacks of them, and nothing that only looks like one."""
import pytest
import torch

from paper_2101_00745_amd import nn
from paper_2101_00745_amd.optim import OrthogonalMomentum


def test_depthwise_filters_are_refused():
    block = nn.DWSCCBlock(32, 64, device="cpu")
    with pytest.raises(ValueError, match="depthwise"):
        OrthogonalMomentum(block.parameters())
    OrthogonalMomentum([p for p in block.parameters() if p is not block.dw_weight])


@pytest.mark.parametrize("bad", [(7,), (2, 3, 4, 5), (), (64, 3, 3), (2, 3, 3)])
def test_groups_that_come_later_are_looked_at_too(bad):
    first = torch.nn.Parameter(torch.zeros(8, 4))
    opt = OrthogonalMomentum([first], lr=0.1)
    good = torch.nn.Parameter(torch.zeros(2, 8, 4))
    for params in ([torch.nn.Parameter(torch.zeros(bad))], [good, torch.nn.Parameter(torch.zeros(bad))], torch.nn.Parameter(torch.zeros(bad))):
        with pytest.raises(ValueError):
            opt.add_param_group({"params": params, "lr": 0.5})
        assert len(opt.param_groups) == 1 and opt.param_groups[0]["params"] == [first]
        with pytest.raises(ValueError):
            OrthogonalMomentum([{"params": [first]}, {"params": params}])
    opt.add_param_group({"params": [good, torch.nn.Parameter(torch.zeros(3, 8, 4))], "lr": 0.5})
    assert len(opt.param_groups) == 2 and opt.param_groups[1]["lr"] == 0.5 and opt.param_groups[1]["momentum"] == 0.95


def test_every_matrix_of_the_modules_is_taken():
    block = nn.GatedFeedForward(32, 64, device="cpu")
    OrthogonalMomentum(list(block.parameters()) + [nn.SCC(8, 6, device="cpu").weight])
