"""Calls that write tensors of the caller's tell autograd so."""

import pytest
import torch

import paper_2101_00745_amd as S
from paper_2101_00745_amd import scc as B

ROUTES = ["native", "general"]


def route(name, monkeypatch):
    if name == "general":
        monkeypatch.setattr(B, "_native", B._NoNative)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ROUTES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_a_step_raises_the_versions_of_what_it_moves(name, dtype, monkeypatch):
    route(name, monkeypatch)
    ws, gs = [[torch.randn(s, device="cuda").to(dtype) for s in ((40, 24), (200, 130))] for _ in range(2)]
    ms = [torch.zeros_like(w, dtype=torch.float32) for w in ws]
    before = [[t._version for t in l] for l in (ws, gs, ms)]
    S.scc_orthogonal_step(ws, gs, ms, lr=0.1)
    after = [[t._version for t in l] for l in (ws, gs, ms)]
    assert after[1] == before[1]
    for i in (0, 2):
        assert all(a > b for a, b in zip(after[i], before[i]))
    with torch.inference_mode():            # tensors without a version
        ws, gs, ms = [[t.clone() for t in l] for l in (ws, gs, ms)]
        S.scc_orthogonal_step(ws, gs, ms, lr=0.1)
    S.scc_orthogonal_step(ws, gs, ms, lr=0.1)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ROUTES)
def test_a_graph_over_moved_weights_is_an_error(name, monkeypatch):
    """The gated layer computes its projections again from the weights it saved: with others its gradients would be of neither."""
    from paper_2101_00745_amd.nn import GatedFeedForward
    from paper_2101_00745_amd.optim import OrthogonalMomentum
    route(name, monkeypatch)
    block = GatedFeedForward(32, 64)
    opt = OrthogonalMomentum(block.parameters(), lr=0.1)
    x = torch.randn(4, 32, 3, 3, device="cuda", requires_grad=True)
    loss = block(x).square().sum()
    loss.backward(retain_graph=True)
    opt.step()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    block(x).sum().backward()               # a new graph is fine
