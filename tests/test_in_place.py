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


@pytest.mark.gpu
def test_an_out_tensor_is_written_in_place():
    """Whatever a call takes to write its result into counts as modified; what it reads does not."""
    x, dy, w = (torch.randn(s, device="cuda") for s in ((3, 32, 8, 8), (3, 48, 8, 8), (48, 16)))
    kdw, gated = torch.randn(32, 3, 3, device="cuda"), torch.randn(2, 48, 16, device="cuda")

    def room(*shape):
        return torch.empty(shape, device="cuda")

    calls = [(lambda y: S.scc_gated_forward(x, gated, 2, 0.5, out=y), [room(3, 48, 8, 8)]),
             (lambda y: S.scc_forward(x, w, 2, 0.5, out=y), [room(3, 48, 8, 8)]),
             (lambda dx: S.scc_backward_input(dy, w, 32, 2, 0.5, out=dx), [room(3, 32, 8, 8)]),
             (lambda dw: S.scc_backward_weight(x, dy, 2, 0.5, out=dw), [room(48, 16)]),
             (lambda dw: S.scc_backward_weight_static(x, dy, 2, 0.5, dw), [room(48, 16)]),
             (lambda dx, dw: S.scc_backward(x, dy, w, 2, 0.5, out_dx=dx, out_dw=dw), [room(3, 32, 8, 8), room(48, 16)]),
             (lambda dw: S.scc_backward(x, dy, w, 2, 0.5, out_dw=dw), [room(48, 16)]),
             (lambda z: S.scc_depthwise3x3_forward(x, kdw, out=z), [room(3, 32, 8, 8)]),
             (lambda dx, dk: S.scc_depthwise3x3_backward(x, kdw, x, out_dx=dx, out_dk=dk), [room(3, 32, 8, 8), room(32, 3, 3)]),
             (lambda dk: S.scc_depthwise3x3_backward(x, kdw, x, need_dx=False, out_dk=dk), [room(32, 3, 3)]),
             (lambda y: S.scc_dw_forward(x, kdw, w, 2, 0.5, out=y), [room(3, 48, 8, 8)]),
             (lambda y: S.scc_dw_forward(x, kdw, w, 2, 0.5, out=y, fused=False), [room(3, 48, 8, 8)])]
    read = [t._version for t in (x, dy, w, kdw, gated)]
    for call, outs in calls:
        before = [t._version for t in outs]
        call(*outs)
        assert all(t._version > b for t, b in zip(outs, before))
        again = torch.empty_like(outs[0], requires_grad=True)
        kept = (again * outs[0]).sum()
        call(*outs)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            kept.backward()
    assert [t._version for t in (x, dy, w, kdw, gated)] == read
