"""Calls that write tensors of the caller's tell autograd so, one that fails is not made again, and one that would write memory twice not at all."""

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


class Recorder:
    """In the native module's place: one call answers what it is told to."""

    def __init__(self, answer):
        self.answer, self.calls = answer, 0

    def orthogonal_step(self, *args):
        self.calls += 1
        return self.answer


def test_a_step_that_failed_is_not_made_again(monkeypatch):
    """A list of more matrices than a launch takes may have moved in part; the general way would move that part once more."""
    def again(*args):
        raise AssertionError("the call was made a second time")

    monkeypatch.setattr(B, "_orthogonal", again)
    m = torch.zeros(4, 4)
    for status in (-6, -8):
        native = Recorder(status)
        monkeypatch.setattr(B, "_native", native)
        with pytest.raises(B.SccError) as e:
            S.scc_orthogonal_step([m], [m], [m], lr=0.1)
        assert e.value.status == status and native.calls == 1
    monkeypatch.setattr(B, "_native", Recorder(0))
    S.scc_orthogonal_step([m], [m], [m], lr=0.1)


@pytest.mark.gpu
def test_the_native_step_answers_its_status(monkeypatch):
    def again(*args):
        raise AssertionError("the call was made a second time")

    w, g, m = (torch.ones(4, 6, device="cuda") for _ in range(3))
    with monkeypatch.context() as patch:
        patch.setattr(B, "_orthogonal", again)
        with pytest.raises(B.SccError) as e:
            S.scc_orthogonal_step([w], [g], [m], lr=0.1, steps=101)
        assert e.value.status == -8
        S.scc_orthogonal_step([w], [g], [m], lr=0.1)
    with pytest.raises(ValueError):             # not a plain call: the general way says what is wrong with it
        S.scc_orthogonal_step([w.t()], [g.t()], [m.t()], lr=0.1)


@pytest.mark.gpu
def test_the_general_way_raises_versions_where_something_may_have_moved(monkeypatch):
    monkeypatch.setattr(B, "_native", B._NoNative)
    w, g, m = (torch.ones(4, 6, device="cuda") for _ in range(3))
    for status, raised in ((-6, 1), (-8, 0)):
        def fail(*args):
            raise B.SccError(status, "")

        with monkeypatch.context() as patch:
            patch.setattr(B, "_orthogonal", fail)
            before = [t._version for t in (w, g, m)]
            with pytest.raises(B.SccError):
                S.scc_orthogonal_step([w], [g], [m], lr=0.1)
        assert [t._version - b for t, b in zip((w, g, m), before)] == [raised, 0, raised]


def test_memory_that_would_be_written_twice():
    """The matrices of a list are moved at the same time, by different workgroups."""
    a, b, c, d = (torch.zeros(6, 8) for _ in range(4))
    stack = torch.zeros(3, 6, 8)
    assert not B._overlap([a, b], [c, d]) and not B._overlap([a], [c, c]) and not B._overlap([], [c, c])
    assert not B._overlap([stack[0], stack[2]], [stack[1]])             # neighbours
    for written, read in (([a, a], []), ([a], [a]), ([a, stack.flatten()[40:100]], [stack[1]]), ([stack[1]], [a, stack]), ([stack], [stack[2, 5:]]),
                          ([stack[0], b, stack.flatten()[47:60]], [])):
        assert B._overlap(written, read)


@pytest.mark.gpu
@pytest.mark.parametrize("name", ROUTES)
def test_shared_memory_is_refused(name, monkeypatch):
    from paper_2101_00745_amd.optim import OrthogonalMomentum
    route(name, monkeypatch)
    w, v, g, m, n = (torch.ones(4, 6, device="cuda") for _ in range(5))
    for lists in (([w, w], [g, g], [m, n]), ([w, v], [g, g], [m, m]), ([w], [w], [m]), ([w], [g], [g]), ([w], [g], [w])):
        with pytest.raises(ValueError, match="share memory"):
            S.scc_orthogonal_step(*lists, lr=0.1)
    S.scc_orthogonal_step([w, v], [g, g], [m, n], lr=0.1)               # one gradient, read twice
    p = torch.nn.Parameter(torch.ones(4, 6, device="cuda"))
    p.grad = g
    with pytest.warns(UserWarning, match="duplicate"):
        opt = OrthogonalMomentum([p, p])
    with pytest.raises(ValueError, match="share memory"):
        opt.step()
