"""Residual norm and vocabulary loss under what is not a plain call: functional transforms, forward mode, tracing, torch.compile, saved-tensor hooks, checkpoints;
and what is said of a second derivative."""
import pytest
import torch

from paper_2101_00745_amd import nn as N

pytestmark = pytest.mark.gpu
DTYPES = [pytest.param(torch.float32, id="f32"), pytest.param(torch.bfloat16, id="bf16")]


def tensors(dtype=torch.float32):
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, r = (torch.randn(6, 64, 5, 1, generator=gen, device="cuda").to(dtype) for _ in range(2))
    w, head = (torch.randn(*s, generator=gen, device="cuda").to(dtype) for s in ((64,), (200, 64)))
    target = torch.randint(200, (6, 5, 1), generator=gen, device="cuda")
    return [t.requires_grad_() for t in (x, r, w, head)] + [target]


def both(x, r, w, head, target):
    """A norm whose y goes into the loss, and its h."""
    y, h = N.residual_norm(x, w, r)
    return N.vocabulary_loss(y, head, target) + h.float().mean()


def grads(f, x, r, w, head, target):
    out = f(x, r, w, head, target)
    return [out.detach(), *torch.autograd.grad(out, (x, r, w, head))]


def same(a, b):
    assert len(a) == len(b) and all(s.dtype == t.dtype and torch.equal(s, t) for s, t in zip(a, b))


def test_functional_transforms_and_forward_mode_are_refused():
    x, r, w, head, target = (t.detach() for t in tensors())
    for call in (lambda t: N.residual_norm(t, w, r)[0].sum(), lambda t: N.residual_norm(t, w)[0].sum(), lambda t: N.vocabulary_loss(t, head, target)):
        with pytest.raises(RuntimeError):
            torch.func.grad(call)(x)
        with pytest.raises(RuntimeError):
            torch.func.vmap(call)(x[None])
        with torch.autograd.forward_ad.dual_level(), pytest.raises(RuntimeError):
            call(torch.autograd.forward_ad.make_dual(x, torch.ones_like(x)))
        leaf = x.clone().requires_grad_()
        with torch.autograd.forward_ad.dual_level(), pytest.raises(RuntimeError):
            call(torch.autograd.forward_ad.make_dual(leaf, torch.ones_like(x)))


@pytest.mark.parametrize("dtype", DTYPES)
def test_compiled(dtype):
    """torch.compile leaves the calls as they are."""
    t = tensors(dtype)
    want = grads(both, *t)
    compiled = torch.compile(both, backend="eager")
    for _ in range(2):
        same(grads(compiled, *t), want)


@pytest.mark.parametrize("dtype", DTYPES)
def test_traced(dtype):
    t = tensors(dtype)
    want = both(*t).detach()
    traced = torch.jit.trace(both, tuple(a.detach() for a in t), check_trace=False)
    assert torch.equal(traced(*(a.detach() for a in t)), want)


@pytest.mark.parametrize("dtype", DTYPES)
def test_hooks_and_checkpoints(dtype):
    t = tensors(dtype)
    want = grads(both, *t)
    with torch.autograd.graph.saved_tensors_hooks(lambda s: s.cpu(), lambda s: s.cuda()):
        out = both(*t)
    same([out.detach(), *torch.autograd.grad(out, t[:4])], want)
    same(grads(lambda *a: torch.utils.checkpoint.checkpoint(both, *a, use_reentrant=False), *t), want)
    with torch.autograd.graph.saved_tensors_hooks(lambda s: s, lambda s: s.transpose(0, 1).contiguous().transpose(0, 1) if s.dim() > 1 else s):
        out = both(*t)
    with pytest.raises(ValueError, match="contiguous"):
        torch.autograd.grad(out, t[:4])


@pytest.mark.parametrize("native", [True, False])
def test_what_is_said_of_a_second_derivative(native, monkeypatch):
    """It names no operator of another kind."""
    if not native:
        monkeypatch.setattr(N._scc, "_native", N._scc._NoNative)
    x, r, w, head, target = tensors()
    for out, wanted in ((N.residual_norm(x, w, r)[0], (x, r, w)), (N.residual_norm(x, w)[0], (x, w)), (N.vocabulary_loss(x, head, target), (x, head)),
                        (N.gated_scc(x, head.view(2, 100, 64)[:, :, :32].contiguous(), 2, 0.5), (x,))):
        for g in torch.autograd.grad(out.sum(), wanted, create_graph=True):
            with pytest.raises(RuntimeError, match="has no second derivative") as e:
                g.sum().backward(retain_graph=True)
            assert "sliding" not in str(e.value)
