"""Residual norm, vocabulary loss and AdamW through the native calls and through ctypes: the same results, gradients and errors, and the calls that
are not plain take the second way."""
import pytest
import torch

import paper_2101_00745_amd as S
from paper_2101_00745_amd import nn as N
from paper_2101_00745_amd import scc as B

pytestmark = pytest.mark.gpu
DTYPES = [pytest.param(torch.float32, id="f32"), pytest.param(torch.bfloat16, id="bf16")]


def normal(*shape, dtype=torch.float32, seed=0):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype).cuda()


def both_ways(monkeypatch, call):
    """call() natively and through ctypes."""
    native = call()
    with monkeypatch.context() as m:
        m.setattr(B, "_native", B._NoNative)
        general = call()
    return native, general


def same(a, b):
    assert len(a) == len(b)
    for s, t in zip(a, b):
        assert s.dtype == t.dtype and s.shape == t.shape and torch.equal(s.view(torch.uint8) if s.dtype == torch.float8_e4m3fn else s, t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(20, 64, 1, 1), (2, 33, 5, 3)])
def test_norm(shape, dtype, monkeypatch):
    x, r, dy, dh = (normal(*shape, dtype=dtype, seed=i) for i in range(4))
    w = normal(shape[1], dtype=dtype, seed=5)
    calls = []
    plain = B._load_native()

    class Counting:
        def __getattr__(self, name):
            def call(*args):
                out = getattr(plain, name)(*args)
                calls.append((name, out is not None))
                return out
            return call

    monkeypatch.setattr(B, "_native", Counting())
    for residual in (r, None):
        same(*both_ways(monkeypatch, lambda: S.scc_norm_forward(x, w, residual, 1e-5)))
        same(*both_ways(monkeypatch, lambda: S.scc_norm_quantised(x, w, residual, 1e-5)))

        def train(skip=None, graph=False):
            leaves = [t.clone().requires_grad_(i != skip) for i, t in enumerate((x, w) if residual is None else (x, w, residual))]
            y, h = N.residual_norm(leaves[0], leaves[1], *leaves[2:], eps=1e-5)
            wanted = [t for t in leaves if t.requires_grad]
            outs, ds = ((y, h), (dy, dh)) if residual is not None else ((y,), (dy,))
            return torch.autograd.grad(outs, wanted, ds, create_graph=graph)

        for skip in (None, 0, 1):
            same(*both_ways(monkeypatch, lambda: train(skip)))
        same(*both_ways(monkeypatch, lambda: [g.detach() for g in train(graph=True)]))
    assert ("norm_block", True) in calls and ("norm_block", False) in calls and ("norm_forward", True) in calls and ("norm_quantised", True) in calls
    # one output's gradient alone, from the native block
    leaves = [t.clone().requires_grad_() for t in (x, w, r)]
    y, h = N.residual_norm(leaves[0], leaves[1], leaves[2], eps=1e-5)
    got = torch.autograd.grad(h, leaves, dh, retain_graph=True, allow_unused=True)
    assert torch.equal(got[0], dh) and torch.equal(got[2], dh) and (got[1] == 0).all()
    got = torch.autograd.grad(y, leaves, dy)
    same([got[0], got[2]], [got[2], got[0]])
    # tensors that hooks brought back changed in layout
    with torch.autograd.graph.saved_tensors_hooks(lambda t: t.cpu(), lambda t: t.cuda()):
        y, _ = N.residual_norm(leaves[0], leaves[1], leaves[2], eps=1e-5)
    same(torch.autograd.grad(y, leaves, dy), got)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("reduction", ["mean", "none"])
def test_loss(reduction, dtype, monkeypatch):
    x, w = normal(3, 64, 20, 1, dtype=dtype), normal(300, 64, dtype=dtype, seed=1)
    target = torch.randint(300, (3, 20, 1), device="cuda")
    target[1, 3:9] = -100
    same(*both_ways(monkeypatch, lambda: S.scc_vocabulary_loss(x, w, target, reduction)))

    def train(skip=None, graph=False):
        leaves = [t.clone().requires_grad_(i != skip) for i, t in enumerate((x, w))]
        loss = N.vocabulary_loss(leaves[0], leaves[1], target, reduction)
        return torch.autograd.grad(loss.sum(), [t for t in leaves if t.requires_grad], create_graph=graph)

    for skip in (None, 0, 1):
        same(*both_ways(monkeypatch, lambda: train(skip)))
    same(*both_ways(monkeypatch, lambda: [g.detach() for g in train(graph=True)]))
    assert not N.vocabulary_loss(x, w, target).requires_grad
    with torch.no_grad():
        assert torch.equal(N.vocabulary_loss(x.clone().requires_grad_(), w, target, "sum"), S.scc_vocabulary_loss(x, w, target, "sum")[0])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bits", [8, 32])
def test_adamw(bits, dtype, monkeypatch):
    shapes = [(300,), (20, 33), (2, 3, 5, 7)]

    def steps():
        w, g = ([normal(*s, dtype=dtype, seed=i + 10 * j) for i, s in enumerate(shapes)] for j in range(2))
        if bits == 32:
            m, v, more = [torch.zeros(s, device="cuda") for s in shapes], [torch.zeros(s, device="cuda") for s in shapes], {}
        else:
            m, v = ([torch.zeros(s, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for s in shapes] for _ in range(2))
            scales = [[torch.ones(-(-t.numel() // 256), device="cuda") for t in w] for _ in range(2)]
            more = dict(first_scales=scales[0], second_scales=scales[1], seed=(1 << 63) + 12345)
        versions = [t._version for t in (*w, *m, *v)]
        for step in (1, 2):
            S.scc_adamw_step(w, g, m, v, 0.1, step, betas=(0.8, 0.99), eps=1e-6, weight_decay=0.1, **more)
        assert all(t._version > n for t, n in zip((*w, *m, *v), versions))
        return [*w, *m, *v, *more.get("first_scales", ()), *more.get("second_scales", ())]

    same(*both_ways(monkeypatch, steps))


def test_errors_are_the_same(monkeypatch):
    x, w = normal(2, 8, 1, 1), normal(8)
    v, t = normal(5, 8), torch.zeros(2, 1, 1, dtype=torch.int64, device="cuda")
    ws = [normal(6)]
    ms, vs = [torch.zeros(6, device="cuda")], [torch.zeros(6, device="cuda")]
    for call in (lambda: S.scc_norm_forward(x, w, eps=-1.0), lambda: N.residual_norm(x.clone().requires_grad_(), w.clone().requires_grad_(), eps=-1.0),
                 lambda: S.scc_vocabulary_loss(x, v[:, :7], t), lambda: S.scc_vocabulary_loss(x, v, t[:1]), lambda: N.vocabulary_loss(x, v, t, "median"),
                 lambda: S.scc_adamw_step(ws, ws, ms, vs, 0.1, 1), lambda: S.scc_adamw_step(ws, [normal(6)], ms, vs, 0.1, 0),
                 lambda: S.scc_adamw_step(ws, [normal(7)], ms, vs, 0.1, 1)):
        seen = []
        for native in (True, False):
            with monkeypatch.context() as m:
                if not native:
                    m.setattr(B, "_native", B._NoNative)
                with pytest.raises((ValueError, S.SccError)) as e:
                    call()
                seen.append((type(e.value), str(e.value)))
        assert seen[0] == seen[1]
