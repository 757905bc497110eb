"""The gated layer y = act(SCC(x; w[0])) * SCC(x; w[1]): the formula of its gradient on the CPU (64 bits, against differences), its refusals,
and the kernels against it, path by path.

Bars: those of every other pass, max |err| <= 2e-5 max |ref| in binary32 (sums of at most a few thousand products at 2^-24 each, two factors
and an activation behind them) and 1e-2 in bfloat16 (one rounding of 2^-9 at the end, in the gradients one more in between)."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2101_00745_amd as S
from oracle import scc_oracle as O
from paper_2101_00745_amd import scc as B

TOL = {torch.float32: 2e-5, torch.bfloat16: 1e-2}
DTYPES = [pytest.param(torch.float32, id="f32"), pytest.param(torch.bfloat16, id="bf16")]
ANY, ONE, PRODUCT, DIRECT = 0, 1, 2, 3

erf = np.vectorize(math.erf)


def activation(g, act):
    """act(g) and its derivative, 64 bits."""
    if act == "silu":
        s = 1.0 / (1.0 + np.exp(-g))
        return g * s, s + g * s * (1.0 - s)
    phi = 0.5 * (1.0 + erf(g / math.sqrt(2.0)))
    return g * phi, phi + g * np.exp(-0.5 * g * g) / math.sqrt(2.0 * math.pi)


def reference(x, w, cg, co, act, dy=None):
    g, u = O.forward(x, w[0], cg, co), O.forward(x, w[1], cg, co)
    a, slope = activation(g, act)
    if dy is None:
        return a * u
    dg, du = dy * u * slope, dy * a
    Cin = x.shape[1]
    dx = O.backward_input(dg, w[0], Cin, cg, co) + O.backward_input(du, w[1], Cin, cg, co)
    return a * u, dx, np.stack([O.backward_weight(x, dg, cg, co), O.backward_weight(x, du, cg, co)])


def inputs(shape, dtype, seed=0, relu=False):
    """x, w, dy on the CPU in the storage type, and the same values in 64 bits."""
    N, Cin, Cout, H, W, cg, _ = shape
    rng = np.random.default_rng(8800 + seed)
    L = Cin // cg
    x = rng.standard_normal((N, Cin, H, W))
    ts = [torch.from_numpy(v.astype(np.float32)).to(dtype)
          for v in (np.abs(x) if relu else x, rng.standard_normal((2, Cout, L)) * math.sqrt(2.0 / L), rng.standard_normal((N, Cout, H, W)))]
    return ts, [t.double().numpy() for t in ts]


def off(got, ref):
    got = got.double().cpu().numpy()
    assert got.shape == ref.shape
    return float(np.max(np.abs(got - ref)) / max(np.max(np.abs(ref)), 1e-300))


# (N, Cin, Cout, H, W, cg, co), path in float32, path in bfloat16
SHAPES = [
    ((1, 32, 32, 8, 8, 2, 0.5), DIRECT, DIRECT),
    ((3, 64, 96, 9, 7, 4, 0.5), DIRECT, DIRECT),            # odd planes
    ((2, 128, 100, 7, 7, 2, 0.33), DIRECT, DIRECT),         # fewer filters than windows: holes
    ((4, 30, 61, 5, 5, 2, 0.5), DIRECT, DIRECT),            # channels off the chunks of 8
    ((33, 20, 13, 1, 3, 2, 0.33), DIRECT, DIRECT),          # three pixels
    ((7, 24, 40, 2, 1, 1, 0.5), DIRECT, DIRECT),            # dense, rotated
    ((130, 64, 96, 1, 1, 4, 0.5), DIRECT, DIRECT),          # tokens as rows
    ((45, 36, 50, 1, 1, 3, 0.4), DIRECT, DIRECT),           # tokens of an odd width
    ((1, 512, 64, 2, 2, 8, 0.5), DIRECT, DIRECT),           # four columns
    ((1, 96, 40, 3, 1, 1, 0.0), DIRECT, DIRECT),
    ((2, 200, 70, 1, 1, 2, 0.5), DIRECT, DIRECT),
    ((1, 7, 3, 1, 1, 7, 0.0), ONE, ONE),                    # windows of one channel
    ((1, 1, 1, 1, 1, 1, 1.0), ONE, ONE),
    ((1, 510, 77, 1, 1, 2, 0.33), ONE, ONE),                # a token of an odd width
    ((1, 16000, 9, 1, 1, 2, 0.5), DIRECT, DIRECT),          # ... whose channels do not fit that kernel's LDS
    ((9, 1, 2, 1, 1, 1, 0.0), DIRECT, DIRECT),
    ((5, 6, 17, 2, 2, 2, 0.5), DIRECT, DIRECT),             # fewer channels than a load takes
    ((2, 768, 20, 3, 3, 2, 0.33), DIRECT, DIRECT),          # far fewer filters than windows
    ((2, 16, 5, 300, 1, 1, 1.0), DIRECT, DIRECT),           # a sequence, every filter on the same window
    ((40, 1024, 48, 1, 1, 2, 0.5), DIRECT, DIRECT),
    ((2, 1000, 33, 5, 1, 4, 0.25), DIRECT, DIRECT),
    ((6, 2592, 9, 1, 1, 8, 0.5), DIRECT, DIRECT),
    ((64, 64, 300, 16, 16, 1, 0.5), PRODUCT, PRODUCT),
    ((200, 128, 200, 9, 9, 2, 0.33), PRODUCT, PRODUCT),     # windows anywhere, odd planes, holes
    ((90, 250, 141, 10, 9, 2, 0.5), PRODUCT, PRODUCT),      # channels off the chunks of 8, fewer filters than windows
    ((120, 512, 300, 8, 5, 4, 0.5), PRODUCT, PRODUCT),       # binary32 cut when it is read
    ((1000, 200, 400, 1, 3, 1, 0.33), PRODUCT, PRODUCT),    # three pixels: single columns
    ((4300, 264, 264, 1, 1, 1, 0.33), DIRECT, PRODUCT),
    ((4300, 513, 300, 1, 1, 1, 0.33), DIRECT, PRODUCT),     # tokens of an odd width
    ((4099, 512, 520, 1, 1, 1, 0.5), PRODUCT, PRODUCT),     # tokens as rows
    ((80, 1304, 200, 5, 5, 4, 0.5), ANY, PRODUCT),          # channels that do not fit
    ((40, 2592, 70, 5, 5, 1, 0.5), ANY, ANY),
]
IDS = ["x".join(str(v) for v in s[0]) for s in SHAPES]


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gradient_formula_against_differences(act):
    shape = (2, 12, 10, 3, 2, 2, 0.33)
    _, (x, w, dy) = inputs(shape, torch.float32)
    cg, co = shape[5:]
    _, dx, dw = reference(x, w, cg, co, act, dy)
    rng = np.random.default_rng(1)
    h = 1e-5                                    # error of a central difference: h^2 and 2^-53 / h, some 1e-10 each
    for t, grad in ((x, dx), (w, dw)):
        d = rng.standard_normal(t.shape)
        ends = [float(np.sum(dy * reference(*((t + s * h * d, w) if t is x else (x, t + s * h * d)), cg, co, act))) for s in (1, -1)]
        want = float(np.sum(grad * d))
        assert abs((ends[0] - ends[1]) / (2 * h) - want) <= 1e-7 * max(1.0, abs(want))


@pytest.mark.parametrize("shape,f32,bf16", SHAPES, ids=IDS)
def test_paths(shape, f32, bf16):
    lib = S.load()
    assert lib.scc_gated_forward_path(*shape, 0) == f32
    assert lib.scc_gated_forward_path(*shape, 1) == bf16
    for dtype, path in ((0, f32), (1, bf16)):
        assert (lib.scc_gated_forward_workspace_bytes(*shape, dtype) > 0) == (path == PRODUCT)
        assert lib.scc_gated_backward_workspace_bytes(*shape, dtype, 0) > 0


FAKE = ctypes.c_void_p(0x1000)
BAD = [(dict(N=0), -2), (dict(Cin=-4), -2), (dict(Cout=0), -2), (dict(H=0), -2), (dict(cg=0), -2), (dict(cg=3), -2), (dict(co=-0.01), -3),
       (dict(co=math.nan), -3), (dict(dtype=2), -4), (dict(act=2), -8), (dict(act=-1), -8), (dict(N=1 << 20, H=1 << 10, W=1 << 10), -2),
       (dict(Cin=1 << 12, Cout=1 << 18, cg=1), -2)]      # both halves of the weights pass 32 bits


@pytest.mark.parametrize("over,code", BAD)
def test_invalid_arguments_are_rejected_on_the_host(over, code):
    a = dict(N=2, Cin=8, Cout=6, H=3, W=3, cg=2, co=0.5, act=0, dtype=0)
    a.update(over)
    lib = S.load()
    shape = tuple(a[k] for k in ("N", "Cin", "Cout", "H", "W", "cg", "co"))
    assert lib.scc_gated_forward(FAKE, FAKE, FAKE, *shape, a["act"], a["dtype"], FAKE, 1 << 40, None) == code
    assert lib.scc_gated_backward(FAKE, FAKE, FAKE, FAKE, FAKE, *shape, a["act"], a["dtype"], 0, FAKE, 1 << 40, None) == code
    if "act" not in over:
        assert lib.scc_gated_backward_workspace_bytes(*shape, a["dtype"], 0) == 0
    if "Cout" not in over or a["Cout"] == 0:
        if "act" not in over:
            assert lib.scc_gated_forward_workspace_bytes(*shape, a["dtype"]) == 0


def test_null_pointers_and_workspaces_are_rejected():
    lib = S.load()
    shape = (200, 128, 200, 9, 9, 2, 0.33)
    need, back = lib.scc_gated_forward_workspace_bytes(*shape, 0), lib.scc_gated_backward_workspace_bytes(*shape, 0, 1)
    for i in range(3):
        ptrs = [FAKE] * 3
        ptrs[i] = None
        assert lib.scc_gated_forward(*ptrs, *shape, 0, 0, FAKE, need, None) == -1
    for i in range(5):
        ptrs = [FAKE] * 5
        ptrs[i] = None
        assert lib.scc_gated_backward(*ptrs, *shape, 0, 0, 1, FAKE, back, None) == -1
    odd = ctypes.c_void_p(0x1010)
    for ws, size in ((None, 0), (FAKE, need - 1), (odd, need)):
        assert lib.scc_gated_forward(FAKE, FAKE, FAKE, *shape, 0, 0, ws, size, None) == -5
    for ws, size in ((None, 0), (FAKE, back - 1), (odd, back)):
        assert lib.scc_gated_backward(FAKE, FAKE, FAKE, FAKE, FAKE, *shape, 0, 0, 1, ws, size, None) == -5
    assert lib.scc_gated_backward(FAKE, FAKE, FAKE, FAKE, FAKE, *shape, 0, 0, 2, FAKE, back, None) == -4     # grad is no type


def test_binding_refuses():
    x, w = torch.zeros(1, 4, 2, 2), torch.zeros(2, 4, 2)
    with pytest.raises(ValueError):
        S.scc_gated_forward(x, w, 2, 0.5)                   # no CPU path
    with pytest.raises(ValueError):
        S.scc_gated_forward(x, w, 2, 0.5, act="tanh")
    with pytest.raises(ValueError):
        S.scc_gated_backward(x, w, x, 2, 0.5)


@pytest.mark.gpu
def test_binding_refuses_on_the_gpu():
    x, w = torch.zeros(1, 4, 2, 2, device="cuda"), torch.zeros(2, 6, 2, device="cuda")
    for bad in (w[0], w.bfloat16(), torch.zeros(3, 6, 2, device="cuda"), torch.zeros(2, 6, 3, device="cuda"), w.transpose(1, 2)):
        with pytest.raises(ValueError):
            S.scc_gated_forward(x, bad, 2, 0.5)
    with pytest.raises(ValueError):
        S.scc_gated_forward(x[0], w, 2, 0.5)
    with pytest.raises(ValueError):
        S.scc_gated_forward(x.transpose(2, 3)[:, ::2], w, 2, 0.5)
    with pytest.raises(ValueError):
        S.scc_gated_forward(x, w, 2, 0.5, out=torch.zeros(1, 5, 2, 2, device="cuda"))
    with pytest.raises(ValueError):
        S.scc_gated_backward(x, w, torch.zeros(1, 5, 2, 2, device="cuda"), 2, 0.5)
    with pytest.raises(B.SccError):
        S.scc_gated_forward(x, w, 2, 1.5)
    with pytest.raises(TypeError):
        S.scc_gated_forward(x.double(), w.double(), 2, 0.5)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape,f32,bf16", SHAPES, ids=IDS)
def test_forward_and_gradients(shape, f32, bf16, dtype):
    cg, co = shape[5:]
    for act in ("silu", "gelu"):
        (x, w, dy), wide = inputs(shape, dtype, seed=len(act), relu=act == "gelu")
        y, dx, dw = reference(wide[0], wide[1], cg, co, act, wide[2])
        xd, wd, dyd = x.cuda(), w.cuda(), dy.cuda()
        assert off(S.scc_gated_forward(xd, wd, cg, co, act=act), y) <= TOL[dtype]
        got = S.scc_gated_backward(xd, wd, dyd, cg, co, act=act)
        assert got[0].dtype == dtype and got[1].dtype == torch.float32
        assert off(got[0], dx) <= TOL[dtype]
        assert off(got[1], dw) <= TOL[dtype]
        again = S.scc_gated_backward(xd, wd, dyd, cg, co, act=act)
        assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])
        kept = B._gated_backward(xd, wd, dyd, cg, co, act, True)
        assert kept[1].dtype == dtype and torch.equal(kept[1], got[1].to(dtype)) and torch.equal(kept[0], got[0])


@pytest.mark.gpu
def test_float32_keeps_float32_accuracy():
    """Six of nine partial products: the error stays at binary32's rounding, not at bfloat16's (2-norm, some 2^-24 sqrt(L))."""
    for shape in ((8, 256, 128, 8, 8, 1, 0.5), (96, 512, 64, 1, 1, 2, 0.5), (2, 1024, 64, 6, 6, 2, 0.5)):
        (x, w, dy), wide = inputs(shape, torch.float32, seed=5)
        refs = reference(wide[0], wide[1], *shape[5:], "silu", wide[2])
        got = (S.scc_gated_forward(x.cuda(), w.cuda(), *shape[5:]), *S.scc_gated_backward(x.cuda(), w.cuda(), dy.cuda(), *shape[5:]))
        for g, r in zip(got, refs):
            assert np.linalg.norm(g.double().cpu().numpy() - r) <= 2e-6 * np.linalg.norm(r)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_odd_addresses(dtype):
    """Tensors that begin an element behind an aligned address."""
    for shape in ((3, 64, 48, 5, 5, 2, 0.5), (50, 64, 48, 1, 1, 2, 0.5), (2, 64, 48, 1, 1, 2, 0.5)):
        (x, w, dy), wide = inputs(shape, dtype, seed=3)

        def shifted(t):
            room = torch.empty(t.numel() + 1, dtype=dtype, device="cuda")
            room[1:].copy_(t.flatten())
            return room[1:].view(t.shape)

        y, dx, dw = reference(wide[0], wide[1], 2, 0.5, "silu", wide[2])
        args = [shifted(t) for t in (x, w, dy)]
        out = shifted(torch.zeros(y.shape, dtype=dtype))
        S.scc_gated_forward(args[0], args[1], 2, 0.5, out=out)
        assert off(out, y) <= TOL[dtype]
        got = S.scc_gated_backward(*args, 2, 0.5)
        assert off(got[0], dx) <= TOL[dtype] and off(got[1], dw) <= TOL[dtype]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(4, 64, 48, 5, 5, 4, 0.5), (40, 64, 48, 1, 1, 4, 0.5), (3, 64, 48, 1, 1, 4, 0.5)])
def test_infinities_stay_with_their_pixel(shape, dtype):
    (x, w, _), wide = inputs(shape, dtype, seed=4)
    x = x.clone()
    x[1, 3, 0, 0], x[2, 9, -1, -1] = math.inf, math.nan
    y = S.scc_gated_forward(x.cuda(), w.cuda(), 4, 0.5).double().cpu().numpy()
    ref = reference(wide[0], wide[1], 4, 0.5, "silu")
    hit = np.zeros(ref.shape, dtype=bool)
    hit[1, :, 0, 0] = hit[2, :, -1, -1] = True
    assert np.max(np.abs(y - ref)[~hit]) <= TOL[dtype] * np.max(np.abs(ref))
    reached = np.isnan(O.forward(np.where(np.isfinite(x.double().numpy()), 0.0, np.nan), np.ones_like(wide[1][0]), 4, 0.5))
    assert not np.isfinite(y[reached]).any()


@pytest.mark.gpu
def test_large_values_of_the_gate():
    """act is 0 far below zero and the identity far above; nothing in between overflows."""
    for act in ("silu", "gelu"):
        x = torch.tensor([-3e4, -200.0, -88.0, 0.0, 88.0, 200.0, 3e4], device="cuda").view(7, 1, 1, 1)
        w = torch.tensor([[[1.0]], [[0.5]]], device="cuda")
        y = S.scc_gated_forward(x, w, 1, 0.0, act=act).flatten()
        dx, _ = S.scc_gated_backward(x, w, torch.ones_like(x), 1, 0.0, act=act)
        assert torch.equal(y[3:], torch.tensor([0.0, 3872.0, 2e4, 4.5e8], device="cuda"))
        assert y[:3].abs().max() <= 1e-30
        assert torch.allclose(dx.flatten()[[0, 1, 4, 5, 6]], torch.tensor([0.0, 0.0, 88.0, 200.0, 3e4], device="cuda"), rtol=1e-5, atol=1e-30)


@pytest.mark.gpu
def test_module_trains_under_autograd_and_on_a_stream():
    from paper_2101_00745_amd.nn import GatedFeedForward, GatedSCC, gated_scc
    shape = (5, 32, 40, 4, 3, 2, 0.5)
    (x, w, dy), wide = inputs(shape, torch.float32, seed=6)
    y, dx, dw = reference(wide[0], wide[1], 2, 0.5, "gelu", wide[2])
    m = GatedSCC(32, 40, cg=2, co=0.5, act="gelu")
    with torch.no_grad():
        m.weight.copy_(w)
    stream = torch.cuda.Stream()
    xd = x.cuda().requires_grad_(True)
    dyd = dy.cuda().transpose(2, 3).contiguous().transpose(2, 3)        # strides of its own
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        out = m(xd)
        out.backward(dyd)
    stream.synchronize()
    assert off(out.detach(), y) <= 2e-5 and off(xd.grad, dx) <= 2e-5 and off(m.weight.grad, dw) <= 2e-5
    only = gated_scc(x.cuda(), m.weight, 2, 0.5, act="gelu")
    m.weight.grad = None
    only.backward(dyd)
    assert off(m.weight.grad, dw) <= 2e-5
    with pytest.raises(RuntimeError, match="second derivative"):
        g, = torch.autograd.grad(gated_scc(xd, m.weight, 2, 0.5).sum(), xd, create_graph=True)
        g.sum().backward()
    block = GatedFeedForward(32, 64)
    assert block(xd).shape == xd.shape


@pytest.mark.gpu
def test_captured_graph():
    shape = (6, 64, 96, 7, 7, 2, 0.5)
    (x, w, dy), _ = inputs(shape, torch.bfloat16, seed=7)
    x, w, dy = x.cuda(), w.cuda(), dy.cuda()

    def step():
        return (S.scc_gated_forward(x, w, 2, 0.5), *S.scc_gated_backward(x, w, dy, 2, 0.5))

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for i in range(4):
        x.copy_(x * 0.5 + 0.25)
        want = [t.clone() for t in step()]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs, want))
