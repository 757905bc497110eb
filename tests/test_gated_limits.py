"""The gated layer where its kernels' ranges end, its activation by itself, and layers of which one gradient is wanted.

Bars as in the layer's other tests: 2e-5 and 1e-2 of the largest value; the activation's is the one that its comment states."""
import math

import numpy as np
import pytest
import torch

import paper_2101_00745_amd as S
from paper_2101_00745_amd import scc as B
from tests.test_gated import ANY, DIRECT, DTYPES, PRODUCT, TOL, inputs, off, reference

# (N, Cin, Cout, H, W, cg, co) with Cin / gcd(stride, Cin) windows, more than 65536: index times inverse leaves 32 bits
MANY_WINDOWS = [(1, 90000, 64, 1, 1, 2000, 0.5), (3, 90000, 70, 1, 1, 2000, 0.5), (2, 131074, 40, 2, 1, 65537, 0.5), (5, 70000, 33, 1, 1, 7000, 0.1)]


def windows(Cin, Cout, cg, co):
    """Starts of a window that more and more filters would have; scc_window_params counts those of the filters that there are."""
    return Cin // math.gcd(S.scc_window_params(Cin, Cout, cg, co)[1], Cin)


@pytest.mark.parametrize("shape", MANY_WINDOWS)
@pytest.mark.parametrize("dtype", [0, 1])
def test_layers_of_many_windows_take_the_plain_kernel(shape, dtype):
    N, Cin, Cout, H, W, cg, co = shape
    assert windows(Cin, Cout, cg, co) > 65536
    assert S.load().scc_gated_forward_path(*shape, dtype) == ANY


def test_no_direct_layer_has_more_windows_than_its_rows_are_found_for():
    """The kernel finds a row's filter by (m * inv) mod P in 32 bits, m and inv below P; of layers whose rows are the filters in their own order
    it does not look for it."""
    rng = np.random.default_rng(3)
    lib, met = S.load(), 0
    for _ in range(4000):
        cg = int(rng.integers(1, 5000))
        Cin = cg * int(rng.integers(1, 200))
        Cout, N = int(rng.integers(1, 300)), int(rng.integers(1, 40))
        co = float(rng.choice([0.0, 0.25, 0.33, 0.5]))
        if lib.scc_gated_forward_path(N, Cin, Cout, 1, 1, cg, co, int(rng.integers(2))) != DIRECT:
            continue
        L, P = Cin // cg, windows(Cin, Cout, cg, co)
        F = -(-Cout // P)
        span = min(Cin, L + Cin // P * ((14 + F) // F))
        own_order = -(-Cout // 16) * Cin < -(-P * F // 16) * span
        assert own_order or (P - 1) * (P - 1) < 1 << 32, (N, Cin, Cout, cg, co)
        met += not own_order and P > 32768
    assert met > 20


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", MANY_WINDOWS)
def test_layers_of_many_windows(shape, dtype):
    cg, co = shape[5:]
    (x, w, dy), wide = inputs(shape, dtype, seed=11)
    y, dx, dw = reference(wide[0], wide[1], cg, co, "silu", wide[2])
    assert off(S.scc_gated_forward(x.cuda(), w.cuda(), cg, co), y) <= TOL[dtype]
    got = S.scc_gated_backward(x.cuda(), w.cuda(), dy.cuda(), cg, co)
    assert off(got[0], dx) <= TOL[dtype] and off(got[1], dw) <= TOL[dtype]


@pytest.mark.parametrize("dtype,most", [(0, 1240), (1, 2480)])
def test_most_channels_of_the_packed_product(dtype, most):
    """32 columns of all channels in 160 KB: chunks of 8 channels, 33 columns of 16 bytes each, binary32 whole as two."""
    assert most == 8 * ((160 << 10) // (33 * (32, 16)[dtype]))
    lib = S.load()
    for channels, path in ((most, PRODUCT), (most + 8, ANY)):
        assert lib.scc_gated_forward_path(200, channels, 512, 8, 8, 1, 0.5, dtype) == path


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,most", [pytest.param(torch.float32, 1240, id="f32"), pytest.param(torch.bfloat16, 2480, id="bf16")])
def test_layers_on_both_sides_of_the_packed_product(dtype, most):
    for channels in (most, most + 8):
        shape = (120, channels, 100, 5, 5, 1, 0.5)
        path = S.load().scc_gated_forward_path(*shape, int(dtype == torch.bfloat16))
        assert path == (PRODUCT if channels == most else ANY)
        (x, w, dy), wide = inputs(shape, dtype, seed=12)
        y, dx, dw = reference(wide[0], wide[1], 1, 0.5, "gelu", wide[2])
        assert off(S.scc_gated_forward(x.cuda(), w.cuda(), 1, 0.5, act="gelu"), y) <= TOL[dtype]
        got = S.scc_gated_backward(x.cuda(), w.cuda(), dy.cuda(), 1, 0.5, act="gelu")
        assert off(got[0], dx) <= TOL[dtype] and off(got[1], dw) <= TOL[dtype]


@pytest.mark.gpu
def test_error_of_the_gelu():
    """g Phi(g) in binary32 is off by 4e-7 at most.  Two channels, g and 1, which the two projections pick: their products with 1 and 0 and the
    sums of those are exact, and so is the product with 1."""
    g = torch.linspace(-12.0, 12.0, 40001)
    x = torch.stack([g, torch.ones_like(g)], 1)[:, :, None, None].contiguous()
    w = torch.tensor([[[1.0, 0.0]], [[0.0, 1.0]]])
    y = S.scc_gated_forward(x.cuda(), w.cuda(), 1, 1.0, act="gelu").flatten().double().cpu().numpy()
    want = np.array([v * 0.5 * math.erfc(-v / math.sqrt(2.0)) for v in g.double().tolist()])
    assert np.max(np.abs(y - want)) <= 4e-7


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(6, 32, 40, 5, 3, 2, 0.5), (300, 32, 40, 1, 1, 2, 0.5), (200, 128, 200, 9, 9, 2, 0.33)])
def test_frozen_weights_and_inputs(shape, dtype):
    from paper_2101_00745_amd.nn import gated_scc
    cg, co = shape[5:]
    (x, w, dy), _ = inputs(shape, dtype, seed=13)
    x, w, dy = x.cuda().requires_grad_(True), w.cuda().requires_grad_(True), dy.cuda()
    both = torch.autograd.grad(gated_scc(x, w, cg, co), (x, w), dy)
    frozen, data = w.detach(), x.detach()
    dx, = torch.autograd.grad(gated_scc(x, frozen, cg, co), x, dy)
    dw, = torch.autograd.grad(gated_scc(data, w, cg, co), w, dy)
    assert torch.equal(dx, both[0]) and torch.equal(dw, both[1])
    assert not gated_scc(data, frozen, cg, co).requires_grad


@pytest.mark.gpu
@pytest.mark.parametrize("shape,seed", [((2, 5, 1, 7, 7, 5, 0.5), 100), ((9, 8, 2, 4, 4, 8, 0.0), 31), ((300, 14, 1, 1, 1, 7, 0.0), 1), ((40, 6, 1, 6, 8, 3, 0.0), 271),
                                        ((100, 7, 2, 2, 2, 7, 0.5), 218), ((2, 5, 1, 7, 7, 5, 0.5), 30)])
def test_few_weights_whose_products_cancel(shape, seed):
    """Inputs for which the gradients between the stages, rounded to bfloat16, put dw off by 0.024 to 0.11 of its largest value."""
    cg, co = shape[5:]
    (x, w, dy), wide = inputs(shape, torch.bfloat16, seed=seed)
    _, dx, dw = reference(wide[0], wide[1], cg, co, "silu", wide[2])
    got = B._gated_backward(x.cuda(), w.cuda(), dy.cuda(), cg, co, "silu", False)
    assert off(got[0], dx) <= TOL[torch.bfloat16] and off(got[1], dw) <= TOL[torch.bfloat16]


def test_few_weights_of_more_columns_than_one_sample_indexes_are_not_refused():
    lib = S.load()
    for shape in ((1 << 20, 1, 1, 32, 32, 1, 0.5), (1 << 20, 4, 2, 16, 16, 2, 0.5), (1 << 13, 16, 1, 256, 256, 16, 0.5)):
        assert lib.scc_gated_backward_workspace_bytes(*shape, 1, 0) > 0
