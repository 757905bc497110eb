"""The gated layer where its kernels' ranges end.

Bars as in the layer's other tests: 2e-5 and 1e-2 of the largest value."""
import math

import numpy as np
import pytest
import torch

import paper_2101_00745_amd as S
from tests.test_gated import ANY, DIRECT, DTYPES, TOL, inputs, off, reference

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
