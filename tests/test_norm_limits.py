"""The residual norm where a workgroup of its backward pass takes several tokens or tiles, and the forms that only long batches take: sums of dw over rounds in
registers and in the workspace, tiles in runs and in turn, 16 and 64 lanes a token with two vectors each, 256 lanes with four.  Bars as in test_norm.py."""
import pytest
import torch

import paper_2101_00745_amd as S
from paper_2101_00745_amd import scc as B
from tests.test_norm import DTYPES, EPS, HALF, NEAR, backward, forward, inputs

# (N, C, H, W).  Rows: channels just off 32, 128 and 1024 vectors (of 8 in bf16, of 4 in f32), more tokens than 1024 workgroups take in one round.
ROWS = [(40001, 125, 1, 1), (40001, 250, 1, 1), (9001, 500, 1, 1), (9001, 1000, 1, 1), (2500, 2045, 1, 1), (2500, 4090, 1, 1), (40001, 64, 1, 1), (70000, 3, 1, 1)]
# Columns: more than 512 (1024 of few channels) tiles, planes that end at a line of 128 bytes and others; of 700 and 1300 channels, which do not stay in registers
COLUMNS = [(66, 30, 64, 32), (70, 30, 2001, 1), (33, 300, 64, 32), (34, 300, 2001, 1), (20, 700, 64, 32), (21, 700, 2001, 1), (12, 1300, 3001, 1), (9000, 40, 3, 3), (60000, 20, 2, 1),
           (30000, 7, 5, 1)]
SHAPES = ROWS + COLUMNS
IDS = ["x".join(map(str, s)) for s in SHAPES]


def near(got, want, size, dtype, bar=NEAR):
    off = (got.double() - want).abs() - (bar * size + HALF[dtype] * want.abs())
    assert got.shape == want.shape and not torch.isnan(got).any() and float(off.max()) <= 1e-37, "%g over the bar" % float(off.max())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_long_batches(shape, dtype):
    x, r, w, dy, dh = [t.cuda() for t in inputs(shape, dtype, seed=8)]
    y, h = S.scc_norm_forward(x, w, r, EPS)
    want_y, want_h = forward(x.double(), r.double(), w.double())
    near(y, want_y, want_y.abs(), dtype)
    near(h, want_h, want_h.abs(), dtype)
    q, scale, same = S.scc_norm_quantised(x, w, r, EPS)
    assert torch.equal(same, h)
    unit = scale.double().unsqueeze(1)
    most = want_y.abs().amax(1, keepdim=True)
    assert ((most * (1 - 2 * NEAR) <= 448 * unit) & (most * (1 + 2 * NEAR) > 224 * unit)).all()
    assert ((q.float().double() * unit - want_y).abs() <= want_y.abs() * (2.0 ** -4 + 2 * NEAR) + unit * 2.0 ** -10).all()
    dx, dw = S.scc_norm_backward(x, w, dy, r, dh, EPS)
    want_dx, want_dw, dx_size, dw_size = backward(want_h, w.double(), dy.double(), dh.double())
    near(dx, want_dx, dx_size, dtype)
    near(dw, want_dw, dw_size, torch.float32, (shape[0] * shape[2] * shape[3] / 64 + 160) * 2.0 ** -24)
    # a token that a round left out, or took twice, would be off by some of a token's magnitude, which the bar of a long sum does not see; roundings of
    # different tokens are independent and stay below root T times a token's 80 * 2^-24, 0.002 of it for T = 135168
    tokens = shape[0] * shape[2] * shape[3]
    assert float((dw.double() - want_dw).abs().max()) <= 0.25 * float((dw_size / tokens).min())
    stored = B._norm_backward(x, w, dy, r, dh, EPS, True)
    assert torch.equal(stored[0], dx) and torch.equal(stored[1], dw.to(dtype))
