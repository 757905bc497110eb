"""AdamW where its moments leave binary32's normal range."""

import pytest
import torch

import paper_2101_00745_amd as S
from tests.test_adamw import BETAS, LR, ULP, bytes_of


@pytest.mark.gpu
@pytest.mark.parametrize("exponent", [-50, -60, -63, -65, -68])
def test_second_moments_below_the_normal_range(exponent):
    """Gradients of 2^exponent and an eps of 0: v = (1 - b2) g^2 is not normal below 2^-126, its root is (no less than 2^-75).  The step from the v that is
    stored: m, root, correction, reciprocal and products as in test_adamw.py, 24 * 2^-24 of lr m / root."""
    gen = torch.Generator(device="cuda").manual_seed(2)
    g = [(1.0 + torch.rand(5000, generator=gen, device="cuda")) * 2.0 ** exponent]
    w, m, v = ([torch.zeros(5000, device="cuda")] for _ in range(3))
    S.scc_adamw_step(w, g, m, v, LR, 1, betas=BETAS, eps=0.0)
    v64, g64 = v[0].double(), g[0].double()
    assert ((v64 - (1 - BETAS[1]) * g64 * g64).abs() <= 4 * ULP * v64 + 2.0 ** -148).all() and (v64 > 0).all()
    want = -LR * (m[0].double() / (1 - BETAS[0])) / torch.sqrt(v64 / (1 - BETAS[1]))
    assert ((w[0].double() - want).abs() <= 24 * ULP * want.abs()).all()


@pytest.mark.gpu
@pytest.mark.parametrize("exponent", [-50, -60, -63, -65])
def test_eight_bits_of_second_moments_below_the_normal_range(exponent):
    """v is stored as one of the two values next to it: roots of e4m3 are 1/8 apart or closer, in relation, so v is within 1.125^2 - 1 of what it was; its scale brings
    its root into [128, 256)."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    g = [(1.0 + torch.rand(5000, generator=gen, device="cuda")) * 2.0 ** exponent]
    w = [torch.zeros(5000, device="cuda")]
    m, v, (ms, vs) = bytes_of([(5000,)])
    S.scc_adamw_step(w, g, m, v, LR, 1, betas=BETAS, eps=0.0, first_scales=ms, second_scales=vs)
    want = (1 - BETAS[1]) * g[0].double() ** 2
    got = (v[0].double() * vs[0].double()[torch.arange(5000, device="cuda") // 256]) ** 2
    assert ((got - want).abs() <= 0.27 * want + 2.0 ** -148).all()
    w2, m2, v2 = ([torch.zeros(5000, device="cuda")] for _ in range(3))
    S.scc_adamw_step(w2, g, m2, v2, LR, 1, betas=BETAS, eps=0.0)
    assert torch.equal(w[0], w2[0])
