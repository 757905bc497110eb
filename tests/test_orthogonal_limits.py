"""The orthogonalised update at the ends of its ranges.

Bars as in the operator's other tests: 2-norm 2e-5 in float32, 4e-3 in bfloat16."""
import pytest
import torch

import paper_2101_00745_amd as S
from tests.test_orthogonal import BAR, DTYPES, matrices, off, polynomial

SMALL, STAGED = [(20, 12), (33, 64)], [(300, 200), (96, 96), (20, 12)]      # one launch each, and a launch for each stage


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shapes", [SMALL, STAGED], ids=["small", "staged"])
def test_zero_matrices_without_eps(shapes, dtype):
    """O(0) = 0 also where nothing is added to the norm."""
    gs = matrices(shapes, dtype, seed=20)
    gs[0].zero_()
    out = S.scc_orthogonalise([g.cuda() for g in gs], eps=0.0)
    assert not out[0].any()
    for g, o in zip(gs[1:], out[1:]):
        assert off(o, polynomial(g.double().numpy(), eps=0.0)) <= BAR[dtype]
    ws = [w.cuda() for w in matrices(shapes, dtype, seed=21)]
    before = ws[0].clone()
    ms = [torch.zeros(s, device="cuda") for s in shapes]
    S.scc_orthogonal_step(ws, [g.cuda() for g in gs], ms, lr=0.5, eps=0.0)
    assert torch.equal(ws[0], before)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale", ["least", 1e-38, 1e36, 1e37])
@pytest.mark.parametrize("shapes", [SMALL, STAGED], ids=["small", "staged"])
def test_norms_outside_float32(shapes, scale, dtype):
    """Every value is a number of the type; the norm is beyond its largest, or so small that too few bits of it are left."""
    scale = {torch.float32: 3e-43, torch.bfloat16: 3e-39}[dtype] if scale == "least" else scale       # multiples of the least value
    gs = [torch.from_numpy(g.double().numpy() * scale).to(dtype) for g in matrices(shapes, torch.float32, seed=22, scale=1.0)]
    for g, o in zip(gs, S.scc_orthogonalise([g.cuda() for g in gs], eps=0.0)):
        assert torch.isfinite(g).all() and off(o, polynomial(g.double().numpy(), eps=0.0)) <= BAR[dtype], tuple(g.shape)
