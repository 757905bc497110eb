"""The orthogonalised update at the ends of its ranges, and every form of the products of large lists.

Bars as in the operator's other tests: 2-norm 2e-5 in float32, 4e-3 in bfloat16, and of large lists half as much again as the same iteration
in plain float32 products is off by."""
import pytest
import torch

import paper_2101_00745_amd as S
from tests.test_orthogonal import BAR, DTYPES, iterate, matrices, off, polynomial

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


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_long_sides_and_uneven_lists(dtype):
    """Sides beyond a thousand, and matrices of one tile among them: the blocks of a launch differ by a hundredfold in work."""
    for shapes in ([(2048, 96), (96, 2049), (1, 4096), (3001, 1), (33, 5000)], [(1100, 1500)], [(1, 1), (1500, 40), (16, 16), (700, 1030), (31, 33), (5, 2)]):
        gs = matrices(shapes, dtype, seed=23)
        dev = [g.cuda() for g in gs]
        out = S.scc_orthogonalise(dev)
        for g, o in zip(gs, out):
            assert off(o, polynomial(g.double().numpy())) <= BAR[dtype], tuple(g.shape)
        assert all(torch.equal(a, b) for a, b in zip(out, S.scc_orthogonalise(dev)))


# x in 192 blocks of 4 x 4 tiles, so a workgroup a CU; p and q in 288, so two
WIDE = [[(1000, 1024)] * 3, [(1000, 1024), (1024, 1000)] * 4]


@pytest.mark.gpu
@pytest.mark.parametrize("shapes", WIDE, ids=["x-alone-on-a-cu", "p-two-on-a-cu"])
@pytest.mark.parametrize("dtype", DTYPES)
def test_other_forms_of_the_products_of_large_lists(shapes, dtype):
    dev = [g.cuda() for g in matrices(shapes, dtype, seed=24)]
    out = S.scc_orthogonalise(dev)
    for g, o in zip(dev, out):
        ref = iterate(g, torch.float64).numpy()
        assert off(o, ref) <= (1.5 * off(iterate(g, torch.float32), ref) if dtype == torch.float32 else BAR[dtype]), tuple(g.shape)
    assert all(torch.equal(a, b) for a, b in zip(out, S.scc_orthogonalise(dev)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_weights_moved_by_a_workgroup_a_cu(dtype):
    shapes = WIDE[0]
    ws, gs = ([t.cuda() for t in matrices(shapes, dtype, seed=s, scale=0.05)] for s in (25, 26))
    ms = [t.cuda() for t in matrices(shapes, torch.float32, seed=27)]
    before = [(w.double(), m.double()) for w, m in zip(ws, ms)]
    S.scc_orthogonal_step(ws, gs, ms, lr=0.1, momentum=0.9, weight_decay=0.1)
    for w, g, m, (w0, m0) in zip(ws, gs, ms, before):
        moved = 0.9 * m0 + g.double()
        assert off(m, moved.cpu().numpy()) <= 1e-6
        ref = (1 - 0.1 * 0.1) * w0.cpu() - 0.1 * iterate(g.double() + 0.9 * moved, torch.float64)
        assert off(w, ref.numpy()) <= BAR[dtype]
