"""AdamW where a step is refused, and where its moments leave binary32's normal range."""
import math

import pytest
import torch

import paper_2101_00745_amd as S
from paper_2101_00745_amd import optim
from tests.test_adamw import BETAS, LR, ULP, bytes_of


def snapshot(opt, params):
    ages = [int(opt.state[p]["step"]) if p in opt.state and opt.state[p] else 0 for p in params]
    values = [t.clone() for p in params for t in (p.detach(), *(v for k, v in sorted(opt.state[p].items() if p in opt.state else ()) if k != "step"))]
    return ages, values


def unchanged(before, opt, params):
    ages, values = snapshot(opt, params)
    return ages == before[0] and len(values) == len(before[1]) and all(torch.equal(a.float(), b.float()) for a, b in zip(values, before[1]))


def test_a_refused_step_leaves_no_state_on_the_cpu():
    p = torch.nn.Parameter(torch.zeros(3))
    p.grad = torch.ones(3)
    opt = optim.AdamW([p])
    for _ in range(2):
        with pytest.raises(ValueError, match="GPU"):
            opt.step()
        assert not opt.state


def spoil(how, opt, params):
    """Makes the next step one that is refused; returns what undoes that."""
    last = params[-1]
    if how == "not contiguous":
        kept = last.data
        last.data = kept.t().contiguous().t()
        last.grad = torch.ones_like(last)

        def undo():
            last.data, last.grad = kept, torch.ones_like(kept)
    elif how == "shared memory":
        last.grad = last.detach()

        def undo():
            last.grad = None
    elif how == "a state of another shape":
        state = opt.state[last]
        kept = state["first"]
        state["first"] = kept.reshape(-1)

        def undo():
            state["first"] = kept
    elif how == "option":
        opt.param_groups[-1]["lr"] = math.nan

        def undo():
            opt.param_groups[-1]["lr"] = LR
    else:
        kept = last.grad
        last.grad = kept.to_sparse()

        def undo():
            last.grad = kept
    return undo


@pytest.mark.gpu
@pytest.mark.parametrize("capturable", [False, True])
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("how", ["not contiguous", "shared memory", "a state of another shape", "option", "sparse gradient"])
@pytest.mark.parametrize("groups", [1, 2])
def test_a_refused_step_moves_nothing(groups, how, bits, capturable):
    """Lists of two types and two ages, the last of them refused: ages, weights and states stay what they were, and the next step is the one that would
    have been."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    new = lambda *s, dtype=torch.float32: torch.nn.Parameter(torch.randn(*s, generator=gen, device="cuda").to(dtype))  # noqa: E731
    params = [new(700), new(30, 20, dtype=torch.bfloat16), new(5), new(12, 40)]
    twins = [torch.nn.Parameter(p.detach().clone()) for p in params]

    def make(l):
        return optim.AdamW([{"params": l}] if groups == 1 else [{"params": l[:2]}, {"params": l[2:]}], lr=LR, betas=BETAS, state_bits=bits, capturable=capturable)

    def give(l, some):
        for i, p in enumerate(l):
            p.grad = torch.full_like(p, 0.5 + i) if i in some else None

    opt, plain = make(params), make(twins)
    for some in ((0, 1, 3), (0, 1, 2, 3)):
        give(params, some)
        give(twins, some)
        opt.step()
        plain.step()
    undo = spoil(how, opt, params)
    before = snapshot(opt, params)
    for _ in range(2):
        with pytest.raises((ValueError, RuntimeError, S.SccError)):
            opt.step()
        assert unchanged(before, opt, params)
    undo()
    give(params, (0, 1, 2, 3))
    give(twins, (0, 1, 2, 3))
    opt.step()
    plain.step()
    assert all(torch.equal(p, q) for p, q in zip(params, twins))
    assert snapshot(opt, params)[0] == snapshot(plain, twins)[0]


@pytest.mark.gpu
@pytest.mark.parametrize("capturable", [False, True])
def test_a_refused_first_step_leaves_no_states(capturable):
    good, bad = torch.nn.Parameter(torch.ones(40, device="cuda")), torch.nn.Parameter(torch.ones(6, 5, device="cuda").t())
    opt = optim.AdamW([good, bad], capturable=capturable)
    good.grad, bad.grad = torch.ones_like(good), torch.ones_like(bad)
    with pytest.raises(ValueError, match="contiguous"):
        opt.step()
    assert not opt.state and (good == 1).all()


@pytest.mark.gpu
def test_a_capture_with_a_refused_group_captures_nothing():
    a, b = ([torch.nn.Parameter(torch.ones(n, device="cuda"))] for n in (30, 50))
    opt = optim.AdamW([{"params": a}], lr=LR, capturable=True)
    a[0].grad, b[0].grad = torch.ones_like(a[0]), torch.ones_like(b[0])
    opt.step()
    opt.add_param_group({"params": b})          # has made no step
    before, other = snapshot(opt, [*a, *b]), torch.zeros(4, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        other.add_(1)
        with pytest.raises(RuntimeError, match="before the capture"):
            opt.step()
    graph.replay()
    torch.cuda.synchronize()
    assert unchanged(before, opt, [*a, *b]) and (other == 1).all()


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
