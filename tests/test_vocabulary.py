"""Cross entropy over a vocabulary and its gradients, without the logits in memory: the formulas on the CPU against differences, refusals, and
the kernels against 64 bits.

Bars.  A logit is a sum of C products: off by (2^-21 for three-piece products, 0 for bf16's) and some sqrt(C) roundings at 2^-24 of the magnitudes
m = sum |x w| that it adds up: D = (2^-21 + 4 sqrt(C) 2^-24 + 2^-23) max_v m.  A loss is off by 2 D, and by a few roundings of |lse| and of itself.  p is off by 2 D + 8 |lse|
2^-24 of itself (and in bfloat16 by half a step of fp16, 2^-11, or 2^-39), its one-hot part by as much of exp(l - lse) as of 1.  dx and dw add up as
many terms: that much of sum |p w| (|p x|), where |p| counts exp(l - lse) and the one apart, 4 sqrt(terms) 2^-24 of it more, and half a step at the end;
d x in fp16 once more 2^-11."""
import math

import pytest
import torch

import paper_2101_00745_amd as S
from paper_2101_00745_amd import nn as N
from paper_2101_00745_amd import scc as B

DTYPES = [pytest.param(torch.float32, id="f32"), pytest.param(torch.bfloat16, id="bf16")]
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
ULP = 2.0 ** -24
IGNORED = -100


def rows(t):
    return t.double().movedim(1, -1).reshape(-1, t.shape[1])


def back(t, like):
    return t.view(like.shape[0], *like.shape[2:], like.shape[1]).movedim(-1, 1)


def reference(x, w, target, ignored=IGNORED):
    """lse, loss per token and p without its one, all of tokens x vocabulary, in 64 bits."""
    x, w, y = rows(x), w.double(), target.flatten()
    logits = x @ w.t()
    lse = torch.logsumexp(logits, 1)
    kept = y != ignored
    loss = torch.where(kept, lse - logits.gather(1, y.clamp(0, w.shape[0] - 1)[:, None])[:, 0], 0.0)
    return lse, loss, torch.exp(logits - lse[:, None]), kept


def gradients(x, w, target, d, ignored=IGNORED):
    """dx, dw (64 bits) for the gradients d of the tokens' losses, and the magnitudes they add up."""
    _, _, p, kept = reference(x, w, target, ignored)
    d = torch.where(kept, d.double().flatten(), 0.0)
    one = torch.zeros_like(p).scatter_(1, target.flatten().clamp(min=0)[:, None], 1.0)
    xr, wd = rows(x), w.double()
    q, size = (p - one) * d[:, None], (p + one) * d[:, None].abs()
    return back(q @ wd, x), q.t() @ xr, back(size @ wd.abs(), x), size.t() @ xr.abs()


def logit_bar(x, w):
    C = x.shape[1]
    m = rows(x).abs() @ w.double().abs().t()
    return (2.0 ** -21 * (x.dtype == torch.float32) + (4 * math.sqrt(C) + 2) * ULP) * m.amax(1)


def inputs(shape, V, dtype, ignored=0.0, seed=0, spread=1.0):
    gen = torch.Generator(device="cuda").manual_seed(500 + seed)
    N_, C, H, W = shape
    w = torch.randn(V, C, generator=gen, device="cuda") * spread / math.sqrt(C)
    target = torch.randint(V, (N_, H, W), generator=gen, device="cuda")
    known = torch.rand(N_, 1, H, W, generator=gen, device="cuda") * 6
    x = torch.randn(shape, generator=gen, device="cuda") + known * w[target].movedim(-1, 1)
    target = target.masked_fill(torch.rand(N_, H, W, generator=gen, device="cuda") < ignored, IGNORED)
    return x.to(dtype), w.to(dtype), target


def check_loss(x, w, target, ignored=IGNORED):
    lse, loss, _, kept = reference(x, w, target, ignored)
    bar = 2 * logit_bar(x, w) + 8 * ULP * (lse.abs() + loss.abs()) + 4 * ULP
    got, got_lse = S.scc_vocabulary_loss(x, w, target, "none", ignored)
    assert got.shape == target.shape and got.dtype == torch.float32
    assert ((got.double().flatten() - loss).abs() <= bar).all()
    assert ((got_lse.double().flatten() - torch.where(kept, lse, 0.0)).abs() <= bar).all()
    assert (got.flatten()[~kept] == 0).all()
    count = int(kept.sum())
    for name, scale in (("sum", 1.0), ("mean", 1.0 / max(1, count))):
        one, same = S.scc_vocabulary_loss(x, w, target, name, ignored)
        assert one.shape == () and torch.equal(same, got_lse)
        want = float(got.double().sum()) * scale
        assert abs(float(one) - want) <= 2 * ULP * abs(want)
    return got_lse


def check_gradients(x, w, target, lse, reduction="mean", dloss=None, ignored=IGNORED):
    kept = target != ignored
    if reduction == "none":
        d = dloss
    else:
        d = dloss * torch.ones_like(lse) / (max(1, int(kept.sum())) if reduction == "mean" else 1)
    dx, dw, dx_size, dw_size = gradients(x, w, target, d, ignored)
    got_dx, got_dw = S.scc_vocabulary_gradients(x, w, target, lse, dloss, reduction, ignored)
    half = x.dtype == torch.bfloat16
    # the worst token's bar for all of a sum over tokens
    tokens = 2 * logit_bar(x, w) + 8 * ULP * (1 + rows_lse(x, w).abs()) + (2.0 ** -11 if half else 2.0 ** -20)
    by_token = tokens.view(target.shape).unsqueeze(1)
    V, T = w.shape[0], target.numel()
    bar = (by_token + 4 * math.sqrt(V) * ULP) * dx_size + HALF[x.dtype] * dx.abs()
    if half:        # fp16 below its normal range: 2^-25 of 2^14, and the channel's smallest
        bar += 2.0 ** -39 * d.double().abs().unsqueeze(1) * w.double().abs().sum(0).view(1, -1, 1, 1) + 2.0 ** -39 * dx_size.amax()
    assert ((got_dx.double() - dx).abs() <= bar + 1e-37).all()
    assert (got_dx.movedim(1, -1)[~kept] == 0).all()
    bar = (float(tokens.max()) + (2.0 ** -11 if half else 0.0) + 4 * math.sqrt(T) * ULP) * dw_size
    if half:
        bar += 2.0 ** -39 * (d.double().abs().flatten() @ rows(x).abs()) + 2.0 ** -39 * dw_size.amax()
    assert got_dw.dtype == torch.float32
    assert ((got_dw.double() - dw).abs() <= bar + 1e-37).all()
    again = S.scc_vocabulary_gradients(x, w, target, lse, dloss, reduction, ignored)
    assert torch.equal(again[0], got_dx) and torch.equal(again[1], got_dw)
    stored = B._vocabulary_gradients(x, w, target, lse, dloss, B.REDUCTIONS[reduction], ignored, True)
    assert torch.equal(stored[0], got_dx) and torch.equal(stored[1], got_dw.to(x.dtype))


def rows_lse(x, w):
    return torch.logsumexp(rows(x) @ w.double().t(), 1)


def test_gradient_formula_against_differences():
    gen = torch.Generator().manual_seed(8)
    x, w = torch.randn(2, 5, 3, 1, generator=gen, dtype=torch.float64), torch.randn(7, 5, generator=gen, dtype=torch.float64)
    target = torch.tensor([[[1], [IGNORED], [6]], [[0], [0], [3]]])
    d = torch.randn(2, 3, 1, generator=gen, dtype=torch.float64)
    dx, dw, _, _ = gradients(x, w, target, d)
    step = 1e-5
    for t, grad in ((x, dx), (w, dw)):
        e = torch.randn(t.shape, generator=gen, dtype=torch.float64)
        ends = [float((reference(*((t + s * step * e, w) if t is x else (x, t + s * step * e)), target)[1] * d.flatten()).sum()) for s in (1, -1)]
        assert abs((ends[0] - ends[1]) / (2 * step) - float((grad * e).sum())) <= 1e-7 * max(1.0, abs(float((grad * e).sum())))


def test_refusals():
    lib = S.load()
    one = 1 << 20                               # an address that no refused call reads
    for sizes in ((0, 4, 1, 1, 5), (1, 0, 1, 1, 5), (1, 4, 0, 1, 5), (1, 4, 1, 0, 5), (1, 4, 1, 1, 0), (1 << 14, 4, 1 << 13, 1, 5), (1, 1 << 21, 1, 1, 5),
                  (1, 4, 1, 1, (1 << 26) + 1), (1, 4, 1 << 16, 1 << 16, 5)):
        assert lib.scc_vocabulary_loss(one, one, one, one, one, *sizes, -100, 0, 0, one, 1 << 40, None) == -2
        assert lib.scc_vocabulary_gradients(one, one, one, one, one, one, one, *sizes, -100, 0, 0, 0, one, 1 << 40, None) == -2
        assert lib.scc_vocabulary_loss_workspace_bytes(*sizes, 0, 0) == 0 and lib.scc_vocabulary_gradients_workspace_bytes(*sizes, 0) == 0
    sizes = (1, 4, 1, 1, 5)
    assert lib.scc_vocabulary_loss(one, one, one, one, one, *sizes, -100, 3, 0, one, 1 << 40, None) == -8
    assert lib.scc_vocabulary_loss(one, one, one, one, one, *sizes, -100, 0, 2, one, 1 << 40, None) == -4
    assert lib.scc_vocabulary_gradients(one, one, one, one, one, one, one, *sizes, -100, 0, 0, 1, one, 1 << 40, None) == -4
    for i in range(5):
        assert lib.scc_vocabulary_loss(*[None if i == j else one for j in range(5)], *sizes, -100, 0, 0, one, 1 << 40, None) == -1
    for i in range(7):
        assert lib.scc_vocabulary_gradients(*[None if i == j else one for j in range(7)], *sizes, -100, 0, 0, 0, one, 1 << 40, None) == -1
    for dtype in (0, 1):
        need = lib.scc_vocabulary_loss_workspace_bytes(*sizes, 2, dtype)
        for ws, size in ((None, need), (one, need - 1), (one + 16, need)):
            assert lib.scc_vocabulary_loss(one, one, one, one, one, *sizes, -100, 2, dtype, ws, size, None) == -5
        need = lib.scc_vocabulary_gradients_workspace_bytes(*sizes, dtype)
        for ws, size in ((None, need), (one, need - 1), (one + 16, need)):
            assert lib.scc_vocabulary_gradients(one, one, one, one, one, one, one, *sizes, -100, 2, dtype, 0, ws, size, None) == -5
    with pytest.raises(ValueError):
        S.scc_vocabulary_loss(torch.zeros(1, 4, 1, 1), torch.zeros(5, 4), torch.zeros(1, 1, 1, dtype=torch.int64))
    with pytest.raises(ValueError, match="reduction"):
        N.VocabularyLoss(4, 5, reduction="median", device="cpu")


def test_workspaces_of_many_sizes():
    lib = S.load()
    for T in (1, 63, 64, 65, 4096, 33000, 1 << 22, 1 << 26):
        for C in (1, 64, 65, 513, 1 << 14, 1 << 20):
            for V in (1, 64, 257, 5200, 70000, 1 << 26):
                if T * V > 1 << 45:
                    assert lib.scc_vocabulary_gradients_workspace_bytes(T, C, 1, 1, V, 0) == 0
                    continue
                for dtype in (0, 1):
                    assert lib.scc_vocabulary_loss_workspace_bytes(T, C, 1, 1, V, 2, dtype) > 0
                    need = lib.scc_vocabulary_gradients_workspace_bytes(T, C, 1, 1, V, dtype)
                    assert need >= (10 if dtype == 0 else 8) * T * C        # its copies of x and one part of dx


@pytest.mark.gpu
def test_refusals_of_the_binding():
    x, w, t = torch.zeros(2, 4, 3, 1, device="cuda"), torch.zeros(5, 4, device="cuda"), torch.zeros(2, 3, 1, dtype=torch.int64, device="cuda")
    for bad in ((x[0], w, t), (x, w[:, :3], t), (x, w.bfloat16(), t), (x, w, t.int()), (x, w, t[:1]), (x, w.t(), t), (x, w, t, "median")):
        with pytest.raises((ValueError, TypeError)):
            S.scc_vocabulary_loss(*bad)
    loss, lse = S.scc_vocabulary_loss(x, w, t)
    for bad in ((lse[:1], loss), (lse, loss[None]), (lse, lse), (lse.double(), loss), (lse, loss.double())):
        with pytest.raises((ValueError, TypeError)):
            S.scc_vocabulary_gradients(x, w, t, *bad)


# (N, C, H, W), V
CASES = [((1, 64, 1, 1), 1000), ((1, 1, 1, 1), 1), ((3, 5, 1, 1), 2), ((48, 128, 1, 1), 4099), ((64, 100, 1, 1), 64), ((65, 64, 1, 1), 257), ((130, 192, 1, 1), 5000),
         ((300, 513, 1, 1), 700), ((2, 64, 9, 1), 255), ((3, 33, 7, 7), 129), ((2, 320, 70, 1), 1025), ((5, 8, 2, 3), 40), ((1, 1000, 129, 1), 300),
         ((700, 64, 1, 1), 3001)]
IDS = ["x".join(map(str, s)) + "_%d" % v for s, v in CASES]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape,V", CASES, ids=IDS)
def test_loss_and_gradients(shape, V, dtype):
    x, w, target = inputs(shape, V, dtype, ignored=0.3 if shape[0] * shape[2] > 4 else 0.0)
    lse = check_loss(x, w, target)
    check_gradients(x, w, target, lse, "mean", torch.tensor(0.7, device="cuda"))
    check_gradients(x, w, target, lse, "sum", torch.tensor(-2.0, device="cuda"))
    check_gradients(x, w, target, lse, "none", torch.randn(target.shape, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_several_pieces_of_the_vocabulary(dtype):
    """So many tokens that p of the whole vocabulary is taken in three pieces, the last of them shorter."""
    x, w, target = inputs((33000, 16, 1, 1), 5200, dtype, ignored=0.1)
    lse = check_loss(x, w, target)
    check_gradients(x, w, target, lse, "mean", torch.tensor(1.0, device="cuda"))


@pytest.mark.gpu
def test_more_tokens_than_a_grid_has_rows():
    """Three million tokens, of which a few thousand count; what they are not part of stays zero."""
    T, C, V = 3_000_000, 8, 40
    x, w, target = inputs((T, C, 1, 1), V, torch.bfloat16)
    target.fill_(IGNORED)
    some = torch.arange(0, T, 700, device="cuda")
    target[some] = torch.randint(V, (some.numel(), 1, 1), device="cuda")
    picked = x[some].contiguous()
    want, want_lse = S.scc_vocabulary_loss(picked, w, target[some].contiguous(), "none")
    got, lse = S.scc_vocabulary_loss(x, w, target, "none")
    assert torch.equal(got[some], want) and torch.equal(lse[some], want_lse) and int((got != 0).sum()) == int((want != 0).sum())
    d = torch.tensor(1.0, device="cuda")
    dx, dw = S.scc_vocabulary_gradients(x, w, target, lse, d, "sum")
    want_dx, want_dw, dx_size, dw_size = gradients(picked, w, target[some], torch.ones_like(want))
    assert int((dx != 0).any(1).sum()) == some.numel()
    assert ((dx[some].double() - want_dx).abs() <= 2.0 ** -8 * want_dx.abs() + 2.0 ** -9 * dx_size).all()
    assert ((dw.double() - want_dw).abs() <= 2.0 ** -9 * dw_size).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_split_sums_over_a_long_vocabulary(dtype):
    x, w, target = inputs((70, 24, 1, 1), 70000, dtype)
    lse = check_loss(x, w, target)
    check_gradients(x, w, target, lse, "sum", torch.tensor(1.0, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape,V", [((9000, 40, 1, 1), 70), ((3, 150, 40, 50), 300), ((2600, 200, 1, 1), 500)])
def test_split_sums_over_many_tokens(shape, V, dtype):
    x, w, target = inputs(shape, V, dtype, ignored=0.4)
    lse = check_loss(x, w, target)
    check_gradients(x, w, target, lse, "mean", torch.tensor(1.0, device="cuda"))
    target.fill_(IGNORED)
    dx, dw = S.scc_vocabulary_gradients(x, w, target, lse, torch.tensor(1.0, device="cuda"))
    assert (dx == 0).all() and (dw == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape", [(40, 64, 1, 1), (2, 48, 100, 1)])
def test_no_token_counts(shape, dtype):
    x, w, target = inputs(shape, 333, dtype)
    target.fill_(7)
    lse = check_loss(x, w, target, ignored=7)
    loss, _ = S.scc_vocabulary_loss(x, w, target, "mean", 7)
    assert float(loss) == 0.0
    for reduction, d in (("mean", torch.tensor(3.0, device="cuda")), ("none", torch.ones_like(lse))):
        dx, dw = S.scc_vocabulary_gradients(x, w, target, lse, d, reduction, 7)
        assert (dx == 0).all() and (dw == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_channels_of_different_sizes(dtype):
    """Channels of x and w between 2^-20 and 2^20: each has its own power of two where products are taken in fewer bits."""
    x, w, target = inputs((90, 64, 1, 1), 500, dtype)
    powers = torch.exp2(torch.randint(-20, 21, (64,), device="cuda").float())
    x, w = (x.float() * powers.view(1, -1, 1, 1)).to(dtype), (w.float() / powers).to(dtype)
    lse = check_loss(x, w, target)
    _, _, p, _ = reference(x, w, target)
    one = torch.zeros_like(p).scatter_(1, target.flatten()[:, None], 1.0)
    want = (p - one).t() @ rows(x)
    size = (p + one).t() @ rows(x).abs()
    dw = S.scc_vocabulary_gradients(x, w, target, lse, torch.tensor(1.0, device="cuda"), "sum")[1].double()
    assert ((dw - want).abs() <= 3e-3 * size).all()              # 2^-11 of p, of x and of the logits, with room


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_large_logits(dtype):
    """Logits of some hundreds: exponentials that leave binary32 without their maximum; tokens that are sure of their target."""
    x, w, target = inputs((100, 64, 1, 1), 900, dtype, spread=20.0)
    x = x * 8
    lse = check_loss(x, w, target)
    check_gradients(x, w, target, lse, "sum", torch.tensor(1.0, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tokens", [20, 200])
def test_targets_outside_and_values_that_are_not_finite(tokens, dtype):
    x, w, target = inputs((tokens, 64, 1, 1), 300, dtype)
    clean, _ = S.scc_vocabulary_loss(x, w, target, "none")
    bad = target.clone()
    bad[3], bad[5], bad[7] = 300, -1, 1 << 40
    loss, lse = S.scc_vocabulary_loss(x, w, bad, "none")
    outside = torch.zeros(tokens, dtype=torch.bool, device="cuda")
    outside[[3, 5, 7]] = True
    assert torch.isnan(loss.flatten()[outside]).all() and torch.equal(loss.flatten()[~outside], clean.flatten()[~outside])
    dx, dw = S.scc_vocabulary_gradients(x, w, bad, lse, torch.ones_like(lse), "none")
    assert torch.isnan(dx[outside]).all() and torch.isfinite(dx[~outside]).all()
    x = x.clone()
    x[11, 2] = math.nan
    loss, _ = S.scc_vocabulary_loss(x, w, target, "none")
    assert torch.isnan(loss.flatten()[11]) and torch.isfinite(loss.flatten()[12:]).all() and torch.isfinite(loss.flatten()[:11]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_unaligned_weights(dtype):
    x, w, target = inputs((80, 64, 1, 1), 257, dtype)
    room = torch.zeros(257 * 64 + 1, dtype=dtype, device="cuda")
    w1 = room[1:].view(257, 64)
    w1.copy_(w)
    for reduction in ("none", "mean"):
        a, b = S.scc_vocabulary_loss(x, w, target, reduction), S.scc_vocabulary_loss(x, w1, target, reduction)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    d = torch.tensor(1.0, device="cuda")
    a, b = (S.scc_vocabulary_gradients(x, v, target, a[1], d) for v in (w, w1))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_autograd(dtype):
    x, w, target = inputs((3, 96, 40, 1), 600, dtype, ignored=0.2)
    for reduction in ("mean", "sum", "none"):
        xs, ws = x.clone().requires_grad_(), w.clone().requires_grad_()
        loss = N.vocabulary_loss(xs, ws, target, reduction)
        d = torch.randn(loss.shape, device="cuda")
        loss.backward(d)
        want, lse = S.scc_vocabulary_loss(x, w, target, reduction)
        dx, dw = B._vocabulary_gradients(x, w, target, lse, d, B.REDUCTIONS[reduction], IGNORED, True)
        assert torch.equal(loss, want) and torch.equal(xs.grad, dx) and torch.equal(ws.grad, dw)
    loss = N.vocabulary_loss(xs, ws, target)
    for g in torch.autograd.grad(loss, (xs, ws), create_graph=True):
        with pytest.raises(RuntimeError, match="second derivative"):
            g.sum().backward(retain_graph=True)
    assert torch.equal(torch.autograd.grad(N.vocabulary_loss(xs, w, target, "sum"), xs)[0], torch.autograd.grad(N.vocabulary_loss(xs, ws, target, "sum"), xs)[0])
    head = N.VocabularyLoss(96, 600, dtype=dtype)
    head(x, target).backward()
    assert head.weight.grad.dtype == dtype and torch.isfinite(head.weight.grad).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
def test_captured_and_on_another_stream(dtype):
    x, w, target = inputs((150, 64, 1, 1), 700, dtype, ignored=0.2)
    d = torch.tensor(1.0, device="cuda")

    def step():
        loss, lse = S.scc_vocabulary_loss(x, w, target)
        return (loss, *S.scc_vocabulary_gradients(x, w, target, lse, d))

    want = step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step()
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(3):
        x.copy_(torch.randn_like(x.float()))
        target.copy_(torch.where(torch.rand(target.shape, device="cuda") < 0.2 * i, IGNORED, torch.randint_like(target, 700)))
        want = step()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
def test_several_pieces_of_the_vocabulary_for_more_tokens():
    """p of 140000 tokens in bfloat16 in three pieces; dx adds up over them."""
    x, w, target = inputs((140000, 16, 1, 1), 5200, torch.bfloat16, ignored=0.02)
    lse = check_loss(x, w, target)
    check_gradients(x, w, target, lse, "mean", torch.tensor(1.0, device="cuda"))


@pytest.mark.gpu
def test_offsets_of_more_than_32_bits():
    """A vocabulary of 2^25 + 300 rows of 128 channels, all zeros but a few, the targets' among them: every other row has exp(0) in the sum."""
    V, C = (1 << 25) + 300, 128
    w = torch.zeros(V, C, dtype=torch.bfloat16, device="cuda")
    special = torch.tensor([0, 1 << 24, 1 << 25, V - 1], device="cuda")
    w[special] = torch.randn(4, C, device="cuda").bfloat16()
    x = (torch.randn(3, C, 1, 1, device="cuda") + 1.5 * w[special[1:]].float()[:, :, None, None]).bfloat16()
    target = special[1:].view(3, 1, 1).contiguous()
    rows_, some = x.double().view(3, C), w[special].double()
    l = rows_ @ some.t()
    total = torch.exp(l).sum(1) + (V - 4)
    loss, lse = S.scc_vocabulary_loss(x, w, target, "none")
    # logits as in the other tests; the sum's 2^25 equal terms and its 500000 tiles' joins stay below 64 roundings of the whole
    assert ((lse.double().view(3) - torch.log(total)).abs() <= 1e-5 * l.abs().amax() + 64 * ULP * torch.log(total)).all()
    assert ((loss.double().view(3) - (torch.log(total) - l[torch.arange(3), torch.arange(1, 4)])).abs() <= 1e-5 * l.abs().amax() + 64 * ULP * torch.log(total)).all()
    dx, dw = S.scc_vocabulary_gradients(x, w, target, lse, torch.tensor(1.0, device="cuda"), "sum")
    p = torch.exp(l) / total[:, None]
    size = p.clone()
    p[torch.arange(3), torch.arange(1, 4)] -= 1
    size[torch.arange(3), torch.arange(1, 4)] += 1
    # p is 1 for a sure token, and what is left of p - 1 is the error of its exponent l - lse: of a logit (twice, the lse has it too), of eight roundings of numbers of
    # the lse's size, and of p as it is stored; in relation to p + [target].  As in check_gradients.
    off = (2 * logit_bar(x, w[special]) + 8 * ULP * (1 + torch.log(total)) + 2.0 ** -11).view(3, 1)
    want = p @ some
    assert ((dx.double().view(3, C) - want).abs() <= 2.0 ** -8 * want.abs() + (off * size) @ some.abs()).all()
    want = p.t() @ rows_
    assert ((dw[special].double() - want).abs() <= ((off + 2.0 ** -11) * size).t() @ rows_.abs() + 2.0 ** -37 * rows_.abs().amax()).all()
    # a row of zeros: p = 1 / total for each token, stored as fp16 times 2^14: 2^-11 of it, or all of what is below 2^-25
    want = (rows_ / total[:, None]).sum(0)
    for v in (1, (1 << 24) + 1, (1 << 25) + 1, V - 2):
        assert ((dw[v].double() - want).abs() <= 2.0 ** -9 * (rows_.abs() / total[:, None]).sum(0) + 2.0 ** -37 * rows_.abs().amax()).all()
