"""The vocabulary loss where its exponents are large, and the forms of its products that take many tokens.

Logits here are exact: x has one channel that is not 0, w one that is 1 for the target.  So what is off is the loss's own."""
import math

import pytest
import torch

import paper_2101_00745_amd as S
from paper_2101_00745_amd import nn as N
from tests.test_vocabulary import DTYPES, ULP, check_gradients, check_loss, inputs

C, V, Y = 64, 2000, 777


def sure(dtype, tokens):
    """Tokens whose target's logit is between 12 and 20000 and whose other logits are 0."""
    x = torch.zeros(tokens, C, 1, 1, device="cuda")
    x[:, 5, 0, 0] = torch.exp2(torch.linspace(math.log2(12.0), math.log2(20000.0), tokens, device="cuda"))
    w = torch.zeros(V, C, device="cuda")
    w[Y, 5] = 1.0
    return x.to(dtype), w.to(dtype), torch.full((tokens, 1, 1), Y, device="cuda")


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [40, 500, 3000])
@pytest.mark.parametrize("dtype", DTYPES)
def test_a_token_that_is_sure_of_its_target(tokens, dtype):
    """total = 1 + (V - 1) exp(-l).  The 1 is exact, so the loss is never below 0, and it is 0 from l = 40 on, where the rest is less than half a
    step of the 1.  Below that: a lane adds up to 64 terms (64 roundings of a sum near 1), some 24 more join them, the exponents l log2(e) are rounded
    by 2^-24 l, which the term exp(-l) makes at most 12 exp(-12) V of it, and the logarithm is rounded: 96 * 2^-24."""
    x, w, target = sure(dtype, tokens)
    l = x[:, 5, 0, 0].double()
    want = torch.log1p((V - 1) * torch.exp(-l))
    for reduction in ("none", "sum"):
        loss, lse = S.scc_vocabulary_loss(x, w, target, reduction)
        if reduction == "none":
            loss = loss.double().flatten()
            assert (loss >= 0).all()
            assert (loss[l >= 40] == 0).all()
            assert ((loss - want).abs() <= 96 * ULP).all()
        # half a step of the lse on top
        assert ((lse.double().flatten() - l - want).abs() <= 96 * ULP + ULP * (l + want)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("tokens", [40, 500, 3000])
@pytest.mark.parametrize("dtype", DTYPES)
def test_what_is_left_of_p_for_a_sure_token(tokens, dtype):
    """p - 1 = -(V - 1) exp(-l) / total for the target; w is 1 there and 0 elsewhere, so dx has it alone.  From l = 40 on the lse is l, p is 1 and
    nothing is left.  Below: the lse's half step (2^-24 of at most 64) and error (96 * 2^-24, as above), the exponent's and the exponential's roundings (4 * 2^-24);
    in bfloat16 the 14 that p is raised by costs the exponent half a step of 16 (12 * 2^-24 of p), and what is left is stored in fp16 and then in
    bfloat16 (2^-11 and 2^-8 of it, or 2^-39)."""
    x, w, target = sure(dtype, tokens)
    l = x[:, 5, 0, 0].double()
    rest = (V - 1) * torch.exp(-l)
    want = -rest / (1 + rest)
    lse = S.scc_vocabulary_loss(x, w, target, "none")[1]
    dx, dw = S.scc_vocabulary_gradients(x, w, target, lse, torch.tensor(1.0, device="cuda"), "sum")
    bar = (64 + 96 + 4 + (12 if dtype == torch.bfloat16 else 0)) * ULP * (l < 40) + (2.0 ** -7 * want.abs() + 2.0 ** -38 if dtype == torch.bfloat16 else 2.0 ** -22 * want.abs())
    # from 40 on p is exp(0): what is left is 0, which is off by all of want, 2000 exp(-40) = 9e-15 at most
    bar = torch.where(l < 40, bar, 9e-15)
    assert ((dx[:, 5, 0, 0].double() - want).abs() <= bar).all()
    few = l >= 40
    xs, ts = x[few].contiguous(), target[few].contiguous()
    dx, dw = S.scc_vocabulary_gradients(xs, w, ts, lse[few].contiguous(), torch.tensor(1.0, device="cuda"), "sum")
    # terms of at most exp(-40) times 20000
    assert float(dx.abs().max()) <= 1e-9 and float(dw[Y].abs().max()) <= 1e-9
    xs, ws = xs.requires_grad_(), w.clone().requires_grad_()
    dx, dw = torch.autograd.grad(N.vocabulary_loss(xs, ws, ts, "sum"), (xs, ws))
    assert float(dx.abs().max()) <= 1e-9 and float(dw[Y].abs().max()) <= 1e-9


@pytest.mark.gpu
@pytest.mark.parametrize("offset", [0, 100, 100000])
@pytest.mark.parametrize("dtype", DTYPES)
def test_what_all_logits_of_a_token_have_in_common(dtype, offset):
    """Logits offset + 0 .. 15: the loss is that of 0 .. 15, whatever the offset.  Sums of at most 64 terms of a lane and a dozen joins, exponents of at most 15
    log2(e), whose terms are the small ones: 110 * 2^-24 of the whole."""
    x = torch.zeros(300, C, 1, 1, device="cuda")
    x[:, 0] = 1.0
    x[:, 1:3] = 256.0
    w = torch.zeros(V, C, device="cuda")
    w[:, 0] = torch.arange(V, device="cuda") % 16
    # both factors in bfloat16: 100 = 256 * 0.390625, 100000 = 256 * (390 + 0.625)
    w[:, 1], w[:, 2] = (offset // 256) & ~1, offset / 256 - ((offset // 256) & ~1)
    target = torch.randint(V, (300, 1, 1), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    logits = w[:, 0].double()
    want = torch.logsumexp(logits, 0) - logits[target.flatten()]
    loss = S.scc_vocabulary_loss(x.to(dtype), w.to(dtype), target, "none")[0].double().flatten()
    assert torch.equal(w.to(dtype).float(), w)
    assert ((loss - want).abs() <= 110 * ULP * (1 + want)).all()


# bf16: tiles of 256 x 256 in both gradients' products (350 of them or more), with and without sums in parts, and over two pieces of the vocabulary
LARGE = [((4099, 513, 1, 1), 9001, 0.0), ((3, 600, 1000, 1), 9001, 0.3), ((20000, 300, 1, 1), 600, 0.1), ((2100, 513, 1, 1), 140001, 0.0)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("shape,V,ignored", LARGE, ids=["x".join(map(str, s)) + "_%d" % v for s, v, _ in LARGE])
def test_large_tiles(shape, V, ignored, dtype):
    x, w, target = inputs(shape, V, dtype, ignored=ignored)
    lse = check_loss(x, w, target)
    check_gradients(x, w, target, lse, "mean", torch.tensor(0.7, device="cuda"))
    check_gradients(x, w, target, lse, "none", torch.randn(target.shape, device="cuda"))
