"""What the operators around a gated feed-forward block are measured on: the norm in front of it with the residual's addition, the loss over
a vocabulary that a model of such blocks is trained on, and the AdamW step of the weights that the orthogonalised update does not take.

A case is one of six kinds:

    norm_infer    h = x + residual, y = h / rms(h) * weight over the channels: serving, from one token to long sequences
    norm_8bit     the same with y in 8 bits, e4m3 with a power of two for each token
    norm_train    the same and, from dy and dh, the gradients of x, the residual and the weight: a training step through autograd
    loss_score    -log softmax(x W^T)[target] of each token: scoring answers
    loss_train    its mean over the tokens that count and, through autograd, the gradients of x and W
    adamw         a step of AdamW on a list of weights, its states in 32 bits or in 8

Activations are [N, C, H, W]: a sequence of S tokens is a map of S x 1, N single tokens are N maps of 1 x 1.  A list of weights is a text of
shapes.  States in 8 bits come in blocks of 256 elements with a power of two each: the first moment as e4m3 times that, the second as the square
of e4m3 times that; both are rounded up or down at random, so that their expectations are what is rounded, by a hash of the seed, the step, the
weight's place in the list and the element's in the weight.
"""
import math

import torch

own = False     # whether run() calls the package's operators or computes them in elementary torch operations

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
NORM_EPS = 1e-6
IGNORED = -100
LR, BETAS, ADAM_EPS, DECAY, STEP, SEED = 1e-3, (0.9, 0.999), 1e-8, 0.01, 100, 745
BLOCK = 256

# weights of the thirteen sliding-channel layers of the MobileNet-shaped stack at cg = 2, and the weights of eight norms between them
STACK = "64x16,128x32,128x64,256x64,256x128,512x128,512x256,512x256,512x256,512x256,512x256,1024x256,1024x512"
NORMS = "128,128,256,256,512,512,512,1024"

MAX_NORM = {"f32": 128 * 512 * 1024, "bf16": 128 * 512 * 1024}      # elements of a drawn norm's map: the largest listed one's
MAX_LOSS = {"f32": 2000 * 512 * 32000, "bf16": 16000 * 1024 * 64001 // 2}   # tokens * channels * vocabulary of a drawn loss
MAX_LOGITS = 16000 * 64001
MAX_ADAMW = 64001 * 1024                                            # elements of a drawn list


def _norm(kind, N, C, H, W, dtype="f32", residual=True, name=None):
    case = {"kind": kind, "N": N, "C": C, "H": H, "W": W, "dtype": dtype, "residual": residual}
    if name:
        case["name"] = name
    return case


def _loss(kind, N, C, H, W, V, dtype="bf16", ignored=0.0, name=None):
    case = {"kind": kind, "N": N, "C": C, "H": H, "W": W, "V": V, "dtype": dtype, "ignored": ignored}
    if name:
        case["name"] = name
    return case


def _adamw(shapes, dtype="f32", bits=32, name=None):
    case = {"kind": "adamw", "shapes": shapes, "dtype": dtype, "bits": bits}
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # one token in front of a serving model's feed-forward block: the latency of a call
        _norm("norm_infer", 1, 512, 1, 1, dtype="bf16", name="norm_1_token_bf16"),
        # a prompt's tokens as rows, handed on in 8 bits
        _norm("norm_8bit", 4096, 1024, 1, 1, dtype="bf16", name="norm_4096_tokens_8bit"),
        # eight sequences of 2000 tokens as columns, mixed-precision training
        _norm("norm_train", 8, 512, 2000, 1, dtype="bf16", name="norm_train_8x2000_bf16"),
        # the maps that the channel-expanding layer writes, full precision: the largest activations
        _norm("norm_train", 128, 512, 32, 32, name="norm_train_n128_c512_32x32"),
        # the answers of 48 requests scored, one token each
        _loss("loss_score", 48, 512, 1, 1, 32000, name="loss_score_48_tokens"),
        # tokens as rows, mixed-precision training
        _loss("loss_train", 4096, 512, 1, 1, 32000, name="loss_train_4096_tokens_bf16"),
        # two sequences whose first third is a prompt that does not count, full precision
        _loss("loss_train", 2, 512, 1000, 1, 32000, dtype="f32", ignored=0.33, name="loss_train_2x1000_prompted_f32"),
        # eight sequences of 2000 tokens, twice the vocabulary and off every tile: the largest product
        _loss("loss_train", 8, 1024, 2000, 1, 64001, name="loss_train_8x2000_bf16"),
        # one norm's weight: latency of a step
        _adamw("64", name="adamw_64"),
        # all weights of the thirteen-layer stack and of its norms, full precision
        _adamw(STACK + "," + NORMS, name="adamw_stack"),
        # a smaller model kept in bfloat16: embedding, two blocks, their norms
        _adamw("32000x512,2x1024x512,512x1024,512,2x1024x512,512x1024,512", dtype="bf16", bits=8, name="adamw_embedding_8bit_bf16"),
        # an embedding of a large odd vocabulary, full-precision weights, states in 8 bits
        _adamw("64001x1024", bits=8, name="adamw_large_embedding_8bit"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _form(rng, most):
    """(N, H, W) of a map, of sequences or of single tokens, at most so many columns."""
    form = rng.choice(["map", "sequence", "tokens"])
    if form == "map":
        H = rng.choice([2, 4, 5, 7, 8, 12, 14, 16, 20, 28, 32])
        W = H if rng.random() < 0.8 else rng.choice([3, 6, 7, 9, 16, 24])
    else:
        H, W = (_log_uniform(rng, 2, 4096) if form == "sequence" else 1), 1
    H, W = (H, W) if H * W <= most else (min(H, most), 1)
    most = max(1, most // (H * W))
    return _log_uniform(rng, 1, min(most, 64) if form == "sequence" else min(most, 65536)), H, W


def draw(rng):
    """One more case: norms of one token to the largest maps, losses of one token to half of the largest product, lists of one to twelve weights."""
    kind = rng.choice(["norm_infer", "norm_8bit", "norm_train", "norm_train", "loss_score", "loss_train", "loss_train", "adamw", "adamw"])
    dtype = rng.choice(["f32", "bf16"])
    if kind.startswith("norm"):
        C = max(1, _log_uniform(rng, 16, 4096) // rng.choice([1, 8, 8, 8]) * rng.choice([1, 8, 8]))
        N, H, W = _form(rng, max(1, MAX_NORM[dtype] // C))
        return _norm(kind, N, C, H, W, dtype=dtype, residual=rng.random() < 0.8)
    if kind.startswith("loss"):
        C = _log_uniform(rng, 2, 128) * 8 - rng.choice([0, 0, 0, 3])
        V = _log_uniform(rng, 64, 64000)
        N, H, W = _form(rng, max(1, min(16000, MAX_LOSS[dtype] // (C * V), MAX_LOGITS // V)))
        return _loss(kind, N, C, H, W, V, dtype=dtype, ignored=rng.choice([0.0, 0.0, 0.2, 0.33, 0.6]))
    shapes, left = [], MAX_ADAMW
    for _ in range(_log_uniform(rng, 1, 12)):
        shape = [_log_uniform(rng, 1, 64000), _log_uniform(rng, 16, 1024)] if rng.random() < 0.7 else [_log_uniform(rng, 1, 4096)]
        if math.prod(shape) <= left:
            shapes.append("x".join(map(str, shape)))
            left -= math.prod(shape)
    return _adamw(",".join(shapes) or "64", dtype=dtype, bits=rng.choice([8, 32]))


def _shapes(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["shapes"].split(",")]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device="cuda") * std

    state = {"case": case}
    if case["kind"] == "adamw":
        state |= {"w": [], "g": [], "m": [], "v": []}
        if case["bits"] == 8:
            state |= {"ms": [], "vs": []}
        for shape in _shapes(case):
            state["w"].append(normal(*shape, std=0.05).to(dtype))
            state["g"].append(normal(*shape, std=0.01).to(dtype))
            m, v = normal(*shape, std=0.004), normal(*shape, std=0.01).square() + normal(*shape, std=0.003).square()
            if case["bits"] == 8:
                (m, ms), (v, vs) = _to_blocks(m, m.abs(), 1), _to_blocks(v.sqrt(), v, 2)
                state["ms"].append(ms)
                state["vs"].append(vs)
            state["m"].append(m)
            state["v"].append(v)
        return state
    N, C, H, W = (case[k] for k in ("N", "C", "H", "W"))
    if case["kind"].startswith("norm"):
        state["x"] = normal(N, C, H, W).to(dtype)
        # the stream has grown over the layers, and some channels stand out of it
        state["residual"] = (normal(N, C, H, W, std=3.0) * (1.0 + normal(1, C, 1, 1).square())).to(dtype) if case["residual"] else None
        state["w"] = (1.0 + normal(C, std=0.2)).to(dtype)
        if case["kind"] == "norm_train":
            state["dy"] = normal(N, C, H, W).to(dtype)
            state["dh"] = normal(N, C, H, W).to(dtype) if case["residual"] else None
        return state
    V = case["V"]
    w = normal(V, C, std=C ** -0.5)
    target = torch.randint(V, (N, H, W), generator=gen, device="cuda")
    # tokens know their target to different degrees
    known = torch.rand(N, 1, H, W, generator=gen, device="cuda") * 12.0
    state["x"] = (normal(N, C, H, W) + known * w[target].movedim(-1, 1)).to(dtype)
    state["w"] = w.to(dtype)
    if H * W > 1:       # the first pixels of each sample are a prompt
        counts = (torch.arange(H * W, device="cuda") >= int(case["ignored"] * H * W)).view(1, H, W)
    else:
        counts = torch.rand(N, 1, 1, generator=gen, device="cuda") >= case["ignored"]
    state["target"] = target.masked_fill(~counts.expand(N, H, W), IGNORED)
    return state


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(state):
    import paper_2101_00745_amd as scc
    from paper_2101_00745_amd import nn

    case = state["case"]
    kind = case["kind"]
    if kind == "norm_infer":
        return scc.scc_norm_forward(state["x"], state["w"], residual=state["residual"], eps=NORM_EPS)
    if kind == "norm_8bit":
        return scc.scc_norm_quantised(state["x"], state["w"], residual=state["residual"], eps=NORM_EPS)
    if kind == "norm_train":
        x, w = state["x"].detach().requires_grad_(True), state["w"].detach().requires_grad_(True)
        if state["residual"] is None:
            y, _ = nn.residual_norm(x, w, eps=NORM_EPS)
            return (y.detach(), *torch.autograd.grad(y, (x, w), state["dy"]))
        r = state["residual"].detach().requires_grad_(True)
        y, h = nn.residual_norm(x, w, residual=r, eps=NORM_EPS)
        return (y.detach(), h.detach(), *torch.autograd.grad((y, h), (x, r, w), (state["dy"], state["dh"])))
    if kind == "loss_score":
        return nn.vocabulary_loss(state["x"], state["w"], state["target"], reduction="none", ignore_index=IGNORED)
    if kind == "loss_train":
        x, w = state["x"].detach().requires_grad_(True), state["w"].detach().requires_grad_(True)
        loss = nn.vocabulary_loss(x, w, state["target"], reduction="mean", ignore_index=IGNORED)
        return (loss.detach(), *torch.autograd.grad(loss, (x, w)))
    scales = {"first_scales": state["ms"], "second_scales": state["vs"], "seed": SEED} if case["bits"] == 8 else {}
    scc.scc_adamw_step(state["w"], state["g"], state["m"], state["v"], LR, STEP, betas=BETAS, eps=ADAM_EPS, weight_decay=DECAY, **scales)
    return _lists(state)


def _lists(state):
    return {k: state[k] for k in ("w", "m", "v", "ms", "vs") if k in state}


# ---- the plain forms: elementary operations in 32 bits, rounded once at the end ----

def _plain_norm(state, case):
    dtype = state["x"].dtype
    h = state["x"].float()
    if state["residual"] is not None:
        h = h + state["residual"].float()
    w = state["w"].float().view(1, -1, 1, 1)
    rstd = torch.rsqrt(h.square().mean(1, keepdim=True) + NORM_EPS)
    hat = h * rstd
    y = hat * w
    if case["kind"] == "norm_infer":
        return y.to(dtype), h.to(dtype)
    if case["kind"] == "norm_8bit":
        scale = _power(y.abs().amax(1), 448.0)
        return (y / scale.unsqueeze(1)).to(torch.float8_e4m3fn), scale, h.to(dtype)
    dy = state["dy"].float()
    a = dy * w
    dx = (a - hat * (a * hat).mean(1, keepdim=True)) * rstd
    dw = (dy * hat).sum((0, 2, 3)).to(dtype)
    if state["residual"] is None:
        return y.to(dtype), dx.to(dtype), dw
    dx = (dx + state["dh"].float()).to(dtype)
    return y.to(dtype), h.to(dtype), dx, dx, dw


def _power(most, limit):
    """The smallest power of two that brings `most` to `limit` or less; 1 where there is nothing to bring."""
    mantissa, exponent = torch.frexp(most / limit)
    exponent = exponent - (mantissa == 0.5).int()
    return torch.where(most > 0, torch.ldexp(torch.ones_like(most), exponent.clamp(-120, 120)), 1.0)


def _plain_loss(state, case):
    N, C, H, W = state["x"].shape
    x = state["x"].float().flatten(2).transpose(1, 2).reshape(-1, C)
    w = state["w"].float()
    target = state["target"].flatten()
    counts = target != IGNORED
    target = torch.where(counts, target, 0)
    logits = x @ w.t()
    known = logits.gather(1, target[:, None])[:, 0]
    most = logits.amax(1, keepdim=True)
    p = logits.sub_(most).exp_()
    total = p.sum(1, keepdim=True)
    loss = torch.where(counts, total[:, 0].log() + (most[:, 0] - known), 0.0)
    if case["kind"] == "loss_score":
        return loss.view(N, H, W)
    count = counts.sum().clamp(min=1)
    mean = (loss.double().sum() / count).float()
    p.div_(total).scatter_add_(1, target[:, None], torch.full_like(total, -1.0))
    p.mul_((counts / count).float()[:, None])
    dx = (p @ w).view(N, H * W, C).transpose(1, 2).reshape(state["x"].shape)
    return mean, dx.to(state["x"].dtype), (p.t() @ x).to(state["w"].dtype)


def _plain_adamw(state, case):
    b1, b2 = BETAS
    for i, (w, g) in enumerate(zip(state["w"], state["g"])):
        g, small = g.float(), case["bits"] == 8
        m, v = state["m"][i], state["v"][i]
        if small:
            m = _from_blocks(m, state["ms"][i])
            v = _from_blocks(v, state["vs"][i])
            v = v * v
        m = m * b1 + g * (1.0 - b1)
        v = v * b2 + (g * g) * (1.0 - b2)
        update = (m / (1.0 - b1 ** STEP)) / ((v / (1.0 - b2 ** STEP)).sqrt() + ADAM_EPS)
        w.copy_(w.float() * (1.0 - LR * DECAY) - LR * update)
        if not small:
            state["m"][i].copy_(m)
            state["v"][i].copy_(v)
            continue
        random = _random(m.numel(), i, m.device)
        for name, new in (("m", m), ("v", v)):
            values, scales = _round_blocks(new, name == "v", random)
            state[name][i].copy_(values)
            state[name + "s"][i].copy_(scales)
    return _lists(state)


def _mix(x):
    """A permutation of 32-bit numbers in which each bit depends on all."""
    x = x & 0xffffffff
    x = ((x ^ (x >> 16)) * 0x6A09E667) & 0xffffffff
    x = ((x ^ (x >> 15)) * 0xBB67AE85) & 0xffffffff
    return x ^ (x >> 16)


def _random(n, index, device):
    key = _mix(_mix(SEED + STEP * 0x9E3779B1) + index * 0x9E3779B1)
    return _mix(torch.arange(n, device=device) + key)


def _blocks(t):
    flat = t.reshape(-1)
    return torch.nn.functional.pad(flat, (0, -flat.numel() % BLOCK)).view(-1, BLOCK)


def _exponents(most, root):
    """For each block the power of two that brings its largest value, or that one's root, into [128, 256)."""
    exponent = torch.frexp(most)[1] - 1
    exponent = (exponent >> 1 if root == 2 else exponent) - 7
    return torch.where(most > 0, exponent, -100).clamp(-100, 120)


def _from_blocks(values, scales):
    return (_blocks(values.float()) * scales[:, None]).view(-1)[:values.numel()].view(values.shape)


def _to_blocks(t, most, root):
    """t rounded to nearest: (e4m3, scales)."""
    exponent = _exponents(_blocks(most).amax(1), root)
    scales = torch.ldexp(torch.ones(exponent.shape, device=t.device), exponent)
    return (_blocks(t) / scales[:, None]).view(-1)[:t.numel()].view(t.shape).to(torch.float8_e4m3fn), scales


def _round_blocks(t, square, random):
    """t, or its root, in blocks: (e4m3, scales).  Between two neighbours the random number decides, so that the expectation is t."""
    n, shape = t.numel(), t.shape
    t, random = _blocks(t), _blocks(random)
    exponent = _exponents(t.abs().amax(1), 2 if square else 1)
    scales = torch.ldexp(torch.ones(exponent.shape, device=t.device), exponent)
    t = (t / scales[:, None]) / scales[:, None] if square else t / scales[:, None]
    a = t.double().sqrt() if square else t.double().abs()
    step = torch.ldexp(torch.ones_like(a), torch.frexp(a)[1].clamp(min=-5) - 4)
    low = (a / step).floor() * step
    if square:
        high = low + step
        up = (random >> 8).double() * 2.0 ** -24 * (high * high - low * low) < t.double() - low * low
        up |= (low == 0) & (t > 0)          # what is positive stays so
    else:
        up = ((((random & 0xffff) << 4) | 8) + ((a - low) / step * 2 ** 20).floor().long()) >> 20 > 0
    q = torch.where(up, low + step, low)
    q = (q if square else torch.where(t < 0, -q, q)).float()
    return q.view(-1)[:n].view(shape).to(torch.float8_e4m3fn), scales


def _run_plain(state):
    case = state["case"]
    if case["kind"] == "adamw":
        return _plain_adamw(state, case)
    return (_plain_norm if case["kind"].startswith("norm") else _plain_loss)(state, case)


# ---- the definitions in 64 bits ----

def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "adamw":
        b1, b2 = BETAS
        out = {"w": [], "m": [], "v": []}
        for i, w in enumerate(state["w"]):
            w, g = w.double().flatten(), state["g"][i].double().flatten()
            m, v = state["m"][i].double().flatten(), state["v"][i].double().flatten()
            if case["bits"] == 8:
                block = torch.arange(w.numel(), device=w.device) // BLOCK
                m, v = m * state["ms"][i].double()[block], (v * state["vs"][i].double()[block]) ** 2
            m, v = m + (1 - b1) * (g - m), v + (1 - b2) * (g ** 2 - v)
            root = torch.sqrt(v / -math.expm1(STEP * math.log(b2)))
            w = w - LR * (DECAY * w + m / -math.expm1(STEP * math.log(b1)) / (root + ADAM_EPS))
            out["w"].append(w.view(state["w"][i].shape))
            # a state in 8 bits has no value of its own: which neighbour it is rounded to is chance
            out["m"].append(m.view(state["w"][i].shape) if case["bits"] == 32 else None)
            out["v"].append(v.view(state["w"][i].shape) if case["bits"] == 32 else None)
        return out
    N, C, H, W = state["x"].shape
    rows = lambda t: t.double().movedim(1, -1).reshape(-1, C)   # noqa: E731  (tokens x channels)
    back = lambda t: t.view(N, H, W, C).movedim(-1, 1)          # noqa: E731
    x, w = rows(state["x"]), state["w"].double()
    if case["kind"].startswith("norm"):
        h = x if state["residual"] is None else x + rows(state["residual"])
        rms = torch.sqrt((h * h).sum(1) / C + NORM_EPS)
        y = h * w / rms[:, None]
        if case["kind"] == "norm_8bit":
            most = y.abs().amax(1)
            scale = torch.where(most > 0, torch.exp2(torch.ceil(torch.log2(most / 448.0))), torch.ones_like(most))
            return back(y / scale[:, None]), scale.view(N, H, W), back(h)
        if case["kind"] == "norm_infer":
            return back(y), back(h)
        dy = rows(state["dy"])
        inner = (dy * w * h).sum(1) / (C * rms ** 3)
        dx = dy * w / rms[:, None] - h * inner[:, None]
        dw = (dy * h / rms[:, None]).sum(0)
        if state["residual"] is None:
            return back(y), back(dx), dw
        dx = back(dx + rows(state["dh"]))
        return back(y), back(h), dx, dx, dw
    V, target = case["V"], state["target"].flatten()
    T = target.numel()
    kept = target.ne(IGNORED)
    piece = max(1, min(V, (1 << 28) // T))
    most = torch.full((T,), -math.inf, dtype=torch.float64, device=x.device)
    total = torch.zeros_like(most)
    for at in range(0, V, piece):
        logits = x @ w[at:at + piece].t()
        new = torch.maximum(most, logits.amax(1))
        total = total * torch.exp(most - new) + torch.exp(logits - new[:, None]).sum(1)
        most = new
    lse = most + torch.log(total)
    picked = w[target.clamp(min=0)]
    loss = torch.where(kept, lse - (x * picked).sum(1), 0.0)
    if case["kind"] == "loss_score":
        return loss.view(N, H, W)
    share = kept.double() / max(1, int(kept.sum()))
    dx = -picked * share[:, None]
    dw = torch.zeros_like(w).index_add_(0, target.clamp(min=0), -x * share[:, None])
    for at in range(0, V, piece):
        p = torch.exp(x @ w[at:at + piece].t() - lse[:, None]) * share[:, None]
        dx += p @ w[at:at + piece]
        dw[at:at + piece] += p.t() @ x
    return (loss * share).sum(), back(dx), dw


def work(case):
    """Inputs read once, outputs written once (of a training step: of its forward and of its backward), and the multiply-adds of the
    logits and their two gradients; of the rest some operations for each element."""
    es = 4 if case["dtype"] == "f32" else 2
    if case["kind"] == "adamw":
        n = sum(math.prod(s) for s in _shapes(case))
        return {"bytes": n * (3 * es + (16 if case["bits"] == 32 else 4)), "flops": 15 * n}
    N, C, H, W = (case[k] for k in ("N", "C", "H", "W"))
    T = N * H * W
    if case["kind"].startswith("norm"):
        n, streams = T * C, 2 if case["residual"] else 1
        total = n * es * (2 * streams) if case["kind"] != "norm_8bit" else n * (es * (2 * streams - 1) + 1) + 4 * T
        if case["kind"] == "norm_train":
            return {"bytes": total + n * es * (3 + (streams - 1)) + 3 * es * C, "flops": 16 * n}
        return {"bytes": total + es * C, "flops": 5 * n}
    V, train = case["V"], case["kind"] == "loss_train"
    inputs = es * C * (T + V) + 8 * T
    return {"bytes": inputs * (3 if train else 1) + 4 * T, "flops": (6 if train else 2) * T * C * V}
