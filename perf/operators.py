"""What the gated feed-forward operators are measured on: the gated sliding-channel layer that a feed-forward block opens with, its
training step, and the orthogonalised momentum update of such layers' weights.

A case is one of four kinds:

    gated_infer   y = act(SCC(x; w[0])) * SCC(x; w[1]) alone: serving, from one token to an evaluation batch
    gated_train   the same and, from dy, the gradients of x and of both weight matrices: a training step through autograd
    orthogonalise the Newton-Schulz products alone: matrices in, their orthogonalised forms out
    update        the optimiser's step on a list of weight matrices: momentum, Newton-Schulz, weight decay and the new weights

A gated layer is (N, Cin, Cout, H, W, cg, co, dtype, act); a sequence of S tokens is a map of S x 1, N single tokens are N maps of 1 x 1.
A list of matrices is a text of rows x columns.  Activations and gradients are N(0, 1), or half-normal activations where the layer sits
behind a ReLU, weights He-initialised as in scc_workloads.py.  The plain form multiplies by the dense Cout x Cin matrix with the windows' weights
in it: in elementary operations the widened matrix is the fastest way, and its zeros are not counted as work.
"""
import math

import torch

own = False     # whether run() calls the package's operators or computes them in elementary torch operations

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
NS_COEFFICIENTS = (3.4445, -4.7750, 2.0315)     # x -> a x + b x^3 + c x^5 on the singular values
NS_EPS = 1e-7
LR, MOMENTUM, DECAY = 0.02, 0.95, 0.01

# weights of the thirteen sliding-channel layers of the MobileNet-shaped stack at cg = 2
STACK = "64x16,128x32,128x64,256x64,256x128,512x128,512x256,512x256,512x256,512x256,512x256,1024x256,1024x512"

MAX_ELEMENTS = 128 * 512 * 1024                              # of a drawn layer's larger activation: the channel-expanding layer's
MAX_MACS = {"gated_infer": 128 * 1024 * 512 * 192,           # N * H * W * Cout * L of a drawn layer: that of the same layer, and in
            "gated_train": 128 * 1024 * 512 * 64}            # serving, which takes a third of the products, three times that
MAX_UPDATE = 6 * 1024 ** 3                                   # sum over a drawn list of short * short * long


def _gated(kind, N, Cin, Cout, H, W, cg, co, dtype="f32", act="silu", relu=False, name=None):
    case = {"kind": kind, "N": N, "Cin": Cin, "Cout": Cout, "H": H, "W": W, "cg": cg, "co": co, "dtype": dtype, "act": act, "relu": relu}
    if name:
        case["name"] = name
    return case


def _update(kind, shapes, dtype="f32", name=None):
    case = {"kind": kind, "shapes": shapes, "dtype": dtype}
    if name:
        case["name"] = name
    return case


def listed():
    return [
        # one token through a serving model's layer: the latency of a call, and a megabyte of weights read once
        _gated("gated_infer", 1, 512, 1024, 1, 1, 2, 0.5, dtype="bf16", name="serve_1_token_bf16"),
        # a batch of 48 requests' single tokens
        _gated("gated_infer", 48, 512, 1024, 1, 1, 2, 0.5, dtype="bf16", name="serve_48_tokens_bf16"),
        # the headline layer as a gated one, full precision, evaluation
        _gated("gated_infer", 128, 256, 256, 16, 16, 4, 0.5, name="eval_n128_c256_16x16"),
        # one channel group, so both projections are dense: eight prompts of 2000 tokens in mixed precision
        _gated("gated_infer", 8, 512, 1024, 2000, 1, 1, 0.5, dtype="bf16", act="gelu", name="prompt_8x2000_dense_bf16"),
        # late stage of an image network, behind a ReLU, mixed-precision training
        _gated("gated_train", 64, 512, 512, 14, 14, 8, 0.5, dtype="bf16", relu=True, name="train_n64_c512_14x14_bf16"),
        # last stage: odd map, a filter count off every tile, windows that start anywhere
        _gated("gated_train", 64, 512, 1000, 7, 7, 2, 0.33, act="gelu", name="train_n64_c512to1000_7x7"),
        # channel-expanding layer with windows that wrap several times, full precision: the largest activations
        _gated("gated_train", 128, 128, 512, 32, 32, 2, 0.33, name="train_n128_c128to512_32x32"),
        # tokens as rows, mixed-precision training
        _gated("gated_train", 4096, 256, 512, 1, 1, 2, 0.5, dtype="bf16", name="train_4096_tokens_bf16"),
        # one layer's weights: latency of a step
        _update("update", "256x64", name="update_256x64"),
        # all weights of the thirteen-layer stack in one step, full precision, and kept in bfloat16
        _update("update", STACK, name="update_stack"),
        _update("update", STACK, dtype="bf16", name="update_stack_bf16"),
        # gate, up and down matrices of two wide dense blocks, one side odd
        _update("orthogonalise", "1000x1024,1000x1024,1024x1000,1000x1024,1000x1024,1024x1000", name="orthogonalise_6_wide"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: gated layers from one token to the channel-expanding layer's size, lists of one to twelve matrices."""
    kind = rng.choice(["gated_infer", "gated_infer", "gated_train", "gated_train", "gated_train", "update", "update", "orthogonalise"])
    dtype = rng.choice(["f32", "bf16"])
    if not kind.startswith("gated"):
        shapes, left = [], MAX_UPDATE
        for _ in range(_log_uniform(rng, 1, 12)):
            rows, cols = _log_uniform(rng, 16, 1024), _log_uniform(rng, 16, 1024)
            cost = min(rows, cols) ** 2 * max(rows, cols)
            if cost <= left:
                shapes.append("%dx%d" % (rows, cols))
                left -= cost
        return _update(kind, ",".join(shapes), dtype=dtype)
    cg = rng.choice([1, 2, 2, 4, 4, 8])
    co = rng.choice([0.0, 0.25, 0.33, 0.5, 0.5, 0.75])
    unit = cg * rng.choice([8, 8, 8, 1])
    Cin = max(unit, _log_uniform(rng, 32, 1024) // unit * unit)
    Cout = max(8, int(Cin * rng.choice([0.5, 1, 1, 2, 2.5])) - rng.choice([0, 0, 0, 3]))
    form = rng.choice(["map", "map", "sequence", "tokens"])
    if form == "map":
        H = rng.choice([2, 4, 5, 7, 8, 12, 14, 16, 16, 20, 28, 32])
        W = H if rng.random() < 0.8 else rng.choice([4, 6, 7, 9, 16, 24])
    else:
        H, W = (_log_uniform(rng, 2, 4096) if form == "sequence" else 1), 1
    most = max(1, min(1024 if form == "map" else 65536, MAX_ELEMENTS // (max(Cin, Cout) * H * W), MAX_MACS[kind] // (Cout * (Cin // cg) * H * W)))
    N = _log_uniform(rng, 1, min(most, 64) if form == "sequence" else most)
    return _gated(kind, N, Cin, Cout, H, W, cg, co, dtype=dtype, act=rng.choice(["silu", "silu", "gelu"]), relu=rng.random() < 0.3)


def _windows(case):
    """(L, stride) of the layer's windows: filter k reads channels (k * stride + j) mod Cin, j < L."""
    L = case["Cin"] // case["cg"]
    return L, L - int(case["co"] * L)


def _shapes(case):
    return [tuple(int(v) for v in s.split("x")) for s in case["shapes"].split(",")]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dtype = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, relu=False):
        t = torch.randn(*shape, generator=gen, device="cuda")
        return ((t.abs() if relu else t) * std).to(dtype)

    if case["kind"].startswith("gated"):
        N, Cin, Cout, H, W = (case[k] for k in ("N", "Cin", "Cout", "H", "W"))
        L = _windows(case)[0]
        state = {"case": case, "x": normal(N, Cin, H, W, relu=case["relu"]), "w": normal(2, Cout, L, std=math.sqrt(2.0 / L))}
        if case["kind"] == "gated_train":
            state["dy"] = normal(N, Cout, H, W)
        return state
    state = {"case": case, "w": [], "g": [], "m": []}
    for rows, cols in _shapes(case):
        # a gradient: noise and a few directions that stand out of it
        few = normal(rows, 4, std=1.0).float() @ normal(4, cols, std=1.0).float()
        state["g"].append((normal(rows, cols).float() + few).mul_(0.01).to(dtype))
        if case["kind"] == "update":
            state["w"].append(normal(rows, cols, std=math.sqrt(2.0 / cols)))
            state["m"].append(normal(rows, cols, std=0.05).float())
    return state


def run(state):
    return (_run_own if own else _run_plain)(state)


def _run_own(state):
    import paper_2101_00745_amd as scc
    from paper_2101_00745_amd import nn

    case = state["case"]
    if case["kind"] == "gated_infer":
        return scc.scc_gated_forward(state["x"], state["w"], case["cg"], case["co"], act=case["act"])
    if case["kind"] == "gated_train":
        x, w = state["x"].detach().requires_grad_(True), state["w"].detach().requires_grad_(True)
        y = nn.gated_scc(x, w, case["cg"], case["co"], act=case["act"])
        y.backward(state["dy"])
        return y.detach(), x.grad, w.grad
    if case["kind"] == "orthogonalise":
        return scc.scc_orthogonalise(state["g"])
    scc.scc_orthogonal_step(state["w"], state["g"], state["m"], lr=LR, momentum=MOMENTUM, weight_decay=DECAY)
    return state["w"] + state["m"]


# ---- the plain forms: elementary operations in 32 bits, rounded once at the end ----

def _dense(w, case):
    """The 2 Cout x Cin matrix of both projections, and the channel that each weight multiplies."""
    (L, stride), Cin, Cout = _windows(case), case["Cin"], case["Cout"]
    k, j = torch.arange(Cout, device=w.device), torch.arange(L, device=w.device)
    channel = ((k * stride)[:, None] + j) % Cin
    channel = torch.cat([channel, channel])
    return torch.zeros(2 * Cout, Cin, device=w.device).scatter_(1, channel, w.float().reshape(2 * Cout, L)), channel


def _project(dense, x, tokens):
    return (x.flatten(1) @ dense.t()).view(x.shape[0], -1, 1) if tokens else dense @ x.flatten(2)


def _act(g, act):
    """act(g) and its derivative."""
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1.0 + g * (1.0 - s))
    phi = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return g * phi, phi + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))


def _newton_schulz(u):
    a, b, c = NS_COEFFICIENTS
    flip = u.shape[0] > u.shape[1]
    x = (u.t() if flip else u) / (u.norm() + NS_EPS)
    for _ in range(5):
        p = x @ x.t()
        x = a * x + (b * p + c * (p @ p)) @ x
    return x.t() if flip else x


def _run_plain(state):
    case = state["case"]
    if case["kind"] == "orthogonalise":
        return [_newton_schulz(g.float()).to(g.dtype) for g in state["g"]]
    if case["kind"] == "update":
        for w, g, m in zip(state["w"], state["g"], state["m"]):
            g = g.float()
            m.mul_(MOMENTUM).add_(g)
            o = _newton_schulz(g + MOMENTUM * m)
            w.copy_(w.float() * (1.0 - LR * DECAY) - LR * math.sqrt(max(1.0, w.shape[0] / w.shape[1])) * o)
        return state["w"] + state["m"]
    x, dtype, Cout = state["x"].float(), state["x"].dtype, case["Cout"]
    tokens = case["H"] * case["W"] == 1
    shape = (case["N"], Cout, case["H"], case["W"])
    dense, channel = _dense(state["w"], case)
    h = _project(dense, x, tokens)
    u = h[:, Cout:]
    a, da = _act(h[:, :Cout], case["act"])
    y = (a * u).view(shape).to(dtype)
    if case["kind"] == "gated_infer":
        return y
    dy = state["dy"].float().flatten(2)
    dh = torch.cat([dy * u * da, dy * a], 1)
    dx = _project(dense.t().contiguous(), dh, tokens).view(x.shape).to(dtype)
    columns = [t.flatten(2).transpose(0, 1).reshape(t.shape[1], -1) for t in (dh, x)]
    dw = (columns[0] @ columns[1].t()).gather(1, channel).view(state["w"].shape).to(dtype)
    return y, dx, dw


# ---- the definitions in 64 bits ----

def exact(case, seed):
    state = prepare(case, seed)
    if not case["kind"].startswith("gated"):
        outs, momenta = [], []
        for i, g in enumerate(state["g"]):
            u = g.double().cpu()
            if case["kind"] == "update":
                m = MOMENTUM * state["m"][i].double().cpu() + u
                momenta.append(m)
                u = u + MOMENTUM * m
            # an odd polynomial of a matrix acts on its singular values
            left, s, right = torch.linalg.svd(u, full_matrices=False)
            s = s / (s.square().sum().sqrt() + NS_EPS)
            a, b, c = NS_COEFFICIENTS
            for _ in range(5):
                s = s * (a + s * s * (b + s * s * c))
            o = (left * s) @ right
            if case["kind"] == "update":
                rows, cols = o.shape
                o = state["w"][i].double().cpu() * (1.0 - LR * DECAY) - LR * math.sqrt(max(1.0, rows / cols)) * o
            outs.append(o)
        return outs + momenta
    N, Cin, Cout, H, W = (case[k] for k in ("N", "Cin", "Cout", "H", "W"))
    L, stride = _windows(case)
    train = case["kind"] == "gated_train"
    x = state["x"].double().flatten(2).transpose(0, 1).reshape(Cin, -1)      # channels x columns
    w = state["w"].double()
    y = torch.empty(Cout, x.shape[1], dtype=torch.float64, device=x.device)
    if train:
        dy = state["dy"].double().flatten(2).transpose(0, 1).reshape(Cout, -1)
        dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    shared = {}
    for k in range(Cout):
        shared.setdefault(k * stride % Cin, []).append(k)
    for start, filters in shared.items():       # filters of one window at a time
        c = (torch.arange(L, device=x.device) + start) % Cin
        k = torch.tensor(filters, device=x.device)
        window = x[c]
        g, u = w[0][k] @ window, w[1][k] @ window
        if case["act"] == "silu":
            e = torch.exp(-g)
            a, slope = g / (1 + e), (1 + e + g * e) / (1 + e) ** 2
        else:
            a = g * 0.5 * torch.erfc(-g / math.sqrt(2.0))
            slope = 0.5 * torch.erfc(-g / math.sqrt(2.0)) + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        y[k] = a * u
        if train:
            dg, du = dy[k] * u * slope, dy[k] * a
            dx[c] += w[0][k].t().contiguous() @ dg + w[1][k].t().contiguous() @ du
            dw[0][k], dw[1][k] = dg @ window.t(), du @ window.t()

    def back(t, channels):
        return t.view(channels, N, H * W).transpose(0, 1).reshape(N, channels, H, W).cpu()

    return (back(y, Cout), back(dx, Cin), dw.cpu()) if train else back(y, Cout)


def work(case):
    """Inputs read once, outputs written once (of a training step: of its forward and of its backward), and the multiply-adds of the windows;
    of a Newton-Schulz step half of the two symmetric products."""
    es = 4 if case["dtype"] == "f32" else 2
    if case["kind"].startswith("gated"):
        train = case["kind"] == "gated_train"
        Q, L = case["N"] * case["H"] * case["W"], case["Cin"] // case["cg"]
        x, y, w = Q * case["Cin"], Q * case["Cout"], 2 * case["Cout"] * L
        total = es * (x + w + y) + (es * (2 * x + y + 2 * w) if train else 0)
        return {"bytes": total, "flops": (6 if train else 2) * Q * w}
    total = flops = 0
    for rows, cols in _shapes(case):
        short, long = min(rows, cols), max(rows, cols)
        total += rows * cols * (3 * es + 8 if case["kind"] == "update" else 2 * es)
        flops += 5 * short * short * (3 * long + short)
    return {"bytes": total, "flops": flops}
