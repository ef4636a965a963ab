"""The operators of a training step beside the quantised products: the work that is measured, its plain form and its exact one.

Four operators.  `norm`: the norm before a layer's projections (layer norm or root mean square), with the residual stream's addition, forward and backward.
`rotary`: positions turned into the heads of queries and keys.  `loss`: cross entropy over the vocabulary straight from the hidden states, with the gradient
that starts the backward pass (the head is frozen, as the base weights are).  `adamw`: the optimiser's step over all factors together, states in 32 or in 8 bits.

    norm:    h = X + residual;  Y = (h - mu) / sqrt(var + eps) * weight + bias   (rms: mu = 0, no bias)
             dX = rstd (g - mean g - xh mean(g xh)) + dsum, g = dY * weight, xh = (h - mu) rstd;  dweight = sum dY xh;  dbias = sum dY
    rotary:  (a, b) -> scale * (a cos t - b sin t, b cos t + a sin t),  t = position * frequency;  the gradient turns back
    loss:    L = log sum_v exp(X W_v) - X W_label;  dX = scale * weight * (softmax - onehot) W
    adamw:   m' = b1 m + (1 - b1) g;  v' = b2 v + (1 - b2) g^2;  w' = w (1 - lr wd) - lr m' / (1 - b1^t) / (sqrt(v' / (1 - b2^t)) + eps)
             8 bits: of every 256 values m' / s and sqrt(v') / s as e4m3, s = largest / 448 (a root that is not zero is kept off zero)
"""
import math

import torch

own = False

EPS = 1e-5
STEP = dict(lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01)
T = 37                         # the optimiser's step
BLOCK = 256                    # values of a scale
LOSS_SCALE = 1.0 / 512
IGNORED = -100
SCALINGS = {                   # of the frequencies, for contexts longer than those trained on
    "none": dict(),
    "linear": dict(factor=4.0),
    "ntk": dict(factor=8.0),
    "yarn": dict(factor=16.0, original=4096, beta_fast=32.0, beta_slow=1.0),
    "bands": dict(factor=8.0, original=8192, low=1.0, high=4.0),
}


def _layer(hidden, inner, r):
    """The low-rank factors of a decoder layer's seven matrices, A and B of each."""
    return [s for N, K in [(hidden, hidden)] * 4 + [(inner, hidden)] * 2 + [(hidden, inner)] for s in ((K, r), (r, N))]


def _text(shapes):
    return " ".join(f"{a}x{b}" for a, b in shapes)


def _shapes(case):
    return [tuple(map(int, s.split("x"))) for s in case["shapes"].split()] * case["layers"]


def listed():
    return [
        # generation for one user: the norm before a block's projections, the residual stream added on the way
        dict(name="norm_token", op="norm", M=1, N=4096, kind="rms", backward=False, residual=True, params="bf16"),
        # a ragged prompt through a layer norm with bias
        dict(name="norm_prompt", op="norm", M=333, N=5120, kind="layer", backward=False, residual=True, params="fp32"),
        # fine-tuning, a full batch: backward with the weight's gradient, the residual stream's gradient added
        dict(name="norm_backward", op="norm", M=4096, N=4096, kind="rms", backward=True, residual=True, params="bf16"),
        # a small model's layer norm at a ragged batch
        dict(name="norm_backward_layer", op="norm", M=1001, N=1024, kind="layer", backward=True, residual=False, params="bf16"),
        # a decode batch far into long contexts, frequencies scaled, half of each head turned
        dict(name="rotary_tokens", op="rotary", M=16, q=32, k=8, D=128, R=64, interleaved=True, inverse=False, fused=False, far=1000000, scaling="yarn"),
        # fine-tuning: queries and keys of a full batch, slices of one projection
        dict(name="rotary_train", op="rotary", M=4096, q=32, k=32, D=128, R=128, interleaved=False, inverse=False, fused=True, far=4096, scaling="none"),
        # scoring a few tokens
        dict(name="loss_tokens", op="loss", M=16, V=32000, K=4096, grad=False, ignored=0.0, weighted=False),
        # a small model with a wide, odd vocabulary, padded batch
        dict(name="loss_wide", op="loss", M=777, V=50265, K=1024, grad=True, ignored=0.3, weighted=True),
        # fine-tuning: loss and gradient of a full batch
        dict(name="loss_train", op="loss", M=4096, V=32000, K=4096, grad=True, ignored=0.05, weighted=False),
        # one small layer's two factors
        dict(name="adamw_pair", op="adamw", shapes="1024x16 16x4096", layers=1, grad="bf16", bits=32, clip=False),
        # a decoder layer's fourteen factors, states in 8 bits, the gradient's norm clipped
        dict(name="adamw_layer_8bit", op="adamw", shapes=_text(_layer(4096, 11008, 64)), layers=1, grad="bf16", bits=8, clip=True),
        # all factors of a model of 32 layers
        dict(name="adamw_model", op="adamw", shapes=_text(_layer(4096, 11008, 64)), layers=32, grad="bf16", bits=32, clip=False),
    ]


def draw(rng):
    def spread(lo, hi, step=1):      # even over the logarithm, a multiple of step
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))

    op = rng.choice(["norm", "rotary", "loss", "adamw"])
    if op == "norm":
        N = spread(256, 13824, 8)
        kind = rng.choice(["layer", "rms"])
        return dict(op=op, M=max(1, min(spread(1, 8192), 4096 * 4096 // N)), N=N, kind=kind, backward=rng.random() < 0.6, residual=rng.random() < 0.5,
                    params=rng.choice(["bf16", "fp32"]))
    if op == "rotary":
        D = rng.choice([64, 80, 96, 128, 256])
        q = spread(1, 64)
        k = max(1, q // rng.choice([1, 2, 4, 8]))
        M = max(1, min(spread(1, 8192), 4096 * 64 * 128 // ((q + k) * D)))
        return dict(op=op, M=M, q=q, k=k, D=D, R=rng.choice([D, D // 32 * 16, 32]), interleaved=rng.random() < 0.5, inverse=rng.random() < 0.4,
                    fused=rng.random() < 0.5, far=spread(64, 2000000), scaling=rng.choice(sorted(SCALINGS)))
    if op == "loss":
        V, K, grad = spread(500, 60000), spread(256, 5120, 8), rng.random() < 0.7
        return dict(op=op, M=max(1, min(spread(1, 4096), 4096 * 32000 * 4096 // (V * K))), V=V, K=K, grad=grad, ignored=rng.choice([0.0, 0.1, 0.5]),
                    weighted=rng.random() < 0.5)
    shapes = [(spread(1, 4096), spread(1, 13824)) for _ in range(rng.randint(1, 40))]
    shapes = [(a, max(1, min(b, 4000000 // a))) for a, b in shapes]
    return dict(op=op, shapes=_text(shapes), layers=1, grad=rng.choice(["bf16", "fp32"]), bits=rng.choice([8, 32]), clip=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + 17)
    return g


def _normal(g, shape, scale, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _params(case):
    return torch.bfloat16 if case["params"] == "bf16" else torch.float32


def _prepare_norm(case, seed):
    g, M, N, layer = _generator(seed), case["M"], case["N"], case["kind"] == "layer"
    # a residual stream: some channels far larger than the others, tokens of unequal size
    size = torch.exp(0.8 * torch.randn(N, generator=g, device="cuda"))
    X = (torch.randn((M, N), generator=g, device="cuda") * size * torch.exp(0.3 * torch.randn((M, 1), generator=g, device="cuda")) + 0.05).bfloat16()
    weight = (1 + 0.2 * torch.randn(N, generator=g, device="cuda")).to(_params(case))
    bias = (0.1 * torch.randn(N, generator=g, device="cuda")).to(_params(case)) if layer else None
    other = _normal(g, (M, N), 0.5 if not case["backward"] else 1e-3) if case["residual"] else None
    state = dict(case=case, X=X, weight=weight, bias=bias, other=other)
    if case["backward"]:
        x = X.double()
        mean = x.mean(1) if layer else torch.zeros(M, dtype=torch.float64, device="cuda")
        state["mean"] = mean.float() if layer else None
        state["rstd"] = (1 / torch.sqrt(((x - mean[:, None]) ** 2).mean(1) + EPS)).float()
        state["dY"] = _normal(g, (M, N), 1e-3)
    if own:
        import paper_2502_08141_b200 as lw

        state["Y"] = torch.empty_like(X)
        if case["backward"]:
            state["dweight"] = torch.empty(N, dtype=torch.float32, device="cuda")
            state["dbias"] = torch.empty(N, dtype=torch.float32, device="cuda") if layer else None
            state["workspace"] = torch.empty(lw.lowra_norm_workspace_bytes(M, N), dtype=torch.uint8, device="cuda")
        else:
            state["sum"] = torch.empty_like(X) if case["residual"] else None
            state["mean"] = torch.empty(M, dtype=torch.float32, device="cuda") if layer else None
            state["rstd"] = torch.empty(M, dtype=torch.float32, device="cuda")
    return state


def _frequencies(case):
    """Of the pairs of a head, in radians a position, and the factor of the turned values."""
    R, base, kind, s = case["R"], 10000.0, case["scaling"], SCALINGS[case["scaling"]]
    if kind == "ntk" and R > 2:
        base *= s["factor"] ** (R / (R - 2))
    f = [base ** (-2.0 * i / R) for i in range(R // 2)]
    if kind == "linear":
        f = [x / s["factor"] for x in f]
    if kind == "yarn":
        place = lambda turns: R * math.log(s["original"] / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        low, high = max(math.floor(place(s["beta_fast"])), 0), min(math.ceil(place(s["beta_slow"])), R - 1)
        ramp = [min(max((i - low) / max(high - low, 0.001), 0.0), 1.0) for i in range(R // 2)]
        f = [x * (1 - t) + x / s["factor"] * t for x, t in zip(f, ramp)]
    if kind == "bands":
        share = [min(max((s["original"] * x / (2 * math.pi) - s["low"]) / (s["high"] - s["low"]), 0.0), 1.0) for x in f]
        f = [x * t + x / s["factor"] * (1 - t) for x, t in zip(f, share)]
    return f, (0.1 * math.log(s["factor"]) + 1.0 if kind == "yarn" else 1.0)


def _prepare_rotary(case, seed):
    g, M, D, q, k = _generator(seed), case["M"], case["D"], case["q"], case["k"]
    if case["fused"]:                # queries, keys and values of a token side by side
        qkv = _normal(g, (M, q + 2 * k, D), 1.0)
        parts = [qkv[:, :q], qkv[:, q:q + k]]
    else:
        parts = [_normal(g, (M, q, D), 1.0), _normal(g, (M, k, D), 1.0)]
    # a batch of sequences, each with its own start
    start = torch.randint(0, case["far"], (1 + M // 512,), generator=g, device="cuda")
    at = torch.arange(M, device="cuda")
    positions = (start[at // 512] + at % 512).to(torch.int32)
    frequencies, factor = _frequencies(case)
    state = dict(case=case, parts=parts, positions=positions, frequencies=torch.tensor(frequencies, dtype=torch.float64, device="cuda"), factor=factor)
    if own:
        import paper_2502_08141_b200 as lw

        turns, state["scale"] = lw.lowra_rotary_turns(case["R"], 10000.0, case["scaling"], **SCALINGS[case["scaling"]])
        state["turns"] = torch.from_numpy(turns.view("int64")).cuda()
        state["out"] = [torch.empty((M, n, D), dtype=torch.bfloat16, device="cuda") for n in (q, k)]
    return state


def _prepare_loss(case, seed):
    g, M, V, K = _generator(seed), case["M"], case["V"], case["K"]
    spread = 2.5
    W = _normal(g, (V, K), spread / math.sqrt(K))
    labels = torch.randint(0, V, (M,), generator=g, device="cuda")
    # from tokens that the model has no idea of to tokens that it is all but sure of
    known = 14.0 * torch.rand((M, 1), generator=g, device="cuda") * (torch.rand((M, 1), generator=g, device="cuda") < 0.6)
    X = (torch.randn((M, K), generator=g, device="cuda") + known / spread ** 2 * W[labels].float()).bfloat16()
    labels = torch.where(torch.rand(M, generator=g, device="cuda") < case["ignored"], torch.full_like(labels, IGNORED), labels)
    weights = torch.rand(M, generator=g, device="cuda") + 0.5 if case["weighted"] else None
    state = dict(case=case, X=X, W=W, labels=labels, weights=weights)
    if own:
        import paper_2502_08141_b200 as lw

        state["loss"] = torch.empty(M, dtype=torch.float32, device="cuda")
        state["dX"] = torch.empty_like(X) if case["grad"] else None
        state["workspace"] = torch.empty(lw.lowra_cross_entropy_workspace_bytes(M, V, K, case["grad"]), dtype=torch.uint8, device="cuda")
    return state


def _encode(values):
    """What is kept of values in 8 bits: every BLOCK of them over its scale, and the scales."""
    rows = values.view(-1, BLOCK)
    scale = rows.abs().amax(1) * (1.0 / 448)
    over = torch.where(scale > 0, 1 / scale, torch.zeros_like(scale))
    return (rows * over[:, None]).view(-1), scale


def _prepare_adamw(case, seed):
    g, eight = _generator(seed), case["bits"] == 8
    # the factors' arrays lie one behind the other in one buffer of each kind, from multiples of BLOCK on
    shapes, starts = _shapes(case), [0]
    for a, b in shapes:
        starts.append(starts[-1] + (a * b + BLOCK - 1) // BLOCK * BLOCK)
    n = starts[-1]
    size = torch.zeros(n, device="cuda")
    for (a, b), at in zip(shapes, starts):
        # a gradient's rows and columns are of very unequal size
        size[at:at + a * b] = (torch.exp(torch.randn((a, 1), generator=g, device="cuda")) * torch.exp(torch.randn((1, b), generator=g, device="cuda")) * 1e-4).view(-1)
    draw_ = lambda: torch.randn(n, generator=g, device="cuda")  # noqa: E731
    flat = dict(grad=(draw_() * size).to(torch.bfloat16 if case["grad"] == "bf16" else torch.float32), master=draw_() * 0.01 * (size > 0))
    first, second = draw_() * size * 0.3, (draw_() ** 2 + 0.1) * size ** 2 * 0.1
    if eight:
        x, flat["m_scale"] = _encode(first)
        flat["m"] = x.to(torch.float8_e4m3fn)
        x, flat["v_scale"] = _encode(torch.sqrt(second))
        flat["v"] = torch.where(x > 0, x.clamp_min(2.0 ** -9), x).to(torch.float8_e4m3fn)
    else:
        flat["m"], flat["v"] = first, second
    state = dict(case=case, flat=flat, clip=torch.full((1,), 0.37, device="cuda") if case["clip"] else None)
    if own:
        for name in ("master", "m", "v") + (("m_scale", "v_scale") if eight else ()):
            flat[name + "_out"] = torch.zeros_like(flat[name])
        flat["weight"] = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
        state["members"] = []
        for (a, b), at in zip(shapes, starts):
            end, blocks = at + a * b, (a * b + BLOCK - 1) // BLOCK
            state["members"].append({k: t[at // BLOCK:at // BLOCK + blocks] if "scale" in k else t[at:end].view(a, b) for k, t in flat.items()})
    return state


def prepare(case, seed):
    return {"norm": _prepare_norm, "rotary": _prepare_rotary, "loss": _prepare_loss, "adamw": _prepare_adamw}[case["op"]](case, seed)


# ------------------------------------------------------------------------------------------------ one pass
def _plain_norm(state):
    case, layer = state["case"], state["case"]["kind"] == "layer"
    weight = state["weight"].float()
    if not case["backward"]:
        h, out = state["X"], []
        if case["residual"]:
            h = (h.float() + state["other"].float()).bfloat16()
            out = [h]
        h = h.float()
        mean = h.mean(1, keepdim=True) if layer else torch.zeros_like(h[:, :1])
        rstd = 1 / torch.sqrt(((h - mean) ** 2).mean(1, keepdim=True) + EPS)
        y = (h - mean) * rstd * weight
        if layer:
            y = y + state["bias"].float()
        return [y.bfloat16(), rstd[:, 0]] + ([mean[:, 0]] if layer else []) + out
    dY, rstd = state["dY"].float(), state["rstd"][:, None]
    xh = state["X"].float()
    if layer:
        xh = xh - state["mean"][:, None]
    xh = xh * rstd
    g = dY * weight
    dx = g - xh * (g * xh).mean(1, keepdim=True)
    if layer:
        dx = dx - g.mean(1, keepdim=True)
    dx = dx * rstd
    if case["residual"]:
        dx = dx + state["other"].float()
    return [dx.bfloat16(), (dY * xh).sum(0)] + ([dY.sum(0)] if layer else [])


def _plain_rotary(state):
    case, out = state["case"], []
    R, factor = case["R"], state["factor"]
    angle = state["positions"].double()[:, None] * state["frequencies"]
    c, s = (torch.cos(angle) * factor).float()[:, None], (torch.sin(angle) * factor).float()[:, None]
    if case["inverse"]:
        s = -s
    for x in state["parts"]:
        x = x.float()
        y = x.clone()
        if case["interleaved"]:
            a, b = x[..., 0:R:2], x[..., 1:R:2]
            y[..., 0:R:2], y[..., 1:R:2] = a * c - b * s, b * c + a * s
        else:
            a, b = x[..., :R // 2], x[..., R // 2:R]
            y[..., :R // 2], y[..., R // 2:R] = a * c - b * s, b * c + a * s
        out.append(y.bfloat16())
    return out


def _plain_loss(state):
    W, labels = state["W"].float(), state["labels"]
    counts = labels != IGNORED
    logits = state["X"].float() @ W.t()
    most = logits.amax(1, keepdim=True)
    e = torch.exp(logits - most)
    total = e.sum(1, keepdim=True)
    at = torch.where(counts, labels, torch.zeros_like(labels))[:, None]
    loss = torch.where(counts, (most + torch.log(total) - logits.gather(1, at))[:, 0], torch.zeros_like(total[:, 0]))
    if not state["case"]["grad"]:
        return [loss]
    p = e / total
    p.scatter_add_(1, at, torch.full_like(total, -1.0))
    each = counts.float() * LOSS_SCALE
    if state["weights"] is not None:
        each = each * state["weights"]
    return [loss, ((p @ W) * each[:, None]).bfloat16()]


def _plain_adamw(state):
    k, w = STEP, state["flat"]
    b1, b2 = k["betas"]
    eight = state["case"]["bits"] == 8
    g = w["grad"].float()
    if state["clip"] is not None:
        g = g * state["clip"]
    if eight:
        m = (w["m"].float().view(-1, BLOCK) * w["m_scale"][:, None]).view(-1)
        root = (w["v"].float().view(-1, BLOCK) * w["v_scale"][:, None]).view(-1)
        v = root * root
    else:
        m, v = w["m"], w["v"]
    m = b1 * m + (1 - b1) * g
    v = b2 * v + ((1 - b2) * g) * g
    root = torch.sqrt(v)
    master = w["master"] * (1 - k["lr"] * k["weight_decay"]) - (k["lr"] / (1 - b1 ** T)) * m / (root * (1 / math.sqrt(1 - b2 ** T)) + k["eps"])
    if not eight:
        return [master, master.bfloat16(), m, v]
    x, m_scale = _encode(m)
    y, v_scale = _encode(root)
    y = torch.where(y > 0, y.clamp_min(2.0 ** -9), y)
    return [master, master.bfloat16(), x.to(torch.float8_e4m3fn), m_scale, y.to(torch.float8_e4m3fn), v_scale]


def run(state):
    case = state["case"]
    if not own:
        return {"norm": _plain_norm, "rotary": _plain_rotary, "loss": _plain_loss, "adamw": _plain_adamw}[case["op"]](state)
    import paper_2502_08141_b200 as lw

    if case["op"] == "norm":
        if case["backward"]:
            lw.lowra_norm_backward(state["dY"], state["X"], state["weight"], state["rstd"], mean=state["mean"], dsum=state["other"], dX=state["Y"],
                                   dweight=state["dweight"], dbias=state["dbias"], workspace=state["workspace"])
            return [t for t in (state["Y"], state["dweight"], state["dbias"]) if t is not None]
        lw.lowra_norm_forward(state["X"], state["weight"], state["bias"], eps=EPS, kind=case["kind"], residual=state["other"], sum=state["sum"], Y=state["Y"],
                              mean=state["mean"], rstd=state["rstd"])
        return [t for t in (state["Y"], state["rstd"], state["mean"], state["sum"]) if t is not None]
    if case["op"] == "rotary":
        lw.lowra_rotary(state["parts"][0], state["positions"], state["turns"], k=state["parts"][1], interleaved=case["interleaved"], inverse=case["inverse"],
                        scale=state["scale"], out=state["out"][0], k_out=state["out"][1])
        return state["out"]
    if case["op"] == "loss":
        lw.lowra_cross_entropy(state["X"], state["W"], state["labels"], scale=LOSS_SCALE, weights=state["weights"], ignore_index=IGNORED, loss=state["loss"],
                               dX=state["dX"], workspace=state["workspace"])
        return [t for t in (state["loss"], state["dX"]) if t is not None]
    lw.lowra_adamw(state["members"], step=T, grad_scale=state["clip"], **STEP)
    names = ("master_out", "weight") + (("m_out", "m_scale_out", "v_out", "v_scale_out") if case["bits"] == 8 else ("m_out", "v_out"))
    return [state["flat"][name] for name in names]


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["op"] == "norm":
        n, layer = case["M"] * case["N"], case["kind"] == "layer"
        p = case["N"] * (2 if case["params"] == "bf16" else 4)
        if case["backward"]:
            return dict(bytes=n * 2 * (4 if case["residual"] else 3) + p + case["N"] * 4 * (2 if layer else 1) + case["M"] * 4 * (2 if layer else 1), flops=n * 12)
        return dict(bytes=n * 2 * (4 if case["residual"] else 2) + p * (2 if layer else 1) + case["M"] * 4 * (2 if layer else 1), flops=n * 6)
    if case["op"] == "rotary":
        n = case["M"] * (case["q"] + case["k"])
        return dict(bytes=n * case["D"] * 4 + case["M"] * 4 + case["R"] * 4, flops=n * case["R"] * 3)
    if case["op"] == "loss":
        M, V, K = case["M"], case["V"], case["K"]
        return dict(bytes=V * K * 2 + M * K * 2 * (2 if case["grad"] else 1) + M * 12, flops=2 * M * V * K * (2 if case["grad"] else 1))
    n = sum(a * b for a, b in _shapes(case))
    scales = sum((a * b + BLOCK - 1) // BLOCK for a, b in _shapes(case))
    state = n * 16 if case["bits"] == 32 else n * 4 + scales * 16
    return dict(bytes=n * ((2 if case["grad"] == "bf16" else 4) + 8 + 2) + state, flops=n * 15)


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _exact_eight(values, floor):
    """Values over their blocks' scales in 8 bits, and the scales."""
    rows = values.reshape(-1, BLOCK)
    scale = rows.abs().max(1).values / 448
    x = rows / torch.where(scale == 0, torch.ones_like(scale), scale).unsqueeze(1)
    if floor:
        x = torch.where((x > 0) & (x < 2.0 ** -9), torch.full_like(x, 2.0 ** -9), x)
    return x.flatten().float().to(torch.float8_e4m3fn), scale


def exact(case, seed):
    global own
    was, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = was
    if case["op"] == "norm":
        layer, w = case["kind"] == "layer", state["weight"].double()
        if not case["backward"]:
            h, out = state["X"].double(), []
            if case["residual"]:
                h = h + state["other"].double()
                out = [h]
                h = h.to(torch.bfloat16).double()
            mu = h.sum(1) / case["N"] * (1.0 if layer else 0.0)
            d = h - mu.unsqueeze(1)
            rstd = ((d * d).sum(1) / case["N"] + EPS) ** -0.5
            y = d * rstd.unsqueeze(1) * w + (state["bias"].double() if layer else 0.0)
            return [y, rstd] + ([mu] if layer else []) + out
        # with the statistics as they were kept
        dY, x, rstd = state["dY"].double(), state["X"].double(), state["rstd"].double().unsqueeze(1)
        xh = (x - (state["mean"].double().unsqueeze(1) if layer else 0.0)) * rstd
        g = dY * w
        along = torch.einsum("mn,mn->m", g, xh) / case["N"]
        dx = rstd * (g - along.unsqueeze(1) * xh - (g.sum(1, keepdim=True) / case["N"] if layer else 0.0))
        if case["residual"]:
            dx = dx + state["other"].double()
        return [dx, torch.einsum("mn,mn->n", dY, xh)] + ([dY.sum(0)] if layer else [])
    if case["op"] == "rotary":
        f, factor = _frequencies(case)
        turn = torch.outer(state["positions"].double(), torch.tensor(f, dtype=torch.float64, device="cuda"))
        z = torch.polar(torch.full_like(turn, factor), -turn if case["inverse"] else turn).unsqueeze(1)
        out, R = [], case["R"]
        for x in state["parts"]:
            y = x.double().clone()
            pairs = y[..., :R].reshape(*y.shape[:2], R // 2, 2) if case["interleaved"] else torch.stack([y[..., :R // 2], y[..., R // 2:R]], -1)
            turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * z)
            y[..., :R] = turned.flatten(-2) if case["interleaved"] else torch.cat([turned[..., 0], turned[..., 1]], -1)
            out.append(y)
        return out
    if case["op"] == "loss":
        W, loss, dX = state["W"].double(), [], []
        for i in range(0, case["M"], 512):
            x, y = state["X"][i:i + 512].double(), state["labels"][i:i + 512]
            keep = (y != IGNORED).double()
            logp = torch.log_softmax(x @ W.t(), 1)
            pick = torch.zeros_like(logp)
            rows = torch.nonzero(keep).flatten()
            pick[rows, y[rows]] = 1.0
            loss.append(-(logp * pick).sum(1))
            if case["grad"]:
                c = keep * LOSS_SCALE
                if state["weights"] is not None:
                    c = c * state["weights"][i:i + 512].double()
                dX.append(((torch.exp(logp) - pick) * c.unsqueeze(1)) @ W)
        return [torch.cat(loss)] + ([torch.cat(dX)] if case["grad"] else [])
    w, (b1, b2), eight = state["flat"], STEP["betas"], case["bits"] == 8
    g, m, v = w["grad"].double(), w["m"].double(), w["v"].double()
    if state["clip"] is not None:
        g = g * state["clip"].double()
    if eight:
        m, v = m * w["m_scale"].double().repeat_interleave(BLOCK), (v * w["v_scale"].double().repeat_interleave(BLOCK)) ** 2
    m, v = m + (1 - b1) * (g - m), v + (1 - b2) * (g * g - v)
    master = w["master"].double()
    master = master - STEP["lr"] * (STEP["weight_decay"] * master + m / (1 - b1 ** T) / ((v / (1 - b2 ** T)).sqrt() + STEP["eps"]))
    return [master, master] + ([*_exact_eight(m, False), *_exact_eight(v.sqrt(), True)] if eight else [m, v])
