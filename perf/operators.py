"""The operators around the quantised product, as models and training programs run them: the work that is measured, its plain form and its exact one.

Three operators.  `forward`: the layer as it stands in a model, with a bias, an activation, a second factor (gated layers) and a residual behind the product
of quantised weight and low-rank factors - one weight, several weights of a shape, several adapters on one weight.  `backward`: the gradient through what
stands behind the product.  `update`: the training step's last part, momentum and an update of the low-rank factors that Newton-Schulz products make
orthogonal.  Shapes, precision mixes, token counts and ranks are those of the benchmark's workloads and of the tests.

    Z = X deq(Wq)^T + s (X A) B + bias;   H = act(Z);   Y = H multiply + residual
    dZ = dY multiply act'(Z);   dmultiply = dY act(Z);   dbias = sum over the tokens of dZ
    m' = mu m + g;   u = g + mu m';   X = u / (|u| + eps);   five times X <- a X + X (b G + c G^2) with G = X^T X;   w' = (1 - lr wd) w - lr scale X
"""
import math

import numpy as np
import torch

own = False

# precision mixes: share of the output channels at 1, 2 and 4 bits
MIXES = {
    "1:50 2:50": (0.50, 0.50, 0.0),
    "1:30 2:50 4:20": (0.30, 0.50, 0.20),
    "1:60 2:35 4:5": (0.60, 0.35, 0.05),
    "1:85 2:15": (0.85, 0.15, 0.0),
    "2:75 4:25": (0.0, 0.75, 0.25),
    "4:100": (0.0, 0.0, 1.0),
}
LEVELS = {
    1: [-0.45, 0.45],
    2: [-0.75, -0.2, 0.25, 0.8],
    4: [-1.0, -0.7, -0.53, -0.4, -0.29, -0.19, -0.09, 0.0, 0.08, 0.16, 0.25, 0.34, 0.44, 0.56, 0.72, 1.0],
}
SCALE = 2.0                                        # s, the low-rank term's
ACTIVATIONS = ("none", "relu", "gelu", "gelu_tanh", "silu")
STEP = dict(lr=0.02, momentum=0.95, nesterov=True, weight_decay=0.01, steps=5, coefficients=(3.4445, -4.775, 2.0315), eps=1e-7)


def _layer(hidden, inner, r):
    """The low-rank factors of a decoder layer's seven matrices, A and B of each."""
    return " ".join(f"{K}x{r} {r}x{N}" for N, K in [(hidden, hidden)] * 4 + [(inner, hidden)] * 2 + [(hidden, inner)])


def _shapes(case):
    return [tuple(map(int, s.split("x"))) for s in case["shapes"].split()]


def listed():
    return [
        # generation for one user: a token through an attention block's output projection, added to the residual stream
        dict(name="token_residual", op="forward", N=4096, K=4096, mix="1:60 2:35 4:5", r=64, M=1, count=1, groups=0, activation="none", bias="", multiply=False,
             residual=True, pre=False),
        # a decode batch through the gate projection of a gated layer, the up projection's output at hand
        dict(name="decode_gated", op="forward", N=11008, K=4096, mix="1:60 2:35 4:5", r=64, M=16, count=1, groups=0, activation="silu", bias="", multiply=True,
             residual=False, pre=False),
        # several fine-tunes of a model with biases on one base weight: groups of a few tokens each
        dict(name="adapters_bias", op="forward", N=4096, K=4096, mix="1:30 2:50 4:20", r=64, M=101, count=1, groups=6, activation="none", bias="bf16", multiply=False,
             residual=True, pre=False),
        # a short prompt through the projection back to the residual stream
        dict(name="prompt_down", op="forward", N=4096, K=11008, mix="2:75 4:25", r=64, M=333, count=1, groups=0, activation="none", bias="fp32", multiply=False,
             residual=True, pre=False),
        # fine-tuning: the three attention projections of a layer with their biases, together
        dict(name="train_qkv_bias", op="forward", N=4096, K=4096, mix="1:30 2:50 4:20", r=64, M=2048, count=3, groups=0, activation="none", bias="bf16",
             multiply=False, residual=False, pre=False),
        # fine-tuning: the wide projection with its activation at a full batch, what the backward pass needs kept
        dict(name="train_gelu", op="forward", N=11008, K=4096, mix="1:60 2:35 4:5", r=64, M=4096, count=1, groups=0, activation="gelu", bias="bf16", multiply=False,
             residual=False, pre=True),
        # the gradient through it
        dict(name="backward_gelu", op="backward", N=11008, M=4096, activation="gelu", multiply=False, bias=True),
        # and through a gated layer, at a ragged batch
        dict(name="backward_gated", op="backward", N=13824, M=1001, activation="silu", multiply=True, bias=False),
        # a small layer, a few tokens: nothing but latency
        dict(name="backward_small", op="backward", N=1024, M=16, activation="relu", multiply=False, bias=True),
        # one small layer's two factors
        dict(name="update_pair", op="update", r=16, shapes="1024x16 16x4096", grad="bf16", nesterov=True, update=True),
        # the fourteen factors of a decoder layer
        dict(name="update_layer", op="update", r=64, shapes=_layer(4096, 11008, 64), grad="bf16", nesterov=True, update=False),
        # high rank, odd lengths, gradients added up over several batches
        dict(name="update_rank128", op="update", r=128, shapes="5120x128 128x13824 2304x128 128x1800 13824x128 128x5120", grad="fp32",
             nesterov=False, update=True),
    ]


_FORWARD_COST = 4096 * 11008 * 4096
_BACKWARD_COST = 4096 * 11008


def draw(rng):
    def spread(lo, hi, step):      # even over the logarithm, a multiple of step
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / step)) * step))

    op = rng.choice(["forward", "forward", "backward", "update"])
    if op == "forward":
        N, K = spread(512, 13824, 8), spread(512, 13824, 128)
        kind = rng.choice(["one", "one", "several", "adapters"])
        count = rng.choice([2, 3, 4]) if kind == "several" else 1
        M = spread(1, 4096, 1)
        if kind == "adapters":
            M = max(2, min(M, 512))
        M = max(1, min(M, _FORWARD_COST // (N * K * count)))
        return dict(op=op, N=N, K=K, mix=rng.choice(sorted(MIXES)), r=16 * rng.randint(1, 8), M=M, count=count, groups=min(M, rng.randint(2, 8)) if kind == "adapters" else 0,
                    activation=rng.choice(ACTIVATIONS), bias=rng.choice(["", "bf16", "fp32"]), multiply=rng.random() < 0.4, residual=rng.random() < 0.5,
                    pre=rng.random() < 0.4)
    if op == "backward":
        N = spread(512, 13824, 8)
        return dict(op=op, N=N, M=max(1, min(spread(1, 8192, 1), _BACKWARD_COST // N)), activation=rng.choice(ACTIVATIONS[1:]), multiply=rng.random() < 0.5,
                    bias=rng.random() < 0.5)
    r = 16 * rng.randint(1, 8)
    shapes = []
    for _ in range(rng.randint(1, 12)):
        L = spread(64, 13824, 8)
        shapes.append((L, r) if rng.random() < 0.5 else (r, L))
    while sum(a * b for a, b in shapes) > 78112 * 64:
        shapes.pop()
    return dict(op=op, r=r, shapes=" ".join(f"{a}x{b}" for a, b in shapes), grad=rng.choice(["bf16", "fp32"]), nesterov=rng.random() < 0.5, update=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed, k=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1000003 + k)
    return g


def _normal(g, shape, scale, dtype=torch.bfloat16):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _precisions(case, seed, i):
    N, (one, two, _) = case["N"], MIXES[case["mix"]]
    n1, n2 = int(round(one * N)), int(round(two * N))
    n2 = min(n2, N - n1)
    p = np.full(N, 4, dtype=np.uint8)
    p[:n1] = 1
    p[n1:n1 + n2] = 2
    if MIXES[case["mix"]][2] == 0.0:
        p[n1 + n2:] = 2
    np.random.default_rng([seed, i]).shuffle(p)
    return p


def _weight(case, seed, i, n_tables):
    """A quantised weight as the framework stores it: rows by precision, each row's codes one bit stream; codes, block maxima and levels at random."""
    N, K = case["N"], case["K"]
    g = _generator(seed, 10 + i)
    precs = _precisions(case, seed, i)
    perm = np.concatenate([np.flatnonzero(precs == b) for b in (1, 2, 4)])
    packed = torch.randint(0, 256, (int(precs.astype(np.int64).sum()) * K // 8,), generator=g, device="cuda", dtype=torch.uint8)
    sigma = torch.exp(torch.empty(N, device="cuda").uniform_(math.log(0.005), math.log(0.05), generator=g))
    absmax = sigma[:, None] * torch.empty((N, K // 64), device="cuda").uniform_(1.8, 3.4, generator=g)
    p = torch.from_numpy(precs).cuda()
    maps = torch.zeros((n_tables, N, 16), device="cuda")
    for b in (1, 2, 4):
        rows = (p == b).nonzero().flatten()
        if rows.numel():
            levels = torch.tensor(LEVELS[b], device="cuda")
            maps[:, rows, :1 << b] = levels + 0.03 * torch.randn((n_tables, rows.numel(), 1 << b), generator=g, device="cuda")
    return dict(precs=precs, perm=torch.from_numpy(perm).cuda(), counts=[int((precs == b).sum()) for b in (1, 2, 4)], packed=packed, absmax=absmax.contiguous(), maps=maps)


def _prepare_forward(case, seed):
    N, K, M, r, n = case["N"], case["K"], case["M"], case["r"], max(1, case["groups"])
    g = _generator(seed)
    X = _normal(g, (M, K), 1.0)
    members = []
    for i in range(case["count"]):
        w = _weight(case, seed, i, n)
        w["A"], w["B"] = _normal(g, (n, K, r), 0.01), _normal(g, (n, r, N), 0.01)
        w["bias"] = _normal(g, (N,), 0.3, torch.bfloat16 if case["bias"] == "bf16" else torch.float32) if case["bias"] else None
        w["multiply"] = _normal(g, (M, N), 1.0) if case["multiply"] else None
        w["residual"] = _normal(g, (M, N), 1.0) if case["residual"] else None
        members.append(w)
    cuts = np.sort(np.random.default_rng([seed, 77]).integers(0, M + 1, n - 1)) if case["groups"] else []
    state = dict(case=case, X=X, members=members, starts=[0, *map(int, cuts), M])
    if own:
        import paper_2502_08141_b200 as lw

        for w in members:
            w["layout"] = lw.Layout(w["precs"], K).build_deal()
            w["Y"] = torch.empty((M, N), dtype=torch.bfloat16, device="cuda")
            w["pre"] = torch.empty((M, N), dtype=torch.bfloat16, device="cuda") if case["pre"] else None
        layout = members[0]["layout"]
        size = (lw.lowra_batch_workspace_bytes(layout, 4 if case["groups"] else case["count"], M, r) if case["groups"] or case["count"] > 1
                else lw.lowra_workspace_bytes(layout, M, r))
        state["workspace"] = lw.lowra_workspace_init(torch.empty(size, dtype=torch.uint8, device="cuda"))
        state["batch"] = [dict(layout=w["layout"], packed=w["packed"], absmax=w["absmax"], maps=w["maps"][0], act=X, A=w["A"][0], B=w["B"][0], out=w["Y"],
                               bias=w["bias"], activation=case["activation"], multiply=w["multiply"], residual=w["residual"], pre=w["pre"]) for w in members]
    return state


def _prepare_backward(case, seed):
    g, M, N = _generator(seed), case["M"], case["N"]
    state = dict(case=case, dY=_normal(g, (M, N), 1e-3), pre=_normal(g, (M, N), 1.3), multiply=_normal(g, (M, N), 1.0) if case["multiply"] else None)
    if own:
        import paper_2502_08141_b200 as lw

        state["workspace"] = torch.empty(lw.lowra_epilogue_workspace_bytes(M, N), dtype=torch.uint8, device="cuda")
        state["dZ"] = torch.empty_like(state["dY"])
        state["dmultiply"] = torch.empty_like(state["dY"]) if case["multiply"] else None
        state["dbias"] = torch.empty(N, dtype=torch.float32, device="cuda") if case["bias"] else None
    return state


def _prepare_update(case, seed):
    g, r = _generator(seed), case["r"]
    members = []
    for i, (rows, cols) in enumerate(_shapes(case)):
        L = rows if cols == r else cols
        # a few directions of a gradient are strong, the others fall off
        fall = torch.exp(-torch.arange(r, device="cuda") * (5.0 / r))
        mix = torch.randn((r, r), generator=g, device="cuda") / math.sqrt(r)

        def tall(scale):
            return (torch.randn((L, r), generator=g, device="cuda") * fall) @ mix * scale

        grad, momentum, master = tall(1e-3), tall(1e-2), _normal(g, (L, r), 0.01, torch.float32)
        if cols != r or rows == r:
            grad, momentum, master = grad.t(), momentum.t(), master.t()
        members.append(dict(grad=grad.to(torch.bfloat16 if case["grad"] == "bf16" else torch.float32).contiguous(), momentum=momentum.contiguous(),
                            master=master.contiguous(), scale=math.sqrt(max(1.0, rows / cols))))
    state = dict(case=case, members=members)
    if own:
        import paper_2502_08141_b200 as lw

        for m in members:
            m["momentum_out"], m["master_out"] = torch.empty_like(m["momentum"]), torch.empty_like(m["master"])
            m["weight"] = torch.empty(m["master"].shape, dtype=torch.bfloat16, device="cuda")
            if case["update"]:
                m["update"] = torch.empty_like(m["master"])
        state["workspace"] = torch.empty(lw.lowra_update_workspace_bytes(_shapes(case), r), dtype=torch.uint8, device="cuda")
    return state


def prepare(case, seed):
    return {"forward": _prepare_forward, "backward": _prepare_backward, "update": _prepare_update}[case["op"]](case, seed)


# ------------------------------------------------------------------------------------------------ one pass
def _decoded(w, table, K):
    """deq(Wq) in 32 bits, rounded to bf16 as the weights of the layer are."""
    out, at, row = torch.empty((w["perm"].numel(), K), device="cuda"), 0, 0
    for b, n in zip((1, 2, 4), w["counts"]):
        if n == 0:
            continue
        size = n * K * b // 8
        shifts = torch.arange(0, 8, b, device="cuda", dtype=torch.uint8)
        codes = ((w["packed"][at:at + size].view(n, -1, 1) >> shifts) & ((1 << b) - 1)).view(n, K)
        rows = w["perm"][row:row + n]
        levels = torch.gather(table[rows], 1, codes.long())
        out[rows] = (levels.view(n, K // 64, 64) * w["absmax"][row:row + n, :, None]).view(n, K).bfloat16().float()
        at, row = at + size, row + n
    return out


def _activate(z, kind):
    if kind == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if kind == "gelu":
        return 0.5 * z * torch.erfc(z * -math.sqrt(0.5))
    if kind == "gelu_tanh":
        return z / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if kind == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _slope(z, kind):
    if kind == "relu":
        return (z > 0).to(z.dtype)
    if kind == "gelu":
        return 0.5 * torch.erfc(z * -math.sqrt(0.5)) + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    if kind == "gelu_tanh":
        k = 2 * math.sqrt(2 / math.pi)
        p = 1 / (1 + torch.exp(-k * (z + 0.044715 * z * z * z)))
        return p + z * p * (1 - p) * k * (1 + 3 * 0.044715 * z * z)
    if kind == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    return torch.ones_like(z)


def _plain_forward(state):
    case, X = state["case"], state["X"].float()
    out = []
    for w in state["members"]:
        parts = []
        for a, (m0, m1) in enumerate(zip(state["starts"], state["starts"][1:])):
            if m1 > m0:
                x = X[m0:m1]
                parts.append(x @ _decoded(w, w["maps"][a], case["K"]).t() + SCALE * ((x @ w["A"][a].float()) @ w["B"][a].float()))
        z = torch.cat(parts)
        if w["bias"] is not None:
            z = z + w["bias"].float()
        y = _activate(z, case["activation"])
        if w["multiply"] is not None:
            y = y * w["multiply"].float()
        if w["residual"] is not None:
            y = y + w["residual"].float()
        out.append(y.bfloat16())
        if case["pre"]:
            out.append(z.bfloat16())
    return out


def _plain_backward(state):
    case, dY, z = state["case"], state["dY"].float(), state["pre"].float()
    dh = dY if state["multiply"] is None else dY * state["multiply"].float()
    dz = dh * _slope(z, case["activation"])
    out = [dz.bfloat16()]
    if case["multiply"]:
        out.append((dY * _activate(z, case["activation"])).bfloat16())
    if case["bias"]:
        out.append(dz.sum(0))
    return out


def _plain_update(state):
    case, k = state["case"], STEP
    a, b, c = k["coefficients"]
    out = []
    for m in state["members"]:
        g = m["grad"].float()
        buf = k["momentum"] * m["momentum"] + g
        u = g + k["momentum"] * buf if case["nesterov"] else buf
        wide = u.shape[1] > u.shape[0]
        x = u.t() if wide else u
        x = x / (torch.sqrt((x * x).sum()) + k["eps"])
        for _ in range(k["steps"]):
            gram = x.t() @ x
            x = a * x + x @ (b * gram + c * (gram @ gram))
        x = x.t() if wide else x
        master = (1 - k["lr"] * k["weight_decay"]) * m["master"] - k["lr"] * m["scale"] * x
        out += [buf, master, master.bfloat16()]
        if case["update"]:
            out.append(x.contiguous())
    return out


def run(state):
    case = state["case"]
    if not own:
        return {"forward": _plain_forward, "backward": _plain_backward, "update": _plain_update}[case["op"]](state)
    import paper_2502_08141_b200 as lw

    if case["op"] == "backward":
        lw.lowra_epilogue_backward(state["dY"], state["pre"], case["activation"], multiply=state["multiply"], dZ=state["dZ"], dmultiply=state["dmultiply"],
                                   dbias=state["dbias"], workspace=state["workspace"])
        return [t for t in (state["dZ"], state["dmultiply"], state["dbias"]) if t is not None]
    if case["op"] == "update":
        lw.lowra_update_factors(state["members"], **{**STEP, "nesterov": case["nesterov"]}, workspace=state["workspace"])
        return [m[k] for m in state["members"] for k in ("momentum_out", "master_out", "weight", "update") if k in m]
    if case["count"] > 1:
        lw.lowra_lora_forward_batch_epilogue(state["batch"], SCALE, state["workspace"])
    else:
        w = state["members"][0]
        extra = dict(bias=w["bias"], activation=case["activation"], multiply=w["multiply"], residual=w["residual"], pre=w["pre"], Y=w["Y"], workspace=state["workspace"])
        if case["groups"]:
            lw.lowra_lora_forward_adapters_epilogue(w["layout"], w["packed"], w["absmax"], w["maps"], state["X"], state["starts"], w["A"], w["B"], SCALE, **extra)
        else:
            b = state["batch"][0]
            lw.lowra_lora_forward_epilogue(w["layout"], w["packed"], w["absmax"], b["maps"], state["X"], b["A"], b["B"], SCALE, **extra)
    return [t for w in state["members"] for t in (w["Y"], w["pre"]) if t is not None]


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["op"] == "backward":
        M, N = case["M"], case["N"]
        return dict(bytes=M * N * 2 * (5 if case["multiply"] else 3) + (4 * N if case["bias"] else 0), flops=M * N * (12 if case["activation"] != "relu" else 2))
    if case["op"] == "update":
        r, k = case["r"], STEP["steps"]
        size = [a * b for a, b in _shapes(case)]
        per = (2 if case["grad"] == "bf16" else 4) + 16 + 2 + (4 if case["update"] else 0)
        return dict(bytes=sum(size) * per, flops=sum(s * (r + 1) + 2 * s * r for s in size) + len(size) * (4 * k - 3) * 2 * r ** 3)
    N, K, M, r, n = case["N"], case["K"], case["M"], case["r"], max(1, case["groups"])
    counts = [int((_precisions(case, 0, 0) == b).sum()) for b in (1, 2, 4)]
    codes = sum(c * b for c, b in zip(counts, (1, 2, 4))) * K // 8
    tables = sum(c * 4 * (1 << b) for c, b in zip(counts, (1, 2, 4))) * n
    each = codes + N * (K // 64) * 4 + tables + n * 2 * r * (N + K) + {"": 0, "bf16": 2, "fp32": 4}[case["bias"]] * N
    each += M * N * 2 * (1 + case["multiply"] + case["residual"] + case["pre"])
    return dict(bytes=M * K * 2 + case["count"] * each, flops=case["count"] * (2 * M * N * K + 2 * M * r * (N + K)))


# ------------------------------------------------------------------------------------------------ the definition in 64 bits
def _exact_weight(w, table, precs, K):
    """Element k of stored row p: bits [k b, k b + b) of the row's stream, its row's level of that number times its block's maximum."""
    perm = w["perm"]
    b = torch.from_numpy(precs.astype(np.int64)).cuda()[perm]                       # of the stored rows
    start = torch.cumsum(b * K, 0) - b * K                                           # the rows' first bits
    W = torch.empty((perm.numel(), K), dtype=torch.float64, device="cuda")
    k = torch.arange(K, device="cuda")
    for p0 in range(0, perm.numel(), 1024):
        rows, bb = slice(p0, p0 + 1024), b[p0:p0 + 1024, None]
        bit = start[rows, None] + k * bb
        code = (w["packed"][bit // 8].long() >> (bit % 8)) % (1 << bb)
        flat = perm[rows, None] * 16 + code
        W[perm[rows]] = (table.reshape(-1)[flat] * w["absmax"][rows].repeat_interleave(64, 1)).to(torch.bfloat16).double()
    return W


def exact(case, seed):
    global own
    was, own = own, False
    try:
        state = prepare(case, seed)
    finally:
        own = was
    half = math.sqrt(0.5)
    phi = lambda z: 0.5 * torch.special.erfc(-z * half)  # noqa: E731
    c = math.sqrt(2 / math.pi)
    act = {
        "none": lambda z: z,
        "relu": lambda z: z.clamp_min(0.0),
        "gelu": lambda z: z * phi(z),
        "gelu_tanh": lambda z: 0.5 * z * (1 + torch.tanh(c * (z + 0.044715 * z ** 3))),
        "silu": lambda z: z * torch.sigmoid(z),
    }[case.get("activation", "none")]
    if case["op"] == "forward":
        out = []
        for i, w in enumerate(state["members"]):
            z = torch.empty((case["M"], case["N"]), dtype=torch.float64, device="cuda")
            for a in range(max(1, case["groups"])):
                m0, m1 = state["starts"][a], state["starts"][a + 1]
                if m1 > m0:
                    x = state["X"][m0:m1].double()
                    W = _exact_weight(w, w["maps"][a], w["precs"], case["K"])
                    z[m0:m1] = x @ W.t() + SCALE * (x @ w["A"][a].double() @ w["B"][a].double())
            if w["bias"] is not None:
                z += w["bias"].double()
            y = act(z)
            if w["multiply"] is not None:
                y = y * w["multiply"].double()
            if w["residual"] is not None:
                y = y + w["residual"].double()
            out.append(y)
            if case["pre"]:
                out.append(z)
        return out
    if case["op"] == "backward":
        z = state["pre"].double().requires_grad_(True)
        act(z).backward(torch.ones_like(z))
        dY = state["dY"].double()
        dz = dY * z.grad * (1.0 if state["multiply"] is None else state["multiply"].double())
        out = [dz]
        if case["multiply"]:
            out.append(dY * act(z.detach()))
        if case["bias"]:
            out.append(dz.sum(0))
        return out
    k = STEP
    out = []
    for m in state["members"]:
        g, old, w = m["grad"].double(), m["momentum"].double(), m["master"].double()
        new = k["momentum"] * old + g
        u = g + k["momentum"] * new if case["nesterov"] else new
        side = case["r"]
        x = u if u.shape[0] == side else u.t()
        x = x / (torch.linalg.norm(x) + k["eps"])
        for _ in range(k["steps"]):
            s = x @ x.t()
            x = k["coefficients"][0] * x + (k["coefficients"][1] * s + k["coefficients"][2] * s @ s) @ x
        x = x if u.shape[0] == side else x.t()
        master = w * (1 - k["lr"] * k["weight_decay"]) - k["lr"] * m["scale"] * x
        out += [new, master, master]
        if case["update"]:
            out.append(x)
    return out
