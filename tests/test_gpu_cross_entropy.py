"""Cross entropy from hidden states and its gradient against fp64, elementwise within counted roundings: products accumulated in fp32 (2^-23 of the sum of magnitudes for each of K / 16 + 8
additions, however they round), exponentials to 2^-19 and, as a factor of the second product, to bf16 (2^-8)."""
import pytest
import torch

import paper_2502_08141_b200 as lw

pytestmark = pytest.mark.gpu
IGNORE = -100


def make(M, V, K, seed=0, spread=2.0, known=0.0, ignored=0.2):
    g = torch.Generator(device="cuda").manual_seed(seed * 131 + M + 7 * V + 13 * K)
    W = (torch.randn((V, K), generator=g, device="cuda") * spread / K ** 0.5).bfloat16()
    labels = torch.randint(0, V, (M,), generator=g, device="cuda")
    X = (torch.randn((M, K), generator=g, device="cuda") + known / spread ** 2 * W[labels].float()).bfloat16()
    labels[torch.rand(M, generator=g, device="cuda") < ignored] = IGNORE
    return X, W, labels, torch.rand(M, generator=g, device="cuda") + 0.5


def reference(X, W, labels, weights, scale, grad):
    """loss, its tolerance, dX, its tolerance, a few tokens at a time"""
    V, K = W.shape
    Wd, Wa = W.double(), W.double().abs()
    out = []
    for x, y, c in zip(X.split(256), labels.split(256), weights.split(256)):
        x, c = x.double(), c.double() * scale * (y != IGNORE)
        l = x @ Wd.t()
        off = 2.0 ** -23 * (K / 16 + 8) * (x.abs() @ Wa.t()).amax(1)      # of a logit
        at = torch.where(y == IGNORE, 0, y)[:, None]
        rest = l.scatter(1, at, float("-inf"))                             # the others
        ly, top = l.gather(1, at)[:, 0], rest.amax(1)
        lse = torch.logsumexp(rest, 1)                                     # minus infinity for a vocabulary of one
        loss = torch.where(lse > ly, lse - ly + torch.log1p(torch.exp(ly - lse)), torch.log1p(torch.exp(lse - ly)))
        q = 1 / (1 + torch.exp(ly - lse))                                  # 1 - p of the label
        counts = (y != IGNORE).double()
        out.append([loss * counts, counts * ((2 * off + 2.0 ** -19) * q + 2.0 ** -21 * loss + 1e-37)])
        if grad:
            p = torch.exp(rest - lse[:, None]) * q[:, None] if V > 1 else torch.zeros_like(rest)
            dx, wide, own = p @ Wd, p @ Wa, q[:, None] * Wa[at[:, 0]]
            dx = (dx - q[:, None] * Wd[at[:, 0]]) * c[:, None]
            few = (2 * off + 2.0 ** -18)[:, None]
            tol = c[:, None] * (wide * (2.0 ** -8 + 2 * few + (V / 16 + 24) * 2.0 ** -23) + own * 2 * few) + 2.0 ** -8 * dx.abs() * (1 + 2.0 ** -7) + 1e-37
            out[-1] += [dx, tol]
    return [torch.cat(t) for t in zip(*out)]


def check(X, W, labels, weights=None, scale=1.0, **kw):
    want = reference(X, W, labels, torch.ones(len(X), device="cuda") if weights is None else weights, scale, True)
    V, K = W.shape
    ws = torch.full((lw.lowra_cross_entropy_workspace_bytes(len(X), V, K, True),), 255, dtype=torch.uint8, device="cuda")     # (NaNs wherever nothing was written)
    loss, dX = lw.lowra_cross_entropy(X, W, labels, scale=scale, weights=weights, want_grad=True, workspace=ws, **kw)
    assert lw.lowra_device_status(ws) == 0
    small = torch.full((lw.lowra_cross_entropy_workspace_bytes(len(X), V, K, False),), 255, dtype=torch.uint8, device="cuda")
    only, none = lw.lowra_cross_entropy(X, W, labels, workspace=small, **kw)
    assert none is None and lw.lowra_device_status(small) == 0
    for got in (loss, only):
        assert ((got.double() - want[0]).abs() <= want[1]).all(), ((got.double() - want[0]).abs() / want[1]).max()
    assert ((dX.double() - want[2]).abs() <= want[3]).all(), ((dX.double() - want[2]).abs() / want[3]).max()
    skip = labels == IGNORE
    assert (loss[skip] == 0).all() and (only[skip] == 0).all() and (dX[skip] == 0).all()
    return loss, dX, want


@pytest.mark.parametrize("M, V, K", [(1, 1, 64), (1, 2, 64), (2, 31, 64), (3, 129, 72), (16, 32000, 512), (130, 257, 4096), (257, 1000, 264), (777, 5003, 1024), (256, 256, 256),
                                     (1000, 300, 5120), (64, 100003, 128), (33, 777, 1096), (17, 5000, 4096), (65, 5000, 512)])
@pytest.mark.parametrize("known", [0.0, 14.0])
def test_loss_and_gradient(M, V, K, known):
    X, W, labels, weights = make(M, V, K, known=known, ignored=0.0 if M == 1 else 0.2)
    check(X, W, labels, weights, scale=0.125)


def test_all_tokens_ignored_and_label_edges():
    X, W, labels, _ = make(40, 515, 128)
    labels[:] = IGNORE
    loss, dX = lw.lowra_cross_entropy(X, W, labels, want_grad=True)
    assert (loss == 0).all() and (dX == 0).all()
    labels[::2], labels[1::2] = 0, 514
    check(X, W, labels)
    labels[3] = 7
    loss, dX = lw.lowra_cross_entropy(X, W, labels, want_grad=True, ignore_index=7)
    assert loss[3] == 0 and (dX[3] == 0).all() and (loss[:3] > 0).all()


def test_labels_that_are_no_words():
    X, W, labels, _ = make(300, 700, 128, ignored=0.0)
    good, good_dX = lw.lowra_cross_entropy(X, W, labels, want_grad=True)
    bad = labels.clone()
    bad[5], bad[6], bad[299], bad[290] = 700, -1, 2 ** 40, -2 ** 62
    loss, dX = lw.lowra_cross_entropy(X, W, bad, want_grad=True)
    only, _ = lw.lowra_cross_entropy(X, W, bad)
    hit = bad != labels
    for got in (loss, only):
        assert got[hit].isnan().all() and not got[~hit].isnan().any()
    assert dX[hit].isnan().all() and torch.equal(dX[~hit], good_dX[~hit]) and torch.equal(loss[~hit], good[~hit])


def test_pieces_of_the_vocabulary_and_passes():
    """Sizes that take several pieces (exponentials of 2048 x 40000: 164 MB) and several passes over the tokens, odd ends of both."""
    for M, V, K in ((2048, 40001, 256), (4099, 20011, 64)):
        X, W, labels, weights = make(M, V, K, known=8.0)
        check(X, W, labels, weights, scale=1 / M)


@pytest.mark.parametrize("V", [5000, 40000])
def test_logits_far_apart(V):
    """Logits hundreds above the label's, in some pieces and for some tokens only: exponentials that would be infinite under the label's own logit."""
    M, K = 2048, 128
    X, W, labels, weights = make(M, V, K, ignored=0.05)
    X[:, 0], W[:, 0] = 0, 0
    X[::3, 0] = 16.0
    X[1::3, 0] = -16.0
    W[V // 2 + 5, 0], W[V - 3, 0], W[7, 0], W[V // 3, 0] = 8.0, 20.0, -9.0, -30.0
    labels[::5] = V - 3
    loss, _, want = check(X, W, labels, weights)
    assert (want[0] > 300).any() and (want[0] < 1e-30).any()


def test_sure_tokens_keep_their_digits():
    """p of the label 1 - 1e-7 and nearer to 1: loss and gradient are still right to the roundings of the exponentials, not to those of p."""
    X, W, labels, _ = make(300, 2000, 512, known=26.0, ignored=0.0)
    loss, dX, want = check(X, W, labels)
    assert (want[0] < 1e-6).sum() > 100
    rel = (dX.double() - want[2]).norm(dim=1) / want[2].norm(dim=1)
    assert rel.max() < 2.0 ** -7


def test_bad_values_stay_with_their_token():
    X, W, labels, _ = make(300, 3000, 256, ignored=0.0)
    good, good_dX = lw.lowra_cross_entropy(X, W, labels, want_grad=True)
    bad = X.clone()
    bad[17, 3], bad[256, 9] = float("nan"), float("inf")
    loss, dX = lw.lowra_cross_entropy(bad, W, labels, want_grad=True)
    only, _ = lw.lowra_cross_entropy(bad, W, labels)
    hit = torch.zeros(300, dtype=torch.bool, device="cuda")
    hit[[17, 256]] = True
    assert loss[hit].isnan().all() and only[hit].isnan().all() and dX[hit].isnan().any(1).all()
    assert torch.equal(loss[~hit], good[~hit]) and torch.equal(dX[~hit], good_dX[~hit])
    skip = labels.clone()
    skip[hit] = IGNORE
    loss, dX = lw.lowra_cross_entropy(bad, W, skip, want_grad=True)
    assert (loss[hit] == 0).all() and (dX[hit] == 0).all() and torch.equal(loss[~hit], good[~hit])


def test_gradient_against_differences():
    """Along a direction, the sum of the losses in fp64 changes as dX says."""
    X, W, labels, weights = make(50, 700, 128, known=6.0)
    _, dX = lw.lowra_cross_entropy(X, W, labels, scale=0.5, weights=weights, want_grad=True)
    d = torch.randn(X.shape, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda", dtype=torch.float64)

    def f(x):
        lp = torch.log_softmax(x @ W.double().t(), 1)
        picked = lp.gather(1, labels.clamp_min(0)[:, None])[:, 0]
        return -(picked * weights.double() * 0.5 * (labels != IGNORE)).sum()

    h = 1e-5
    slope = (f(X.double() + h * d) - f(X.double() - h * d)) / (2 * h)
    want = reference(X, W, labels, weights, 0.5, True)
    assert (slope - (dX.double() * d).sum()).abs() <= (want[3] * d.abs()).sum() + 1e-6


def test_repeats_streams_and_graphs():
    X, W, labels, weights = make(600, 4001, 512, known=5.0)
    loss, dX = lw.lowra_cross_entropy(X, W, labels, weights=weights, want_grad=True)
    ws = torch.empty(lw.lowra_cross_entropy_workspace_bytes(600, 4001, 512, True), dtype=torch.uint8, device="cuda")
    out = dict(loss=torch.empty(600, device="cuda"), dX=torch.empty_like(X), workspace=ws)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    lw.lowra_cross_entropy(X, W, labels, weights=weights, stream=side, **out)
    torch.cuda.synchronize()
    assert torch.equal(out["loss"], loss) and torch.equal(out["dX"], dX)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lw.lowra_cross_entropy(X, W, labels, weights=weights, **out)
    for _ in range(3):
        out["loss"].fill_(9)
        out["dX"].fill_(9)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out["loss"], loss) and torch.equal(out["dX"], dX) and lw.lowra_device_status(ws) == 0


def test_refusals():
    X, W, labels, weights = make(16, 100, 64)
    ws = torch.empty(lw.lowra_cross_entropy_workspace_bytes(16, 100, 64, True), dtype=torch.uint8, device="cuda")
    for bad in (dict(X=X.float()), dict(X=X[0]), dict(W=W[:, :32]), dict(W=W.cpu()), dict(X=X.t()), dict(labels=labels.int()), dict(labels=labels[:15]), dict(weights=weights.double()),
                dict(loss=weights[:3]), dict(dX=X[:2]), dict(dX=X.float())):
        with pytest.raises(ValueError):
            lw.lowra_cross_entropy(**{**dict(X=X, W=W, labels=labels), **bad})
    for bad in (dict(workspace=ws[:-256]), dict(workspace=ws[16:]), dict(dX=X), dict(loss=weights, weights=weights), dict(X=X[:0], labels=labels[:0]),
                dict(X=X[:, :32].contiguous(), W=W[:, :32].contiguous())):
        with pytest.raises(lw.LowraError):
            lw.lowra_cross_entropy(**{**dict(X=X, W=W, labels=labels, want_grad=True), **bad})


def test_waits_that_may_run_out():
    """With a limit of a microsecond a wait may run out: the call then says so by its status word, and the next one, with the usual limit, is right."""
    X, W, labels, weights = make(300, 20000, 2048)
    good, good_dX = lw.lowra_cross_entropy(X, W, labels, want_grad=True)
    ws = torch.empty(lw.lowra_cross_entropy_workspace_bytes(300, 20000, 2048, True), dtype=torch.uint8, device="cuda")
    lw.lowra_set_wait_limit(1000)
    try:
        loss, dX = lw.lowra_cross_entropy(X, W, labels, want_grad=True, workspace=ws)
        status = lw.lowra_device_status(ws)
    finally:
        lw.lowra_set_wait_limit(0)
    assert status in (lw.LOWRA_OK, lw.LOWRA_ERR_TIMEOUT)
    if status == lw.LOWRA_OK:
        assert torch.equal(loss, good) and torch.equal(dX, good_dX)
    loss, dX = lw.lowra_cross_entropy(X, W, labels, want_grad=True, workspace=ws)
    assert lw.lowra_device_status(ws) == lw.LOWRA_OK and torch.equal(loss, good) and torch.equal(dX, good_dX)


@pytest.mark.parametrize("M, V", [(5, 900), (300, 900), (3, 1), (257, 1)])
def test_labels_whose_logit_is_no_number(M, V):
    """The label's own logit NaN or +infinity: NaN, although the label's word is left out of the sums; -infinity: the loss is infinite, or NaN where there is no other word."""
    for value, beside in ((float("inf"), True), (float("nan"), True), (float("-inf"), V == 1)):
        X, W, labels, _ = make(M, V, 128, ignored=0.0)
        X[:, 3] = 1.0
        labels[:] = V // 2
        W[V // 2, 3] = value
        loss, dX = lw.lowra_cross_entropy(X, W, labels, want_grad=True)
        only, _ = lw.lowra_cross_entropy(X, W, labels)
        for got in (loss, only):
            assert got.isnan().all() if beside else (got == float("inf")).all()
        assert dX.isnan().any(1).all()


@pytest.mark.parametrize("M", [2, 9, 40, 65, 100, 121, 127, 128, 129, 136, 255])
def test_tiles_of_few_tokens(M):
    """A tile's rows without a token are not loaded: after a call whose numbers are all NaN, what it left in their places changes nothing.  Widths of tiles from 128 to 256, a short last one."""
    for V, K in ((1000, 200), (9473, 72), (18945, 136)):
        X, W, labels, weights = make(M, V, K)
        big = torch.full((512, K), float("nan"), dtype=torch.bfloat16, device="cuda")
        lw.lowra_cross_entropy(big, W, torch.zeros(512, dtype=torch.int64, device="cuda"), want_grad=True)
        check(X, W, labels, weights)
