"""The head's cross entropy and its gradients on the GPU against float64.

A logit is an fp32 sum of d products of bf16 values (exact in fp32; fp32 x as three parts that add up to it): every
addition rounds by u = 2^-24 of a partial sum of at most S = s sum |x w| (the matrix cores may cut off instead of
rounding: 2 u), and there are d / 32 additions of 32 products each after at most 5 inside: with three parts
z_err = 2 u (3 d / 32 + 8) S + 2 u |z|.
lse and loss move by at most the largest z_err and twice it, and lose a few u of the exponentials' sum (relative, so
absolute in the logarithm) and their own rounding.
r = exp(z - lse) - [target] moves by exp(..) (2 z_err + (|z - lse| + 8) u).  For dx it is half a step, 2^-8, off as one bf16
part, u as three.  For dw it is 2^-11 and, below 2^-29 of the largest dloss, 2^-40 of that off as one fp16 part; as two
2^-22 and 2^-40, as fp32 x is then, relative to the largest x, and the product of the second parts, 2^-22, is left out.
The sums over the vocabulary or the tokens add 2 u (terms / 32 + 16) per part of their absolute terms, and a
bf16 result half a step.
"""
import numpy as np
import pytest
import torch

import oracle.model_oracle as M
import paper_2411_12364_amd as U

pytestmark = pytest.mark.gpu
u = 2.0 ** -24
HALF = 2.0 ** -8                # half a step of bf16
BF, F = torch.bfloat16, torch.float32


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def host(x):
    return x.detach().double().cpu().numpy()


def make(T, vocab, d, xt, seed=0, none=0.15, scale=1.0):
    g = gen(seed + 7 * T + d)
    w = (torch.randn((vocab, d), generator=g, device="cuda") * 2.0 / (scale * d ** 0.5)).to(BF)
    y = torch.randint(0, vocab, (T,), generator=g, device="cuda")
    x = torch.randn((T, d), generator=g, device="cuda") + torch.rand((T, 1), generator=g, device="cuda") * w[y].float()
    out = torch.rand((T,), generator=g, device="cuda") < none
    bad = torch.tensor([-1, vocab, -2 ** 31, 2 ** 31 - 1], device="cuda")
    y = torch.where(out, bad[torch.arange(T, device="cuda") % 4], y).to(torch.int32)
    dloss = torch.rand((T,), generator=g, device="cuda") * 2.0 - 0.5
    return x.to(xt), w, y, dloss


def desc(vocab, d, xt, gt, scale):
    return U.umem_head_desc(vocab, d, int(xt == BF), int(gt == BF), scale)


def scratch(size, ds, T):
    st, need = size(ds, T)
    U.check(st)
    return torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")       # NaN in every type


def forward(ds, x, w, y):
    T = len(x)
    loss, lse = torch.full((T,), 9.0, device="cuda"), torch.full((T,), 9.0, device="cuda")
    ws = scratch(U.umem_head_loss_workspace_size, ds, T)
    U.check(U.umem_head_loss(ds, T, x, w, y, loss, lse, ws, ws.numel()))
    return loss, lse


def backward(ds, x, w, y, lse, dloss, gt, dw=None):
    T = len(x)
    dx = torch.full_like(x, 9.0)
    acc = dw is not None
    dw = torch.full(w.shape, 9.0, dtype=gt, device="cuda") if dw is None else dw
    ws = scratch(U.umem_head_backward_workspace_size, ds, T)
    U.check(U.umem_head_backward(ds, T, x, w, y, lse, dloss, dx, dw, int(acc), ws, ws.numel()))
    return dx, dw


def z_error(x, w, scale):
    """[T, vocab]: how far a logit may be off."""
    size = np.abs(scale) * (np.abs(x) @ np.abs(w).T)
    return 2 * u * (3 * x.shape[1] / 32 + 8) * size + 2 * u * np.abs(M.logits(x, w, scale))


def check(T, vocab, d, xt, gt, scale=1.0, none=0.15, seed=0, uniform=False):
    x, w, y, dloss = make(T, vocab, d, xt, seed, none, scale)
    dloss = torch.full_like(dloss, 1.0 / 3.0) if uniform else dloss
    ds = desc(vocab, d, xt, gt, scale)
    loss, lse = forward(ds, x, w, y)
    X, W, Y, G = host(x), host(w), y.cpu().numpy(), host(dloss)
    scale = float(np.float32(scale))
    want_loss, want_lse = M.head_loss(X, W, Y, scale)
    err = z_error(X, W, scale)
    top = err.max(axis=1)
    assert (np.abs(host(lse) - want_lse) <= top + 16 * u + 2 * u * np.abs(want_lse)).all()
    assert (np.abs(host(loss) - want_loss) <= 2 * top + 16 * u + 2 * u * np.abs(want_loss)).all()
    assert (host(loss)[~M.counts(Y, vocab)] == 0).all()
    check_backward(ds, x, w, y, lse, dloss, gt, scale, err)


def bounds(X, W, Y, G, scale, err, wide_x, wide_g):
    """(dx, dw) in float64 and how far they may be off before they are rounded."""
    on = M.counts(Y, len(W))
    lse = M.head_loss(X, W, Y, scale)[1]
    z = M.logits(X, W, scale)
    r = M.head_slope(X, W, Y, G, scale)
    p = np.where(on[:, None], np.exp(z - lse[:, None]), 0.0)
    size = np.abs(scale * G)[:, None]
    off = size * p * (2 * err + err.max(axis=1, keepdims=True) + (np.abs(z - lse[:, None]) + 8) * 2 * u) + 4 * u * np.abs(r)
    off[~on] = 0.0
    T, V = r.shape
    X = np.where(on[:, None], X, 0.0)
    ex, ew = np.abs(W), np.abs(X)
    tx = off @ ex + (np.abs(r) @ ex) * ((u if wide_x else HALF) + (3 if wide_x else 1) * 2 * u * (V / 32 + 16) + 8 * u)
    tw = off.T @ ew + (np.abs(r).T @ ew) * ((3 * 2.0 ** -22 if wide_g else 2.0 ** -11 + 2.0 ** -11) + 3 * 2 * u * (T / 32 + 16) + 8 * u)
    most = np.abs(G[on]).max() * abs(scale) if on.any() else 0.0
    tw += 2.0 ** -40 * (most * ew.sum(axis=0)[None, :] + ew.max() * np.abs(r).sum(axis=0)[:, None])
    return r @ W, r.T @ X, tx, tw


def check_backward(ds, x, w, y, lse, dloss, gt, scale, err):
    X, W, Y, G = host(x), host(w), y.cpu().numpy(), host(dloss)
    wide_x, wide_g = x.dtype == F, gt == F
    dx, dw = backward(ds, x, w, y, lse, dloss, gt)
    want_x, want_w, tx, tw = bounds(X, W, Y, G, scale, err, wide_x, wide_g)
    tx += (0 if wide_x else HALF) * (np.abs(want_x) + tx) + 2.0 ** -130
    tw += (0 if wide_g else HALF) * (np.abs(want_w) + tw) + 2.0 ** -130
    assert (np.abs(host(dx) - want_x) <= tx).all()
    assert (np.abs(host(dw) - want_w) <= tw).all()
    assert (host(dx)[~M.counts(Y, len(W))] == 0).all()
    dx2, dw2 = backward(ds, x, w, y, lse, dloss, gt)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
    if gt == F:
        held = torch.randn(w.shape, generator=gen(1), device="cuda")
        _, both = backward(ds, x, w, y, lse, dloss, gt, held.clone())
        assert (np.abs(host(both) - (host(held) + host(dw))) <= 4 * u * (np.abs(host(held)) + np.abs(host(dw)))).all()


SIZES = [(1, 1, 8), (1, 2, 16), (2, 7, 8), (3, 63, 24), (16, 64, 64), (17, 65, 72), (63, 129, 56), (64, 255, 128),
         (65, 257, 136), (128, 300, 64), (129, 128, 64), (129, 129, 64), (130, 1000, 72), (255, 513, 96), (300, 256, 64),
         (513, 777, 200), (40, 5000, 64)]


@pytest.mark.parametrize("gt", [F, BF])
@pytest.mark.parametrize("xt", [F, BF])
@pytest.mark.parametrize("T,vocab,d", SIZES)
def test_loss_and_gradients(T, vocab, d, xt, gt):
    print(f"[case] head {T} {vocab} {d} {xt} {gt}", flush=True)
    check(T, vocab, d, xt, gt)


@pytest.mark.parametrize("xt,gt", [(F, F), (BF, F), (BF, BF)])
@pytest.mark.parametrize("kw", [dict(scale=0.25), dict(scale=-3.0), dict(none=0.0), dict(none=1.0), dict(uniform=True),
                                dict(none=0.9, scale=8.0), dict(scale=0.0001), dict(scale=-0.0001)])
def test_scales_and_masks(kw, xt, gt):
    print(f"[case] head {kw} {xt} {gt}", flush=True)
    check(150, 400, 128, xt, gt, **kw)


@pytest.mark.parametrize("T,vocab,d,xt,gt", [(130, 40001, 16, BF, F), (20, 33000, 32, F, BF), (2100, 300, 1024, BF, F),
                                             (140, 140, 2048, F, F), (300, 20000, 64, BF, BF)])
def test_pieces_and_long_sums(T, vocab, d, xt, gt):
    """A vocabulary of several pieces, many tokens, wide states."""
    print(f"[case] head {T} {vocab} {d} {xt} {gt}", flush=True)
    check(T, vocab, d, xt, gt)


# Sizes that between them reach every tile, group and split of the four products, in each type.
TILES = [(148, 11497, 72), (3, 10974, 144), (452, 8507, 72), (3, 13437, 200), (6331, 327, 72), (3, 6922, 584), (5634, 656, 72)]
TILES_OF_X = [(4186, 6, 200), (6636, 5, 272), (7168, 4, 392), (6148, 4, 656), (4617, 4, 1688), (4604, 279, 72)]


@pytest.mark.parametrize("T,vocab,d,xt,gt", [(*t, BF, BF) for t in TILES] + [(*t, BF, F) for t in TILES] +
                         [(*t, F, BF) for t in TILES_OF_X] + [(*t, BF, BF) for t in TILES_OF_X] +
                         [(3, 8297, 80, BF, F), (4, 16296, 896, BF, F), (4, 12778, 1736, BF, BF), (3, 5054, 1560, F, BF),
                          (4604, 279, 72, BF, F), (4604, 279, 72, F, F), (6331, 327, 72, F, F), (5634, 656, 72, F, F),
                          (2198, 5574, 16, BF, BF), (6268, 5, 1864, F, F), (3139, 5, 1768, F, F),
                          (4266, 1693, 264, F, F), (929, 8196, 72, F, F), (3000, 700, 264, BF, BF), (263, 17135, 816, BF, F),
                          (2908, 1052, 88, F, BF), (2052, 5024, 72, F, BF), (6209, 1290, 152, F, BF)])
def test_tiles(T, vocab, d, xt, gt):
    print(f"[case] head {T} {vocab} {d} {xt} {gt}", flush=True)
    check(T, vocab, d, xt, gt)


def test_pieces_of_many_tokens():
    """More tokens than the scratch holds 16,384 rows of: pieces of fewer rows; the forward in two bands."""
    T, vocab, d = 40000, 5000, 8
    x, w, y, dloss = make(T, vocab, d, BF)
    ds = desc(vocab, d, BF, F, 1.0)
    loss, lse = forward(ds, x, w, y)
    z = x.double() @ w.double().t()
    want = torch.logsumexp(z, 1)
    on = (y >= 0) & (y < vocab)
    goal = z.gather(1, y.clamp(0, vocab - 1).long()[:, None])[:, 0]
    err = 2 * u * (d / 32 + 16) * float((x.double().abs() @ w.double().abs().t()).max()) + 64 * u
    assert float((lse - want).abs().max()) <= err
    assert float((loss - torch.where(on, want - goal, 0.0)).abs().max()) <= 2 * err
    dx, dw = backward(ds, x, w, y, lse, dloss, F)
    r = torch.exp(z - want[:, None])
    r.scatter_add_(1, y.clamp(0, vocab - 1).long()[:, None], torch.full((T, 1), -1.0, dtype=torch.float64, device="cuda"))
    r *= torch.where(on, dloss.double(), 0.0)[:, None]
    size = r.abs()
    tol = (size @ w.double().abs()) * (HALF + 4 * err) + HALF * (r @ w.double()).abs()
    assert bool(((dx.double() - r @ w.double()).abs() <= tol + 1e-30).all())
    tol = (size.t().contiguous() @ x.double().abs()) * (4 * err + 6 * 2 * u * (T / 32 + 16))
    assert bool(((dw.double() - r.t().contiguous() @ x.double()).abs() <= tol).all())


@pytest.mark.parametrize("T", [1023, 1024, 1025, 300001])
@pytest.mark.parametrize("xt", [F, BF])
def test_few_of_many_tokens_count(T, xt):
    """A few tokens among many that do not count: their gradients are the formula's, the others' rows of dx zero."""
    vocab, d = 40, 16
    x, w, y, dloss = make(T, vocab, d, xt, none=0.0)
    on = torch.zeros(T, dtype=torch.bool, device="cuda")
    on[torch.randperm(T, generator=gen(T), device="cuda")[:60]] = True
    on[T - 1] = True
    y[~on] = -1
    ds = desc(vocab, d, xt, F, 1.0)
    _, lse = forward(ds, x, w, y)
    dx, dw = backward(ds, x, w, y, lse, dloss, F)
    assert not dx[~on].any()
    few = [t[on].contiguous() for t in (x, y, lse, dloss)]
    X, W, Y, G = host(few[0]), host(w), few[1].cpu().numpy(), host(few[3])
    want_x, want_w, tx, tw = bounds(X, W, Y, G, 1.0, z_error(X, W, 1.0), xt == F, True)
    tx += (0 if xt == F else HALF) * (np.abs(want_x) + tx) + 2.0 ** -130
    assert (np.abs(host(dx[on]) - want_x) <= tx).all() and (np.abs(host(dw) - want_w) <= tw + 2.0 ** -130).all()


@pytest.mark.parametrize("xt,gt", [(F, F), (BF, BF), (F, BF)])
@pytest.mark.parametrize("T,vocab,d", [(40, 90, 64), (700, 300, 96)])
def test_powers_of_two(T, vocab, d, xt, gt):
    """Hidden states times 2^100, the weight times 2^-100: the same losses, and gradients that differ by those powers alone;
    states up to the largest, with gradients of the losses so small that the weight's gradient is within fp32."""
    x, w, y, dloss = make(T, vocab, d, xt, none=0.1)
    ds = desc(vocab, d, xt, gt, 0.5)
    loss, lse = forward(ds, x, w, y)
    dx, dw = backward(ds, x, w, y, lse, dloss, gt)
    big, small = x * 2.0 ** 100, w * 2.0 ** -100
    loss2, lse2 = forward(ds, big, small, y)
    assert torch.equal(loss, loss2) and torch.equal(lse, lse2)
    dx2, dw2 = backward(ds, big, small, y, lse, dloss * 2.0 ** 20, gt)
    assert torch.equal(dx2.double(), dx.double() * 2.0 ** -80) and torch.equal(dw2 * 2.0 ** -60, dw * 2.0 ** 60)
    big, small = x.clamp(-7.9, 7.9) * 2.0 ** 125, w * 2.0 ** -115
    w = small * 2.0 ** 115                # (entries of w below 2^-11 lose bits in `small`, which is below 2^-126 there)
    ds, near = desc(vocab, d, xt, gt, 2.0 ** -10), desc(vocab, d, xt, gt, 1.0)
    _, lse = forward(near, x.clamp(-7.9, 7.9), w, y)
    assert torch.equal(forward(ds, big, small, y)[1], lse)
    _, dw = backward(near, x.clamp(-7.9, 7.9), w, y, lse, dloss, gt)
    _, dw2 = backward(ds, big, small, y, lse, dloss * 2.0 ** -100, gt)
    assert torch.equal(dw2 * 2.0 ** -15, dw)


@pytest.mark.parametrize("T,vocab", [(20, 1 << 20), (1 << 20, 70)])
def test_past_4_gib(T, vocab):
    """A weight, and hidden states, of 4.8 GB: the largest vocabulary and the most tokens that the calls take."""
    d = 2304
    print(f"[case] head {T} {vocab} {d}", flush=True)
    g = gen(3)
    fill = lambda n, std: torch.empty((n, d), dtype=BF, device="cuda").normal_(std=std, generator=g)   # noqa: E731
    x, w = fill(T, 1.0), fill(vocab, 2.0 / d ** 0.5)
    y = torch.randint(0, vocab, (T,), generator=g, device="cuda").to(torch.int32)
    y[T - 1], y[0] = vocab - 1, -1
    dloss = torch.rand((T,), generator=g, device="cuda") + 0.5
    ds = desc(vocab, d, BF, F, 1.0)
    loss, lse = forward(ds, x, w, y)
    step = 1 << 14
    z = torch.empty((T, vocab), dtype=torch.float32, device="cuda")      # logits rounded to 32 bits: 2^-24 of their 16
    for t in range(0, T, step):
        for v in range(0, vocab, step):
            z[t:t + step, v:v + step] = x[t:t + step].double() @ w[v:v + step].double().t().contiguous()
    # sums over d of products of about 4 2^-5.6 with fp32 roundings, their rest in the sizes
    err = 2 * u * (d / 32 + 16) * 60 + 64 * u
    want = torch.cat([torch.logsumexp(c.double(), 1) for c in z.split(step)]) if T > step else torch.logsumexp(z.double(), 1)
    goal = z.gather(1, y.clamp(min=0).long()[:, None])[:, 0].double()
    assert float((lse - want).abs().max()) <= err
    assert float((loss - torch.where(y >= 0, want - goal, 0.0)).abs().max()) <= 2 * err
    dx, dw = backward(ds, x, w, y, lse, dloss, F)
    on = (y >= 0).double() * dloss.double()
    rows = torch.tensor([0, 1, 9, T // 2, T - 2, T - 1], device="cuda")
    cols = torch.tensor([0, 1, vocab // 2, vocab - 2, vocab - 1], device="cuda")

    def slope(t, v):
        r = torch.exp(z[t][:, v].double() - want[t][:, None]) - (y[t][:, None] == v[None]).double()
        return r * on[t][:, None]
    every_v, every_t = torch.arange(vocab, device="cuda"), torch.arange(T, device="cuda")
    got, size = torch.zeros((len(rows), d), dtype=torch.float64, device="cuda"), 0.0
    for v in every_v.split(step):
        r = slope(rows, v)
        got += r @ w[v].double()
        size = size + r.abs() @ w[v].double().abs()
    assert bool(((dx[rows].double() - got).abs() <= HALF * got.abs() + (HALF + 4 * err) * size + 1e-12).all())
    got, size = torch.zeros((len(cols), d), dtype=torch.float64, device="cuda"), 0.0
    for t in every_t.split(step):
        r = slope(t, cols).t().contiguous()
        got += r @ x[t].double()
        size = size + r.abs() @ x[t].double().abs()
    lost = 2.0 ** -40 * 1.5 * 8.0 * T                                   # what lies below 2^-40 of the largest r, of each token
    assert bool(((dw[cols].double() - got).abs() <= (4 * err + 6 * 2 * u * (min(T, 1 << 16) / 32 + 16)) * size + lost).all())


def test_no_dloss_is_ones():
    x, w, y, _ = make(70, 200, 64, BF)
    ds = desc(200, 64, BF, F, 1.0)
    _, lse = forward(ds, x, w, y)
    a, b = backward(ds, x, w, y, lse, None, F), backward(ds, x, w, y, lse, torch.ones(70, device="cuda"), F)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("T", [60, 200])
@pytest.mark.parametrize("xt,gt", [(F, F), (BF, BF), (BF, F)])
def test_what_does_not_count_reaches_nothing(T, xt, gt):
    """NaN and infinities in the hidden states and dloss of tokens without a target: the others' losses and
    gradients are those without them; a NaN token's loss is NaN and the other tokens' losses are untouched."""
    vocab, d = 300, 64
    x, w, y, dloss = make(T, vocab, d, xt, none=0.3)
    off = ~((y >= 0) & (y < vocab))
    ds = desc(vocab, d, xt, gt, 1.0)
    loss, lse = forward(ds, x, w, y)
    dx, dw = backward(ds, x, w, y, lse, dloss, gt)
    bad = x.clone()
    bad[off] = float("nan")
    bad[off.nonzero()[0, 0]] = float("inf")
    dbad = dloss.clone()
    dbad[off] = float("nan")
    loss2, lse2 = forward(ds, bad, w, y)
    assert torch.equal(loss, loss2) and torch.equal(lse[~off], lse2[~off])
    dx2, dw2 = backward(ds, bad, w, y, lse2, dbad, gt)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)
    k = int((~off).nonzero()[5, 0])
    bad = x.clone()
    bad[k, 3] = float("nan")
    loss2, lse2 = forward(ds, bad, w, y)
    assert bool(loss2[k].isnan()) and bool(lse2[k].isnan())
    keep = torch.arange(T, device="cuda") != k
    assert torch.equal(loss[keep], loss2[keep])
    dx2, dw2 = backward(ds, bad, w, y, lse2, dloss, gt)
    assert bool(dx2[k].isnan().all()) and torch.equal(dx[keep], dx2[keep]) and bool(dw2.isnan().any())


def test_infinite_logits():
    """Logits of -infinity have no share; a logit of +infinity makes lse infinite."""
    T, vocab, d = 40, 200, 16
    x, w, y, dloss = make(T, vocab, d, BF, none=0.0)
    x[:, 0], w[:, 0] = 1.0, 0.0
    w[150:, 0] = -float("inf")
    y.clamp_(max=149)
    ds = desc(vocab, d, BF, F, 1.0)
    loss, lse = forward(ds, x, w, y)
    few = desc(150, d, BF, F, 1.0)
    loss2, lse2 = forward(few, x, w[:150].contiguous(), y)
    assert float((loss - loss2).abs().max()) <= 64 * u and float((lse - lse2).abs().max()) <= 64 * u * float(lse.abs().max())
    w[150:, 0] = float("inf")
    loss, lse = forward(ds, x, w, y)
    assert bool((lse == float("inf")).all()) and bool((loss == float("inf")).all())


@pytest.mark.parametrize("xt,gt", [(F, F), (BF, BF)])
def test_no_scale(xt, gt):
    """A factor of 0: every logit is 0, and every gradient."""
    T, vocab, d = 70, 300, 64
    x, w, y, dloss = make(T, vocab, d, xt)
    ds = desc(vocab, d, xt, gt, 0.0)
    loss, lse = forward(ds, x, w, y)
    assert float((lse - np.log(300.0)).abs().max()) <= 16 * u
    assert torch.equal(loss, torch.where((y >= 0) & (y < vocab), lse, 0.0))
    dx, dw = backward(ds, x, w, y, lse, dloss, gt)
    assert not dx.any() and not dw.any()


@pytest.mark.parametrize("scale", [3.0e38, -3.0e38])
def test_largest_scale(scale):
    """A factor near the largest fp32: logits of tiny states are finite."""
    T, vocab, d = 9, 150, 8
    g = gen(5)
    x = torch.randn((T, d), generator=g, device="cuda") * 2.0 ** -120
    w = (torch.randn((vocab, d), generator=g, device="cuda") * 2.0 ** -8).to(BF)
    y = torch.arange(T, device="cuda").to(torch.int32)
    loss, lse = forward(desc(vocab, d, F, F, scale), x, w, y)
    X, W = host(x), host(w)
    scale = float(np.float32(scale))
    want, want_lse = M.head_loss(X, W, y.cpu().numpy(), scale)
    # x's bf16 parts below 2^-133 are lost: |x| is off by 2^-134 in each
    err = abs(scale) * 2.0 ** -134 * np.abs(W).sum(axis=1).max() + z_error(X, W, scale).max()
    assert (np.abs(host(lse) - want_lse) <= err + 16 * u + 2 * u * np.abs(want_lse)).all()
    assert (np.abs(host(loss) - want) <= 2 * err + 16 * u + 2 * u * np.abs(want)).all()


def test_large_logits():
    """Logits of thousands, where exp of one would not be finite: the loss of the largest is 0, of others large."""
    T, vocab, d = 33, 100, 8
    x = torch.zeros((T, d), dtype=BF, device="cuda")
    w = torch.zeros((vocab, d), dtype=BF, device="cuda")
    x[:, 0], w[:, 0] = 64.0, torch.arange(vocab, device="cuda").to(BF)
    y = torch.arange(T, device="cuda").to(torch.int32) * 3
    y[0] = 99
    ds = desc(vocab, d, BF, F, 1.0)
    loss, lse = forward(ds, x, w, y)
    assert bool((lse == 6336.0).all()) and torch.equal(loss, (99 - y).float() * 64)
    dx, dw = backward(ds, x, w, y, lse, None, F)
    assert torch.equal(dx[1:, 0].float(), 99.0 - w[y[1:].long(), 0].float())
    # the largest logit's token: sum_v p_v v - 99 = -1 e^-64 + ..., of which the products with w hold 98 e^-64 - 0
    # (r of the target is exp(0) - 1 = 0): 1.57e-26, r and dx each rounded to bf16
    assert abs(float(dx[0, 0]) - 98 * np.exp(-64.0)) <= (2 * HALF + 80 * u) * 98 * np.exp(-64.0)


@pytest.mark.parametrize("scale", (1.0, -1.0))
@pytest.mark.parametrize("T, vocab", ((5, 70), (5, 130), (300, 300), (3000, 5000), (520, 200)))
def test_logits_far_below_zero(T, vocab, scale):
    """All logits about -300, so that a reference of 0 anywhere (of a wave without rows of W) would lose them; some rows'
    are -infinity, a whole tile's among them."""
    d = 8
    rng = np.random.default_rng(vocab)
    x = torch.zeros((T, d), dtype=BF, device="cuda")
    w = torch.zeros((vocab, d), dtype=BF, device="cuda")
    x[:, 0] = 16.0 * scale
    x[:, 1] = torch.tensor(rng.integers(0, 2, size=T), device="cuda").to(BF)
    w[:, 0] = torch.tensor(-19.0 + rng.integers(0, 8, size=vocab) / 8, device="cuda").to(BF)
    w[:, 1] = scale
    w[vocab // 2:vocab - 1, 0] = -float("inf")
    y = torch.tensor(rng.integers(0, vocab // 2, size=T), device="cuda", dtype=torch.int32)
    loss, lse = forward(desc(vocab, d, BF, F, scale), x, w, y)
    z = np.outer(host(x)[:, 0], host(w)[:, 0]) * scale + host(x)[:, 1:2]
    top = z.max(axis=1)
    exact = top + np.log(np.exp(z - top[:, None]).sum(axis=1))
    goal = z[np.arange(T), y.cpu().numpy()]
    # products and z are exact; exp2's argument and value, sums of 256 and a rounding of either output
    slack = 300 * u + u * np.abs(exact)
    assert (np.abs(host(lse) - exact) <= slack).all()
    assert (np.abs(host(loss) - (exact - goal)) <= 300 * u + u * np.abs(exact - goal)).all()


def test_gradients_against_differences():
    """The gradients along random directions against central differences of the float64 loss."""
    T, vocab, d = 90, 150, 64
    x, w, y, dloss = make(T, vocab, d, F)
    ds = desc(vocab, d, F, F, 0.5)
    _, lse = forward(ds, x, w, y)
    dx, dw = backward(ds, x, w, y, lse, dloss, F)
    X, W, Y, G = host(x), host(w), y.cpu().numpy(), host(dloss)
    f = lambda X, W: (M.head_loss(X, W, Y, 0.5)[0] * G).sum()   # noqa: E731
    rng = np.random.default_rng(0)
    for at, grad in ((0, host(dx)), (1, host(dw))):
        v, h = rng.normal(size=grad.shape), 1e-5
        a, b = ((X + h * v, W), (X - h * v, W)) if at == 0 else ((X, W + h * v), (X, W - h * v))
        diff = (f(*a) - f(*b)) / (2 * h)
        assert abs((grad * v).sum() - diff) <= 256 * u * np.abs(grad * v).sum() + 1e-7 * abs(diff) + 1e-8


def test_workspace_of_more_tokens_and_a_stream():
    vocab, d = 500, 64
    ds = desc(vocab, d, BF, F, 1.0)
    ws = torch.empty(max(U.umem_head_loss_workspace_size(ds, 1000)[1], U.umem_head_backward_workspace_size(ds, 1000)[1]),
                     dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    for T in (1, 128, 129, 1000):
        x, w, y, dloss = make(T, vocab, d, BF)
        loss, lse = forward(ds, x, w, y)
        want = backward(ds, x, w, y, lse, dloss, F)
        torch.cuda.synchronize()
        loss2, lse2, dx, dw = torch.empty_like(loss), torch.empty_like(lse), torch.empty_like(x), torch.empty_like(want[1])
        torch.cuda.synchronize()
        U.check(U.umem_head_loss(ds, T, x, w, y, loss2, lse2, ws, ws.numel(), side))
        U.check(U.umem_head_backward(ds, T, x, w, y, lse2, dloss, dx, dw, 0, ws, ws.numel(), side))
        side.synchronize()
        assert torch.equal(loss, loss2) and torch.equal(lse, lse2) and torch.equal(dx, want[0]) and torch.equal(dw, want[1])
