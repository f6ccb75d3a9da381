"""A model's ends in a run together, as a training step uses them: token rows, the norm before the head, the loss, its
gradients, the rows' gradient into the tied weight's, the global norm, clipping and an orthogonalised update of the
norm's matrix; captured and replayed on other inputs."""
import numpy as np
import pytest
import torch

import oracle.block_oracle as B
import oracle.model_oracle as M
import paper_2411_12364_amd as U

from .test_gpu_block_step import host, replayed

pytestmark = pytest.mark.gpu
u = 2.0 ** -24
EPS = 1e-5
COEF = (3.4445, -4.7750, 2.0315)


@pytest.mark.parametrize("T", [1, 50, 300])
def test_training_step(T):
    print(f"[case] model step, {T} tokens", flush=True)
    vocab, d = 700, 64
    g = torch.Generator(device="cuda").manual_seed(T)
    rand = lambda *s, std=1.0: torch.randn(s, generator=g, device="cuda") * std   # noqa: E731
    table = rand(vocab, d, std=0.2).to(torch.bfloat16)
    ids = torch.randint(-1, vocab, (T,), generator=g, device="cuda").to(torch.int32)
    ids[0] = 3
    targets = torch.roll(ids, -1)
    gamma, dloss, weight = 1 + 0.2 * rand(d), torch.full((T,), 1.0 / T, device="cuda"), rand(vocab, d, std=0.1)
    ed = U.umem_embed_desc(vocab, d, 1, 0, 8.0)
    hd = U.umem_head_desc(vocab, d, 0, 0, 0.5)
    bd = U.umem_block_desc(d, U.UMEM_NORM_RMS, U.UMEM_NORM_NONE, 0, 0, 0, 0, EPS, 1.0, 1.0)
    od = U.umem_orth_desc(1, vocab, d, 0, 0, 5, *COEF, 1e-7, 0.99, -0.1)
    t = {k: torch.zeros(s, device="cuda") for k, s in dict(
        h=(T, d), n=(T, d), loss=(T,), lse=(T,), dn=(T, d), dh=(T, d), dw=(vocab, d), dgamma=(d,), norm=(1,), dr=(T, d),
        step=(vocab, d)).items()}
    rows, n_rows = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    table_of = (U.umem_grad * 2)(*[U.umem_grad(t[k].data_ptr(), t[k].data_ptr(), None, 1, t[k].numel(), 0) for k in ("dw", "dgamma")])
    sizes = [U.umem_embed_backward_workspace_size(ed, T), U.umem_head_loss_workspace_size(hd, T),
             U.umem_head_backward_workspace_size(hd, T), U.umem_block_backward_workspace_size(bd, T),
             U.umem_orthogonalize_workspace_size(od), U.umem_grad_workspace_size(2, table_of)]
    for st, _ in sizes:
        U.check(st)
    ws = torch.empty(max(n for _, n in sizes), dtype=torch.uint8, device="cuda")
    limit = 1e9

    def step():
        w = (ws, ws.numel())
        U.check(U.umem_embed(ed, T, table, ids, t["h"]))
        U.check(U.umem_block_in(bd, T, t["h"], gamma, None, t["n"]))
        U.check(U.umem_head_loss(hd, T, t["n"], table, targets, t["loss"], t["lse"], *w))
        U.check(U.umem_head_backward(hd, T, t["n"], table, targets, t["lse"], dloss, t["dn"], t["dw"], 0, *w))
        U.check(U.umem_block_in_backward(bd, T, t["h"], gamma, t["dn"], None, t["dh"], t["dgamma"], None, 0, *w))
        U.check(U.umem_embed_backward_rows(ed, T, ids, t["dh"], rows, t["dr"], n_rows, *w))
        U.check(U.umem_embed_backward(ed, T, ids, t["dh"], t["dw"], *w))
        U.check(U.umem_grad_norm(2, table_of, t["norm"], None, *w))
        U.check(U.umem_grad_clip(2, table_of, limit, t["norm"]))
        t["step"].copy_(weight)
        U.check(U.umem_orthogonalize(od, t["dw"], t["step"], *w))

    step()
    torch.cuda.synchronize()
    W, I, Y, G, gm = host(table), ids.cpu().numpy(), targets.cpu().numpy(), host(dloss), host(gamma)

    def loss_of(w_in, w_out, gm):
        n = B.block_in(M.embed(w_in, I, 8.0), "rms", gm, None, EPS)
        return M.head_loss(n, w_out, Y, 0.5)[0], n

    want, n = loss_of(W, W, gm)
    assert np.abs(host(t["loss"]) - want).max() <= 256 * u * (1 + np.abs(want).max())
    # the tied weight's gradient along a random direction against central differences of the float64 loss
    rng = np.random.default_rng(2)
    for k, grad in (("dw", host(t["dw"])), ("dgamma", host(t["dgamma"]))):
        v, e = rng.normal(size=grad.shape), 1e-5
        f = [(loss_of(W + s * e * v, W + s * e * v, gm)[0] if k == "dw" else loss_of(W, W, gm + s * e * v)[0]) @ G for s in (1, -1)]
        diff = (f[0] - f[1]) / (2 * e)
        assert abs((grad * v).sum() - diff) <= 256 * u * np.abs(grad * v).sum() + 1e-6 * abs(diff) + 1e-8, k
    # the rows' gradient alone, compactly
    k = int(n_rows)
    used = np.unique(I[I >= 0])
    assert np.array_equal(rows[:k].cpu().numpy(), used)
    dense = M.embed_backward(I, host(t["dh"]), vocab, 8.0)
    assert (np.abs(host(t["dr"])[:k] - dense[0][used]) <= (T + 2) * u * dense[1][used]).all()
    whole = B.global_norm([host(t["dw"]), host(t["dgamma"])])
    assert abs(float(t["norm"]) - whole) <= 2 * u * whole
    x, norms = M.newton_schulz(host(t["dw"]), 5, *[float(np.float32(c)) for c in COEF], float(np.float32(1e-7)))
    ref = float(np.float32(0.99)) * host(weight) + float(np.float32(-0.1)) * x
    assert np.linalg.norm(host(t["step"]) - ref) <= 0.1 * 1e-4 * np.linalg.norm(x) + 8 * u * np.linalg.norm(ref)
    limit = 0.5 * whole
    kept = host(t["dw"])
    step()
    torch.cuda.synchronize()
    assert (np.abs(host(t["dw"]) - 0.5 * kept) <= 8 * u * np.abs(kept)).all()

    def change(k):
        ids.copy_((ids + 31 * (k + 1)) % vocab)
        targets.copy_(torch.roll(ids, -1))
        targets[k % T] = -1
        gamma.mul_(1.05)

    replayed(step, [t[k] for k in t] + [n_rows], change)


def test_two_graphs_share_a_workspace():
    """Two captured graphs with one workspace, replayed in turn: each gives what its calls give."""
    T, vocab, d = 140, 300, 64
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn((T, d), generator=g, device="cuda").to(torch.bfloat16)
    w = (torch.randn((vocab, d), generator=g, device="cuda") * 0.2).to(torch.bfloat16)
    y = torch.randint(0, vocab, (T,), generator=g, device="cuda").to(torch.int32)
    hd, od = U.umem_head_desc(vocab, d, 1, 0, 1.0), U.umem_orth_desc(1, vocab, d, 0, 0, 5, *COEF, 1e-7, 0.0, 1.0)
    loss, lse = torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda")
    dx, dw, out = torch.zeros_like(x), torch.zeros((vocab, d), device="cuda"), torch.zeros((vocab, d), device="cuda")
    ws = torch.empty(max(U.umem_head_backward_workspace_size(hd, T)[1], U.umem_head_loss_workspace_size(hd, T)[1],
                         U.umem_orthogonalize_workspace_size(od)[1]), dtype=torch.uint8, device="cuda")

    def first():
        U.check(U.umem_head_loss(hd, T, x, w, y, loss, lse, ws, ws.numel()))
        U.check(U.umem_head_backward(hd, T, x, w, y, lse, None, dx, dw, 0, ws, ws.numel()))

    def second():
        U.check(U.umem_orthogonalize(od, dw, out, ws, ws.numel()))

    first(), second()
    torch.cuda.synchronize()
    want = [v.clone() for v in (loss, lse, dx, dw, out)]
    graphs = []
    for f in (first, second):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            f()
    for _ in range(4):
        for v in (loss, lse, dx, dw, out):
            v.zero_()
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, (loss, lse, dx, dw, out)))
