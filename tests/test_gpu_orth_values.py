"""Newton-Schulz updates on the GPU, held to what distinguishes a right result from a wrong one: every case's tolerance
is asserted to be at most a twentieth of the update's own size.

What a finite precision loses depends on the spectrum (noise in directions next to zero grows by a a step), so it is
measured: the same steps in fp32, one at a time and, where the long side is at least twice the short one, in rounds on m x m
matrices as well.  A matrix in 22 bits is rounded by four times as much as one in fp32 and the sums alike: four times that loss,
and 2^-20 of the update where fp32 happens to lose less (an orthonormal X has rms entries of one size: 2^-22 of each
operand).  A smaller side of at most 64 is in fp64: 2^-14 at most (below).  Then the output's rounding, half a step, and
2 u of what decay keeps.
"""
import numpy as np
import pytest
import torch

import oracle.model_oracle as M
import paper_2411_12364_amd as U

from .test_gpu_block_step import replayed
from .test_gpu_orth import BF, COEF, F, desc, gen, host, plain, run

pytestmark = pytest.mark.gpu
u = 2.0 ** -24
F32 = [float(np.float32(v)) for v in COEF]
EPS = float(np.float32(1e-7))


def few_directions(kind, rows, cols, g):
    """Matrices whose small singular values are next to none, as fp32 leaves them."""
    small = min(rows, cols)
    if kind == "rank 1":
        x = torch.randn((rows, 1), generator=g, device="cuda") * torch.randn((1, cols), generator=g, device="cuda")
    elif kind == "rank 1, exact":                                       # products of small whole numbers
        x = (torch.randint(1, 9, (rows, 1), generator=g, device="cuda") * torch.randint(1, 9, (1, cols), generator=g, device="cuda")).float()
    elif kind == "rank 2":
        x = torch.randn((rows, 2), generator=g, device="cuda") @ torch.randn((2, cols), generator=g, device="cuda")
    else:                                                               # every row (or column) twice
        x = torch.randn((rows, cols), generator=g, device="cuda")
        half = (small + 1) // 2
        if rows <= cols:
            x[small - half:] = x[:half].clone()
        else:
            x[:, small - half:] = x[:, :half].clone()
    return x


# A smaller side of at most 64 goes by powers of A in fp64.  What A loses, 2^-53 times the sums' 64 terms, is
# multiplied by at most |a|^3 a step while X is not formed again: of a pass of r steps with |a|^(3 r) <= 2^33 the slope of P
# (|b| + 2 |c| = 8.9) makes that 8.9 * 64 * 2^-53 * 2^33 / |a|^3 = 2^-16.2 of the small directions' size, three times
# (three passes of up to 6 steps make 16), and across directions 2^-53 * 64 * |a|^16 (2^28.6) = 2^-18.  So 2^-12 of |X|,
# with the outputs' own rounding added.
@pytest.mark.parametrize("kind", ["rank 1", "rank 1, exact", "rank 2", "twice"])
@pytest.mark.parametrize("rows,cols", [(64, 448), (500, 20), (33, 3000), (2, 9)])
@pytest.mark.parametrize("steps", [5, 9, 10, 12, 14, 16])
def test_many_steps_of_few_directions(steps, rows, cols, kind):
    print(f"[case] orth {rows} {cols} {steps} {kind}", flush=True)
    x = torch.stack([few_directions(kind, rows, cols, gen(rows + 7 * cols + j)) for j in range(2)])
    held = torch.randn((2, rows, cols), generator=gen(1), device="cuda")
    for gt, ot, decay, scale in ((F, F, 0.0, 1.0), (BF, F, 0.5, -0.25), (F, BF, 0.0, 2.0)):
        g, out = x.to(gt), held.to(ot)
        before = out.clone()
        run(desc(2, rows, cols, gt, ot, steps, decay=decay, scale=scale), g, out)
        for j in range(2):
            want, _ = M.newton_schulz(host(g[j]), steps, *F32, EPS)
            size = abs(scale) * np.linalg.norm(want)
            ref = decay * host(before[j]) + scale * want
            tol = 2.0 ** -12 * size + ((2.0 ** -8 if ot == BF else 0) + 2 * u) * np.linalg.norm(ref)
            assert tol < 0.05 * size
            assert np.linalg.norm(host(out[j]) - ref) <= tol, (np.linalg.norm(host(out[j]) - ref) / size, tol / size)


def test_many_steps_in_place():
    """The passes between the first X and the last leave G as it is, and an out that is G gets what another would."""
    for rows, cols in ((64, 448), (900, 40)):
        x = few_directions("rank 2", rows, cols, gen(rows)).reshape(1, rows, cols)
        od = desc(1, rows, cols, F, F, 16)
        kept = x.clone()
        want = run(od, x, torch.empty_like(x))
        assert torch.equal(x, kept)
        assert torch.equal(run(od, x, x), want)


# Both ways of taking the steps beside the small sides' one: single steps, and rounds of them on long matrices.
LARGE = [(96, 160), (160, 96), (70, 3000), (3000, 70)]


@pytest.mark.parametrize("gt", [F, BF])
@pytest.mark.parametrize("rows,cols", LARGE + [(64, 96)])
def test_any_scale_of_the_gradient(rows, cols, gt):
    """A power of two times G gives the same bits, where the norm is past the largest fp32 and where values have few bits left."""
    print(f"[case] orth {rows} {cols} {gt}", flush=True)
    x = torch.randn((1, rows, cols), generator=gen(rows), device="cuda").clamp(-3.9, 3.9).to(gt)
    od = desc(1, rows, cols, gt, F, eps=0.0)
    want = run(od, x, torch.empty((1, rows, cols), device="cuda"))
    assert bool(want.isfinite().all()) and float(want.norm()) > 1
    for e in (100, 126, -100, -120 if gt == BF else -126):
        big = torch.ldexp(x.double().cpu(), torch.tensor(e)).to(gt)
        back = torch.ldexp(big.double(), torch.tensor(-e)).to(gt)       # what is left of x
        if e > 0:
            assert torch.equal(back, x.cpu()) and bool(big.isfinite().all())
            assert e < 126 or float(big.double().norm()) > 3.5e38
        ref = run(od, back.cuda(), torch.empty((1, rows, cols), device="cuda"))
        assert torch.equal(run(od, big.cuda(), torch.empty((1, rows, cols), device="cuda")), ref), e
    od = desc(1, rows, cols, gt, F, eps=1e38)                            # an eps of the norm's size
    big = torch.ldexp(x.double().cpu(), torch.tensor(126)).to(gt)
    got = run(od, big.cuda(), torch.empty((1, rows, cols), device="cuda"))
    want, _ = M.newton_schulz(host(big[0]), 5, *F32, float(np.float32(1e38)))
    assert np.linalg.norm(host(got[0]) - want) <= 1e-4 * np.linalg.norm(want)


# Of X in fp32 the product with scale is one rounding (u, or half the smallest subnormal); the small sides' X is rounded
# after the product instead, so X itself differs by a rounding: 2 u and 2^-149 in all.  With decay one sum more.
@pytest.mark.parametrize("rows,cols", LARGE + [(64, 96)])
def test_any_scale_of_the_update(rows, cols):
    """Factors near the smallest and the largest fp32 multiply X as others do."""
    print(f"[case] orth {rows} {cols}", flush=True)
    x = torch.randn((1, rows, cols), generator=gen(rows + 1), device="cuda")
    held = torch.randn((1, rows, cols), generator=gen(rows + 2), device="cuda")
    want = host(run(desc(1, rows, cols, F, F), x, torch.empty_like(x)))
    for f in (1.3 * 2.0 ** -116, -1.7 * 2.0 ** -122, 1.1 * 2.0 ** -40, 1.9 * 2.0 ** 126):
        f = float(np.float32(f))
        got = host(run(desc(1, rows, cols, F, F, scale=f), x, torch.empty_like(x)))
        assert (np.abs(got - f * want) <= 2 * u * np.abs(f * want) + 2.0 ** -149).all(), f
        small = held * min(abs(f), 1.0)
        got = host(run(desc(1, rows, cols, F, F, decay=0.5, scale=f), x, small.clone()))
        ref, size = 0.5 * host(small) + f * want, 0.5 * np.abs(host(small)) + np.abs(f * want)
        assert (np.abs(got - ref) <= 3 * u * size + 2.0 ** -148).all(), f


def by_rounds(g, steps, coef, eps=1e-7):
    """The steps in fp32, up to three at a time on m x m matrices."""
    a, b, c = (np.float32(v) for v in coef)
    most = 3
    while most > 1 and abs(float(a)) ** most > 100:
        most -= 1
    x = g.astype(np.float32)
    x = x / np.float32(np.sqrt((x.astype(np.float64) ** 2).sum()) + eps)
    tall = x.shape[0] > x.shape[1]
    x = np.ascontiguousarray(x.T) if tall else x
    one = np.eye(len(x), dtype=np.float32)
    rounds = -(-steps // most)
    for j in range(rounds):
        gram = x @ x.T
        for i in range(steps // rounds + (j < steps % rounds)):
            p = a * one + (b * gram + c * (gram @ gram))
            q = p if i == 0 else q @ p
            gram = p @ (p @ gram)
        x = q @ x
    return (x.T if tall else x).astype(np.float64)


def exact(g, steps, coef):
    """The update in float64, and how far the kernel's X may be from it."""
    want, _ = M.newton_schulz(g, steps, *[float(np.float32(v)) for v in coef], EPS)
    size, (m, k) = np.linalg.norm(want), sorted(g.shape)
    lost = np.linalg.norm(plain(g, steps, coef) - want)
    if k >= 2 * m:
        lost = max(lost, np.linalg.norm(by_rounds(g, steps, coef) - want))
    lost = min(lost, 2.0 ** -14 * size) if m <= 64 else lost
    return want, 4 * lost + 2.0 ** -20 * size


def batch(kind, n, rows, cols, g):
    if kind in ("broad", "steep"):
        x = torch.randn((n, rows, cols), generator=g, device="cuda") * 1e-3
        return x * torch.logspace(0, -3, cols, device="cuda") if kind == "steep" else x
    return torch.stack([few_directions(kind, rows, cols, g) for _ in range(n)])


def check(n, rows, cols, gt=F, ot=F, steps=5, coef=COEF, decay=0.0, scale=1.0, lead=0, kind="broad", some=None):
    g = gen(rows + 3 * cols + n)
    room = torch.empty(lead + n * rows * cols, dtype=gt, device="cuda")
    x = room[lead:].view(n, rows, cols)
    x.copy_(batch(kind, n, rows, cols, g))
    held = (torch.randn((n, rows, cols), generator=g, device="cuda") * abs(scale) / max(rows, cols) ** 0.5).to(ot)
    room = torch.full((lead + x.numel() + 8,), 5.0, dtype=ot, device="cuda")
    out = room[lead:lead + x.numel()].view(n, rows, cols)
    out.copy_(held if decay else torch.full_like(held, float("nan")))
    kept = x.clone()
    run(desc(n, rows, cols, gt, ot, steps, coef, decay=decay, scale=scale), x, out)
    assert torch.equal(x, kept)
    assert (room[:lead] == 5.0).all() and (room[lead + x.numel():] == 5.0).all()
    decay, scale = float(np.float32(decay)), float(np.float32(scale))
    for j in some or range(n):
        want, tol = exact(host(x[j]), steps, coef)
        ref = (decay * host(held[j]) if decay else 0.0) + scale * want
        tol = abs(scale) * tol + (2.0 ** -8 if ot == BF else 2 * u) * np.linalg.norm(ref)
        tol += 2 * u * (abs(decay) * np.linalg.norm(host(held[j])) + np.linalg.norm(scale * want))
        off, size = np.linalg.norm(host(out[j]) - ref), abs(scale) * np.linalg.norm(want)
        assert tol < 0.05 * size, ("a tolerance that would pass a wrong result", j, tol / size)
        assert off <= tol, (j, off / size, tol / size)


KINDS = ["broad", "steep", "rank 1", "rank 1, exact", "rank 2", "twice"]


@pytest.mark.parametrize("gt,ot", [(F, F), (BF, F), (F, BF), (BF, BF)])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,rows,cols", [(2, 96, 160), (3, 160, 96), (2, 128, 128), (2, 80, 4000), (2, 6000, 72), (1, 333, 700),
                                         (4, 450, 230), (2, 65, 65), (3, 100, 31), (2, 64, 448), (2, 3, 200)])
def test_values(n, rows, cols, kind, gt, ot):
    print(f"[case] orth {n} {rows} {cols} {kind} {gt} {ot}", flush=True)
    check(n, rows, cols, gt, ot, kind=kind)


@pytest.mark.parametrize("rows,cols", [(96, 160), (160, 96), (128, 128), (80, 4000), (6000, 72), (64, 200), (90, 49), (17, 30)])
@pytest.mark.parametrize("kw", [dict(steps=1), dict(steps=2), dict(steps=3), dict(steps=4), dict(steps=6), dict(steps=7),
                                dict(steps=12, coef=(1.5, -0.5, 0.0)), dict(steps=16, coef=(1.5, -0.5, 0.0)),
                                dict(coef=(2.0, -1.5, 0.5)), dict(coef=(6.0, -13.0, 8.0), steps=2),
                                dict(coef=(11.0, -20.0, 10.0), steps=2), dict(decay=0.9, scale=-0.02),
                                dict(decay=-1.0, scale=3.0), dict(decay=0.9, scale=-0.02, ot=BF), dict(lead=1),
                                dict(lead=3, gt=BF, ot=BF), dict(lead=2, decay=0.5, ot=BF), dict(kind="steep", steps=3),
                                dict(kind="rank 1", steps=3), dict(kind="rank 2", decay=0.5, scale=0.3)])
def test_factors(rows, cols, kw):
    print(f"[case] orth {rows} {cols} {kw}", flush=True)
    check(2, rows, cols, **kw)


# Sizes that between them reach every tile, group and split of each of the products; of large batches some matrices.
@pytest.mark.parametrize("n,rows,cols,steps,ot", [(1, 71, 2146, 2, F), (100, 163, 70, 3, F), (100, 69, 81, 2, F), (100, 71, 136, 2, F),
                                                  (30, 326, 326, 1, BF), (1, 71, 143, 2, BF), (2, 4426, 70, 1, BF),
                                                  (2, 69, 4252, 2, BF), (30, 547, 70, 2, BF), (100, 69, 2156, 1, F),
                                                  (30, 321, 790, 2, F), (40, 132, 6457, 1, F), (30, 70, 547, 5, F),
                                                  (100, 163, 70, 6, BF), (60, 66, 300, 5, F), (2, 300, 2000, 5, F), (1, 700, 800, 2, BF),
                                                  (4, 450, 230, 3, F), (1, 1030, 1300, 5, F), (40, 64, 128, 5, BF), (500, 40, 33, 5, F)])
def test_every_tile(n, rows, cols, steps, ot):
    print(f"[case] orth {n} {rows} {cols} {steps} {ot}", flush=True)
    check(n, rows, cols, ot=ot, steps=steps, some=sorted({0, 1 % n, n // 2, n - 1}))


@pytest.mark.parametrize("n,rows,cols", [(300, 65, 65536), (300, 65536, 66), (300, 64, 65536)])
def test_values_past_4_gib(n, rows, cols):
    """The first and the last of matrices that lie past 4 GiB; all of them are theirs alone."""
    print(f"[case] orth {n} {rows} {cols}", flush=True)
    x = torch.empty((n, rows, cols), device="cuda").normal_(generator=gen(n))
    out = run(desc(n, rows, cols, F, F, 2), x, torch.empty_like(x))
    for j in (0, n - 1):
        want, tol = exact(host(x[j]), 2, COEF)
        tol += 4 * u * np.linalg.norm(want)
        assert tol < 0.05 * np.linalg.norm(want)
        assert np.linalg.norm(host(out[j]) - want) <= tol


@pytest.mark.parametrize("rows,cols", LARGE + [(128, 1100), (64, 90)])
@pytest.mark.parametrize("steps", [1, 5])
def test_matrices_of_a_batch_are_apart(rows, cols, steps):
    """Zeros give zeros, a NaN or an infinity stays with its matrix, and the others are what they are beside ordinary ones."""
    print(f"[case] orth {rows} {cols} {steps}", flush=True)
    x = torch.randn((4, rows, cols), generator=gen(rows), device="cuda")
    want = run(desc(4, rows, cols, F, F, steps), x, torch.empty_like(x))
    for bad in (float("nan"), float("inf"), -float("inf")):
        y = x.clone()
        y[1] = 0.0
        y[2, rows // 2, cols - 1] = bad
        got = run(desc(4, rows, cols, F, F, steps), y, torch.empty_like(x))
        assert (got[1] == 0).all() and bool(got[2].isnan().any()) and (bad == bad or bool(got[2].isnan().all()))
        assert torch.equal(got[0], want[0]) and torch.equal(got[3], want[3])
    y = torch.zeros_like(x)                                             # 0 / 0 without an eps
    y[0], y[3] = x[0], x[3]
    alone = run(desc(4, rows, cols, F, F, steps, eps=0.0), y, torch.empty_like(x))
    assert bool(alone[1:3].isnan().all()) and bool(alone[0].isfinite().all()) and bool(alone[3].isfinite().all())


@pytest.mark.parametrize("rows,cols,steps", [(96, 160, 5), (70, 3000, 5), (40, 500, 12)])
def test_captured(rows, cols, steps):
    """Captured and replayed on other matrices, out updated in place."""
    print(f"[case] orth captured {rows} {cols} {steps}", flush=True)
    g = torch.randn((2, rows, cols), generator=gen(rows), device="cuda")
    held = torch.randn((2, rows, cols), generator=gen(cols), device="cuda")
    out, od = torch.empty_like(held), desc(2, rows, cols, F, F, steps, decay=0.9, scale=-0.1)
    ws = torch.empty(U.umem_orthogonalize_workspace_size(od)[1], dtype=torch.uint8, device="cuda")

    def step():
        out.copy_(held)
        U.check(U.umem_orthogonalize(od, g, out, ws, ws.numel()))

    def change(k):
        g.copy_(g.roll(17 * (k + 1), 2) * (0.5 + k))
        held.mul_(0.75)

    step()
    replayed(step, [out], change)
