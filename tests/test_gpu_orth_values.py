"""Newton-Schulz updates on the GPU, held to what distinguishes a right result from a wrong one: every case's tolerance
is well below the size of what it compares.
"""
import numpy as np
import pytest
import torch

import oracle.model_oracle as M

from .test_gpu_orth import BF, COEF, F, desc, gen, host, run

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
