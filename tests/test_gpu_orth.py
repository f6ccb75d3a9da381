"""Newton-Schulz updates on the GPU against float64.

A product loses eps of its size: parts of 22 bits (2^-22 of either operand), a pair of parts left out (2^-22) and fp32
sums over k (2 u (3 k / 32 + 16)), sizes taken as norms.  With singular values of at most 1.22 past the first step,
A's are at most 1.5, and P = a I + b A + c A^2's at most p = a where a is the largest value that it takes.

One step at a time: an error in X grows by at most a (the step's slope at a singular value of 0; less elsewhere), and
the step adds (a + 2 |b| + 4 |c|) eps |X|_F.
r steps on m x m matrices: A is off by eps 1.5 at first; P by (|b| + 3 |c|) times that and eps (a + 1.5 |b| + 2.25 |c|) of its
own; Q by what P and it were off, times the other, and eps of it; the next A = P A P by a^2 what A was off, 3 a what P was,
and 2 eps 1.5 a^2.  X then grows its error by a^r and gains (Q's error + eps |Q|) |X|_F.
Both are bounds for the worst case, the second a wide one (they let bf16's operands fail by their 2^13, no more); what
happens on random matrices is held to eight times what the same steps lose in fp32 as well.
"""
import numpy as np
import pytest
import torch

import oracle.model_oracle as M
import paper_2411_12364_amd as U

pytestmark = pytest.mark.gpu
u = 2.0 ** -24
COEF = (3.4445, -4.7750, 2.0315)
BF, F = torch.bfloat16, torch.float32


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def host(x):
    return x.detach().double().cpu().numpy()


def desc(n, rows, cols, gt, ot, steps=5, coef=COEF, eps=1e-7, decay=0.0, scale=1.0):
    return U.umem_orth_desc(n, rows, cols, int(gt == BF), int(ot == BF), steps, *coef, eps, decay, scale)


def run(od, g, out):
    st, need = U.umem_orthogonalize_workspace_size(od)
    U.check(st)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")         # NaN in every type
    U.check(U.umem_orthogonalize(od, g, out, ws, ws.numel()))
    return out


def tolerance(norms, k, steps, coef):
    a, b, c = (abs(v) for v in coef)
    a = max(a, 1.0)
    eps = 3 * 2.0 ** -22 + 2 * u * (3 * k / 32 + 16)
    one = sum(a ** (steps - 1 - j) * (a + 2 * b + 4 * c) * eps * norms[j] for j in range(steps))
    rounds = -(-steps // 3)
    many, at = 0.0, 0
    for j in range(rounds):
        r = steps // rounds + (j < steps % rounds)
        da, dq, q = 1.5 * eps, 0.0, 1.0
        for i in range(r):
            dp = (b + 3 * c) * da + eps * (a + 1.5 * b + 2.25 * c)
            dq = dp if i == 0 else a * dq + q * dp + eps * a * q
            q *= a
            da = a * a * da + 3 * a * dp + 3 * eps * a * a
        many = a ** r * many + (dq + eps * q) * norms[at]
        at += r
    return max(one, many)


def plain(g, steps, coef, eps=1e-7):
    """The same steps in fp32."""
    x = g.astype(np.float32)
    x = x / np.float32(np.sqrt((x.astype(np.float64) ** 2).sum()) + eps)
    tall = x.shape[0] > x.shape[1]
    x = x.T if tall else x
    a, b, c = (np.float32(v) for v in coef)
    for _ in range(steps):
        gram = x @ x.T
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    return (x.T if tall else x).astype(np.float64)


def check(n, rows, cols, gt=F, ot=F, steps=5, coef=COEF, decay=0.0, scale=1.0, lead=0, kind="broad", seed=0):
    g = gen(seed + rows + 3 * cols)
    x = torch.randn((n, rows, cols), generator=g, device="cuda") * 1e-3
    if kind == "steep":                                                 # singular values over three orders of magnitude
        x = x * torch.logspace(0, -3, cols, device="cuda")
    elif kind == "low":                                                 # rank 1
        x = x[:, :, :1] * x[:, :1, :] * 1e6
    room = torch.empty(lead + x.numel(), dtype=gt, device="cuda")
    room[lead:] = x.reshape(-1).to(gt)
    x = room[lead:].view(n, rows, cols)
    held = (torch.randn((n, rows, cols), generator=g, device="cuda") * 0.1).to(ot)
    room = torch.full((lead + x.numel() + 8,), 5.0, dtype=ot, device="cuda")
    out = room[lead:lead + x.numel()].view(n, rows, cols)
    out.copy_(held if decay else torch.full_like(held, float("nan")))   # without a decay out is not read
    run(desc(n, rows, cols, gt, ot, steps, coef, decay=decay, scale=scale), x, out)
    assert (room[lead + x.numel():] == 5.0).all()
    f32 = [float(np.float32(v)) for v in coef]
    for j in range(n):
        want, norms = M.newton_schulz(host(x[j]), steps, *f32, float(np.float32(1e-7)))
        ref = np.float32(decay) * host(held[j]) + np.float32(scale) * want if decay else np.float32(scale) * want
        got = host(out[j])
        tol = abs(scale) * tolerance(norms, max(rows, cols), steps, coef) + 8 * u * np.linalg.norm(ref)
        tol += (2.0 ** -8 if ot == BF else 0.0) * np.linalg.norm(ref)
        if kind == "broad" and ot == F and not decay and n == 1:
            lost = np.linalg.norm(plain(host(x[j]), steps, coef) - want)
            tol = min(tol, abs(scale) * (8 * lost + 2.0 ** -20 * np.linalg.norm(want)))
        assert np.linalg.norm(got - ref) <= tol, (j, np.linalg.norm(got - ref), tol)


# (the first ones are long enough to go by rounds of steps)
SHAPES = [(1, 70, 3000), (2, 4100, 96), (1, 130, 2500), (1, 200, 8000), (1, 1, 1), (1, 1, 9), (1, 7, 1), (3, 2, 3), (1, 8, 8), (2, 63, 65), (1, 64, 64), (1, 65, 64), (2, 100, 31),
          (1, 127, 129), (1, 130, 260), (3, 33, 500), (1, 500, 33), (1, 256, 256), (1, 200, 1030), (5, 72, 40)]


@pytest.mark.parametrize("gt,ot", [(F, F), (BF, F), (F, BF), (BF, BF)])
@pytest.mark.parametrize("n,rows,cols", SHAPES)
def test_update(n, rows, cols, gt, ot):
    print(f"[case] orth {n} {rows} {cols} {gt} {ot}", flush=True)
    check(n, rows, cols, gt, ot)


@pytest.mark.parametrize("rows,cols", [(96, 160), (160, 96), (128, 128), (80, 4000), (6000, 72), (64, 200), (90, 49), (48, 500), (17, 30),
                                       (333, 16)])
@pytest.mark.parametrize("kw", [dict(steps=3), dict(steps=4), dict(steps=6), dict(steps=7), dict(steps=16, coef=(1.5, -0.5, 0.0)),
                                dict(coef=(6.0, -13.0, 8.0), steps=2), dict(coef=(11.0, -20.0, 10.0), steps=2), dict(steps=1), dict(steps=2), dict(steps=8), dict(coef=(1.5, -0.5, 0.0), steps=12),
                                dict(coef=(2.0, -1.5, 0.5)), dict(decay=0.9, scale=-0.02), dict(decay=-1.0, scale=3.0),
                                dict(decay=0.9, scale=-0.02, ot=BF), dict(lead=1), dict(lead=3, gt=BF, ot=BF),
                                dict(kind="steep"), dict(kind="low"), dict(scale=0.0)])
def test_steps_and_factors(rows, cols, kw):
    print(f"[case] orth {rows} {cols} {kw}", flush=True)
    check(2, rows, cols, **kw)


@pytest.mark.parametrize("n,rows,cols", [(1, 1024, 1300), (1, 1500, 700), (40, 64, 128), (1, 40, 20000), (20000, 2, 3)])
def test_many_and_large(n, rows, cols):
    print(f"[case] orth {n} {rows} {cols}", flush=True)
    if n < 100:
        check(n, rows, cols)
        return
    x = torch.randn((n, rows, cols), generator=gen(1), device="cuda")
    out = run(desc(n, rows, cols, F, F), x, torch.empty_like(x))
    for j in (0, 1, n // 2, n - 1):
        alone = run(desc(1, rows, cols, F, F), x[j:j + 1].clone(), torch.empty((1, rows, cols), device="cuda"))
        assert torch.equal(out[j], alone[0])


# Sizes that between them reach every tile, group and split of each of the products.
@pytest.mark.parametrize("n,rows,cols,steps,ot", [(1, 70, 70, 2, F), (1, 71, 2146, 2, F), (100, 163, 70, 3, F), (100, 69, 81, 2, F),
                                                  (100, 71, 136, 2, F), (30, 326, 326, 1, BF), (1, 70, 71, 1, BF),
                                                  (1, 71, 143, 2, BF), (2, 4426, 70, 1, BF), (2, 69, 4252, 2, F),
                                                  (2, 69, 4252, 2, BF), (30, 547, 70, 2, BF), (100, 69, 2156, 1, F),
                                                  (30, 321, 790, 2, F), (40, 132, 6457, 1, F), (30, 70, 547, 5, F),
                                                  (100, 163, 70, 6, BF), (50, 70, 90, 2, F), (60, 66, 300, 5, F),
                                                  (2, 300, 2000, 5, F), (1, 700, 800, 2, BF), (4, 450, 230, 3, F)])
def test_tiles(n, rows, cols, steps, ot):
    print(f"[case] orth {n} {rows} {cols} {steps} {ot}", flush=True)
    check(n, rows, cols, ot=ot, steps=steps)


@pytest.mark.parametrize("n,rows,cols", [(300, 65, 65536), (300, 65536, 66), (300, 64, 65536)])
def test_past_4_gib(n, rows, cols):
    """Batches of 5 GB: the first and the last matrices."""
    print(f"[case] orth {n} {rows} {cols}", flush=True)
    x = torch.empty((n, rows, cols), device="cuda").normal_(generator=gen(n))
    out = run(desc(n, rows, cols, F, F, 2), x, torch.empty_like(x))
    f32 = [float(np.float32(v)) for v in COEF]
    for j in (0, n - 1):
        want, norms = M.newton_schulz(host(x[j]), 2, *f32, float(np.float32(1e-7)))
        tol = tolerance(norms, max(rows, cols), 2, COEF) + 8 * u * np.linalg.norm(want)
        assert np.linalg.norm(host(out[j]) - want) <= tol
    assert bool(out.isfinite().all())


def test_matrices_are_apart():
    """Zeros give zeros, a NaN or an infinity stays with its matrix, and each matrix is what it is alone."""
    x = torch.randn((4, 48, 80), generator=gen(2), device="cuda")
    x[1] = 0.0
    x[2, 5, 7] = float("nan")
    out = run(desc(4, 48, 80, F, F), x, torch.empty_like(x))
    assert (out[1] == 0).all() and bool(out[2].isnan().all())
    for j in (0, 3):
        assert torch.equal(out[j], run(desc(1, 48, 80, F, F), x[j].clone(), torch.empty_like(x[j])))
    x[2, 5, 7] = float("inf")
    out = run(desc(4, 48, 80, F, F), x, torch.empty_like(x))
    assert bool(out[2].isnan().any()) and bool(out[0].isfinite().all()) and bool(out[3].isfinite().all())


def test_any_scale_of_the_gradient():
    """The norm is fp64: gradients whose squares would overflow or vanish in 32 bits give the same update."""
    x = torch.randn((1, 64, 96), generator=gen(3), device="cuda")
    want = run(desc(1, 64, 96, F, F, eps=0.0), x, torch.empty_like(x))
    for f in (2.0 ** 100, 2.0 ** -100):
        got = run(desc(1, 64, 96, F, F, eps=0.0), x * f, torch.empty_like(x))
        assert float((got - want).abs().max()) <= 64 * u * 140 * float(want.abs().max())


def test_in_place_and_on_a_stream():
    x = torch.randn((2, 130, 70), generator=gen(4), device="cuda")
    want = run(desc(2, 130, 70, F, F), x, torch.empty_like(x))
    y = x.clone()
    assert torch.equal(run(desc(2, 130, 70, F, F), y, y), want)
    od = desc(2, 130, 70, F, F, decay=0.5)
    y, z = x.clone(), x.clone()
    assert torch.equal(run(od, y, y), run(od, x, z))                    # g is what out held
    side = torch.cuda.Stream()
    ws = torch.empty(U.umem_orthogonalize_workspace_size(od)[1], dtype=torch.uint8, device="cuda")
    out = torch.empty_like(x)
    torch.cuda.synchronize()
    U.check(U.umem_orthogonalize(desc(2, 130, 70, F, F), x, out, ws, ws.numel(), side))
    side.synchronize()
    assert torch.equal(out, want)


def test_rows_become_orthonormal():
    """Five steps take the singular values of a random matrix to between 0.6 and 1.3."""
    x = torch.randn((1, 200, 700), generator=gen(5), device="cuda")
    s = np.linalg.svd(host(run(desc(1, 200, 700, F, F), x, torch.empty_like(x))[0]), compute_uv=False)
    assert 0.6 < s.min() and s.max() < 1.3
