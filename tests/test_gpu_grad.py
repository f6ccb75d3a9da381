"""The global gradient norm and clipping on the GPU against float64.

The squares and their sum are fp64: the norm is the rounding of sqrt, u = 2^-24 of it (and 1e-12 of fp64 sums).  A
clipped element goes through the norm's rounding, a division and a product: 3 u, and half a step of
bf16 where it is stored so.
"""
import numpy as np
import pytest
import torch

import oracle.block_oracle as B
import paper_2411_12364_amd as U

pytestmark = pytest.mark.gpu
u = 2.0 ** -24


def table(grads, outs, n_rows=None):
    """n_rows: {tensor: int32 tensor}"""
    rows = []
    for i, (g, o) in enumerate(zip(grads, outs)):
        many = g.shape[0] if g.dim() > 1 else 1
        n = (n_rows or {}).get(i)
        rows.append(U.umem_grad(g.data_ptr(), o.data_ptr(), None if n is None else n.data_ptr(), many,
                                g.numel() // many if many else 0, int(g.dtype == torch.bfloat16)))
    return (U.umem_grad * len(rows))(*rows)


def norm_of(tab, n=None, sumsq=None):
    n = len(tab) if n is None else n
    st, need = U.umem_grad_workspace_size(n, tab)
    U.check(st)
    ws = torch.full((max(need, 256),), 0xA5, dtype=torch.uint8, device="cuda")
    norm = torch.full((1,), -1.0, device="cuda")
    U.check(U.umem_grad_norm(n, tab, norm, sumsq, ws, ws.numel()))
    return norm


def make(shapes, seed, bf16=(), lead=0):
    """Tensors `lead` elements into their storage; those of `bf16` in that type."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for i, s in enumerate(shapes):
        n = int(np.prod(s))
        x = torch.randn(lead + n, generator=g, device="cuda") * 10.0 ** -(i % 4)
        out.append(x.to(torch.bfloat16 if i in bf16 else torch.float32)[lead:].view(s))
    return out


def check(grads, outs, max_norm, norm, n_rows=None):
    full = [g.detach().double().cpu().numpy() for g in grads]
    kept = {i: min(max(int(n), 0), full[i].shape[0]) for i, n in (n_rows or {}).items()}
    used = [g[:kept.get(i, len(g))] for i, g in enumerate(full)]
    want = B.global_norm(used)
    assert abs(float(norm) - want) <= want * (u + 1e-12)
    c = B.clip_factor(want, float(np.float32(max_norm)))
    for i, (g, o) in enumerate(zip(used, outs)):
        o = o.detach().double().cpu().numpy()
        tol = np.abs(g * c) * (3 * u + (2.0 ** -8 if outs[i].dtype == torch.bfloat16 else 0.0)) + 2.0 ** -149
        assert (np.abs(o[:len(g)] - g * c) <= tol).all(), i
        assert (o[len(g):] == 9.0).all(), i                            # rows behind the last one


SHAPES = [
    [(1,)], [(3,)], [(8192,)], [(8193,)], [(5, 7)], [(1,), (2,), (3,), (5,), (1023,), (4096,)],
    [(100, 333), (8191,), (17,), (64, 1024)], [(200, 4097), (1,)],
]


@pytest.mark.parametrize("shapes", SHAPES, ids=[str(i) for i in range(len(SHAPES))])
@pytest.mark.parametrize("lead,out_lead", [(0, 0), (1, 1), (3, 0), (0, 2)])
@pytest.mark.parametrize("factor", [0.25, 4.0])
def test_norm_and_clip(shapes, lead, out_lead, factor):
    print(f"[case] clip {shapes} {lead} {out_lead}", flush=True)
    bf16 = set(range(1, len(shapes), 2)) | ({0} if lead == 3 else set())
    grads = make(shapes, 7 + lead, bf16, lead)
    outs = [torch.full((out_lead + g.numel(),), 9.0, dtype=g.dtype, device="cuda")[out_lead:].view(g.shape) for g in grads]
    tab = table(grads, outs)
    norm = norm_of(tab)
    limit = factor * float(norm)
    U.check(U.umem_grad_clip(len(tab), tab, limit, norm))
    check(grads, outs, limit, norm)
    copies = [g.clone() for g in grads]                                 # in place: the same bits
    tab = table(copies, copies)
    U.check(U.umem_grad_clip(len(tab), tab, limit, norm))
    assert all(torch.equal(a, b) for a, b in zip(copies, outs))


@pytest.mark.parametrize("rows", [-5, 0, 1, 77, 299, 300, 1000, 2 ** 31 - 1])
@pytest.mark.parametrize("width,bf16", [(512, False), (129, True), (7, False)])
def test_rows_counted_on_the_gpu(rows, width, bf16):
    print(f"[case] rows {rows} {width}", flush=True)
    grads = make([(300, width), (40,)], 3, {0} if bf16 else ())
    used = min(max(rows, 0), 300)
    grads[0][used:] = float("nan")                                      # nothing behind the last row is read
    outs = [torch.full_like(g, 9.0) for g in grads]
    n = torch.tensor([rows], dtype=torch.int32, device="cuda")
    tab = table(grads, outs, {0: n})
    norm = norm_of(tab)
    U.check(U.umem_grad_clip(2, tab, 0.5, norm))
    check(grads, outs, 0.5, norm, {0: n})
    kept = grads[0].clone()
    tab = table(grads, grads, {0: n})
    U.check(U.umem_grad_clip(2, tab, 0.5, norm))
    assert torch.equal(grads[0][used:].isnan(), kept[used:].isnan())


def test_more_tensors_than_one_launch_takes():
    shapes = [((i * 37) % 900 + 1,) if i % 5 else (0,) for i in range(331)]
    grads = make(shapes, 11, set(range(0, 331, 3)))
    outs = [torch.full_like(g, 9.0) for g in grads]
    tab = table(grads, outs)
    sumsq = torch.zeros(1, dtype=torch.float64, device="cuda")
    norm = norm_of(tab, sumsq=sumsq)
    U.check(U.umem_grad_clip(len(tab), tab, 0.01, norm))
    check(grads, outs, 0.01, norm)
    assert abs(float(sumsq) - B.global_norm([g.double().cpu().numpy() for g in grads]) ** 2) <= 1e-11 * float(sumsq)


def test_many_counted_on_the_gpu():
    """More tensors with their rows on the GPU than one launch takes, others between them."""
    shapes = [((i * 7) % 40 + 1, 33) if i % 3 == 0 else (100 + i,) for i in range(61)]
    grads = make(shapes, 13, {4, 9, 30})
    outs = [torch.full_like(g, 9.0) for g in grads]
    n_rows = {i: torch.tensor([(i * 5) % 50], dtype=torch.int32, device="cuda") for i in range(0, 61, 3)}
    tab = table(grads, outs, n_rows)
    norm = norm_of(tab)
    U.check(U.umem_grad_clip(len(tab), tab, 0.02, norm))
    check(grads, outs, 0.02, norm, n_rows)


def test_nothing_to_sum():
    norm = norm_of((U.umem_grad * 1)(), 0)
    assert float(norm) == 0.0
    empty = table([torch.empty((0, 5), device="cuda")], [torch.empty((0, 5), device="cuda")])
    assert float(norm_of(empty)) == 0.0
    x = torch.zeros(100, device="cuda")
    assert float(norm_of(table([x], [x]))) == 0.0
    U.check(U.umem_grad_clip(1, table([x], [x]), 0.0, torch.zeros(1, device="cuda")))
    assert (x == 0).all()


def test_values_beyond_the_squares_of_floats():
    """Squares of 1e30 are no floats, those of 1e-30 vanish in them."""
    for v in (1e30, 1e-30, 2.0 ** -149):
        x = torch.full((1000,), v, device="cuda")
        want = np.sqrt(1000.0) * float(np.float32(v))
        got = float(norm_of(table([x], [x])))
        assert abs(got - want) <= u * want + 2.0 ** -150
    x = torch.full((1 << 20,), 3e38, device="cuda")                     # the norm itself is past fp32
    assert float(norm_of(table([x], [x]))) == float("inf")


def test_norms_that_are_not_finite():
    x = torch.arange(-3.0, 4.0, device="cuda")
    bad = torch.tensor([1.0, float("inf"), float("-inf"), float("nan")], device="cuda")
    for value, want in ((float("inf"), torch.zeros(7)), (float("nan"), torch.full((7,), float("nan")))):
        out = torch.full_like(x, 9.0)
        norm = torch.tensor([value], device="cuda")
        U.check(U.umem_grad_clip(1, table([x], [out]), 1.0, norm))
        torch.testing.assert_close(out.cpu(), want, equal_nan=True, rtol=0, atol=0)
    assert np.isnan(float(norm_of(table([bad], [bad])))) and float(norm_of(table([bad[:3]], [bad[:3]]))) == float("inf")
    out = torch.full_like(bad, 9.0)                                     # no limit: the values themselves
    U.check(U.umem_grad_clip(1, table([bad], [out]), float("inf"), torch.tensor([5.0], device="cuda")))
    assert torch.equal(out[:3], bad[:3]) and torch.isnan(out[3])


def test_a_tensor_past_32_bits():
    n = (1 << 31) + 12345
    g = torch.empty((n,), dtype=torch.bfloat16, device="cuda").fill_(0.5)
    g[-1], g[1 << 31] = 4096.0, 2048.0
    tab = table([g], [g])
    norm = norm_of(tab)
    want = np.sqrt((n - 2) * 0.25 + 4096.0 ** 2 + 2048.0 ** 2)
    assert abs(float(norm) - want) <= want * (u + 1e-12)
    U.check(U.umem_grad_clip(1, tab, float(norm) / 2, norm))
    assert float(g[-1]) == 2048.0 and float(g[1 << 31]) == 1024.0 and bool((g[:1 << 31] == 0.25).all())


def test_a_row_count_past_the_rows_of_long_rows():
    """2^31 - 1 rows counted, of 2^32 + 8 elements each: their product is past 63 bits, and the one row there is counts."""
    n = (1 << 32) + 8
    g = torch.empty((1, n), dtype=torch.bfloat16, device="cuda").zero_()
    g[0, 0], g[0, 1 << 32], g[0, n - 1] = 3.0, 12.0, 4.0
    many = torch.tensor([2 ** 31 - 1], dtype=torch.int32, device="cuda")
    tab = table([g], [g], {0: many})
    norm = norm_of(tab)
    assert float(norm) == 13.0
    U.check(U.umem_grad_clip(1, tab, 6.5, norm))
    assert [float(g[0, i]) for i in (0, 1, 1 << 32, n - 1)] == [1.5, 0.0, 6.0, 2.0]


def test_twice_the_same_and_captured():
    """The same bits from every run; a captured norm and clip replayed on new gradients and row counts."""
    grads = make([(500, 512), (4097,), (33,)], 5, {1})
    outs = [torch.zeros_like(g) for g in grads]
    n = torch.tensor([400], dtype=torch.int32, device="cuda")
    tab = table(grads, outs, {0: n})
    st, need = U.umem_grad_workspace_size(3, tab)
    U.check(st)
    ws, norm = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.zeros(1, device="cuda")

    def step():
        U.check(U.umem_grad_norm(3, tab, norm, None, ws, need))
        U.check(U.umem_grad_clip(3, tab, 1.0, norm))

    step()
    first = norm.clone()
    step()
    assert torch.equal(first, norm)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        n.fill_(100 + 150 * k)
        grads[0].mul_(1.5)
        for o in outs:
            o.zero_()
        step()
        torch.cuda.synchronize()
        want = [o.clone() for o in outs] + [norm.clone()]
        for o in outs + [norm]:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs + [norm])), k
