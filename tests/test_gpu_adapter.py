"""Low-rank adapters of many requests on the GPU against the float64 oracle.

u = 2^-24.  Products of bf16 weights with fp32 values are split without loss, so what is rounded are
sums: of d_in terms (each of at most 2 roundings of its size: splitting and adding), then of rank terms,
the scale and the base.  out is off by at most
  u [ (d_in + 64) |s| |B| |A| |x|  +  (rank + 64) |s| |B| |v|  +  4 |base| + 4 |out| ],
and half a step of bf16, 2^-8 of its value, where it is stored so.  (The sums of magnitudes are exact bounds;
no cancellation is counted on.)
"""
import numpy as np
import pytest
import torch

import oracle.block_oracle as B
import oracle.query_oracle as Q
import paper_2411_12364_amd as U
import synth as S
from synth import configs as CF

pytestmark = pytest.mark.gpu
u = 2.0 ** -24


def make(T, n, rank, d_in, d_out, seed, x="f32", o="f32", base=True, scale=True):
    g = torch.Generator(device="cuda").manual_seed(seed)
    t = {"f32": torch.float32, "bf16": torch.bfloat16}

    def rand(shape, s, dt):
        return (torch.randn(shape, generator=g, device="cuda") * s).to(dt)

    return dict(
        desc=U.umem_adapter_desc(n, rank, d_in, d_out, int(x == "bf16"), int(o == "bf16")),
        x=rand((T, d_in), 1.0, t[x]), a=rand((n, rank, d_in), d_in ** -0.5, torch.bfloat16),
        b=rand((n, d_out, rank), rank ** -0.5, torch.bfloat16),
        scale=torch.rand(n, generator=g, device="cuda") + 0.5 if scale else None,
        base=rand((T, d_out), 1.0, t[o]) if base else None, out=torch.full((T, d_out), 9.0, dtype=t[o], device="cuda"),
        g=g)


def call(s, ids, out=None, base="base"):
    T = len(ids)
    st, need = U.umem_adapter_workspace_size(s["desc"], T)
    U.check(st)
    ws = torch.full((max(need, 256),), 0xFF, dtype=torch.uint8, device="cuda")        # NaN wherever it is read unwritten
    out = s["out"] if out is None else out
    U.check(U.umem_adapter_add(s["desc"], T, s["x"], ids, s["a"], s["b"], s["scale"], s[base], out, ws, ws.numel()))
    return out


def host(x):
    return None if x is None else x.detach().double().cpu().numpy()


def check(s, ids, out):
    d = s["desc"]
    x, a, b, scale, base = (host(s[k]) for k in ("x", "a", "b", "scale", "base"))
    i = ids.cpu().numpy()
    want = B.adapter_add(x, i, a, b, scale, base)
    size = B.adapter_add(np.abs(x), i, np.abs(a), np.abs(b), scale, None)
    low = np.zeros_like(size)
    for t, j in enumerate(i):
        if 0 <= j < d.n:
            low[t] = (1.0 if scale is None else scale[j]) * (np.abs(b[j]) @ np.abs(a[j] @ x[t]))
    tol = u * ((d.d_in + 64) * size + (d.rank + 64) * low + 4 * np.abs(want) + (0 if base is None else 4 * np.abs(base)))
    tol += np.abs(want) * (2.0 ** -8 if d.otype else 0.0) + 1e-30
    got = host(out)
    over = np.abs(got - want) - tol
    assert np.isfinite(got).all() and (over <= 0).all(), (float(over.max()), float(np.abs(got - want).max()))
    # the bound is generous where terms cancel: the whole as a norm as well, two roundings a sum on average
    rel = np.linalg.norm(got - want) / max(np.linalg.norm(want), 1e-30)
    assert rel <= (2.0 ** -8 if d.otype else 2e-6), rel


# tokens, adapters, rank, d_in, d_out
SIZES = [(1, 1, 8, 8, 8), (1, 3, 16, 1024, 2048), (2, 2, 128, 264, 136), (5, 64, 16, 72, 4096), (16, 4, 24, 1000, 1000),
         (17, 9, 8, 4096, 512), (33, 2, 64, 2048, 896), (64, 64, 16, 1024, 2048), (100, 7, 40, 520, 1032),
         (255, 3, 32, 128, 264), (300, 300, 8, 64, 64), (513, 5, 56, 1024, 336), (1000, 12, 16, 2048, 896),
         (2049, 16, 32, 256, 520), (4096, 3, 8, 64, 1024), (767, 9, 16, 512, 264), (768, 9, 16, 512, 264),
         (800, 50, 72, 1024, 520), (1024, 1024, 8, 64, 200), (1030, 6, 128, 136, 264), (4097, 3, 48, 2048, 64),
         (4100, 5, 16, 4096, 72), (1535, 9, 16, 264, 520), (1536, 9, 16, 264, 520), (192, 3, 128, 520, 264),
         (400, 90, 64, 264, 1000), (5119, 70, 8, 72, 264), (5121, 3, 8, 520, 136), (5200, 4000, 8, 64, 200),
         (2559, 9, 16, 264, 520), (2560, 400, 16, 264, 520), (1300, 700, 32, 520, 392), (640, 64, 64, 264, 1000),
         (639, 3, 64, 264, 1000), (320, 90, 128, 264, 520), (333, 2, 128, 1032, 264), (700, 80, 56, 4096, 72),
         (1800, 60, 24, 1032, 200), (450, 60, 96, 72, 328)]
TYPES = [("f32", "f32"), ("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16")]


def ids_of(kind, T, n, g):
    if kind == "random":
        return torch.randint(-1, n, (T,), generator=g, device="cuda").to(torch.int32)
    if kind == "one":
        return torch.full((T,), n - 1, dtype=torch.int32, device="cuda")
    runs = torch.sort(torch.randint(0, n, (T,), generator=g, device="cuda")).values
    return ((runs * 7 + 3) % n).to(torch.int32)                          # requests in runs


@pytest.mark.parametrize("i,size", enumerate(SIZES), ids=["x".join(map(str, s)) for s in SIZES])
@pytest.mark.parametrize("kind", ["random", "runs", "one"])
def test_adapters(i, size, kind):
    x, o = TYPES[(i + len(kind)) % 4]
    print(f"[case] adapters {size} {kind} {x} {o}", flush=True)
    s = make(*size, 40 + i, x, o, base=i % 3 != 2, scale=i % 4 != 3)
    ids = ids_of(kind, size[0], size[1], s["g"])
    out = call(s, ids)
    check(s, ids, out)
    if s["base"] is not None:                                            # in place: the same bits
        want, out = out.clone(), s["base"].clone()
        U.check(U.umem_adapter_add(s["desc"], size[0], s["x"], ids, s["a"], s["b"], s["scale"], out, out,
                                   ws := torch.empty(max(256, U.umem_adapter_workspace_size(s["desc"], size[0])[1]),
                                                     dtype=torch.uint8, device="cuda"), ws.numel()))
        assert torch.equal(out, want)


@pytest.mark.parametrize("T", [1, 37, 700, 2001, 2801])
def test_tokens_without_an_adapter(T):
    """ids outside [0, n): the base as it is (or zeros), whatever x holds there."""
    s = make(T, 3, 16, 256, 512, 2)
    ids = torch.tensor([-1, 3, 2 ** 31 - 1, -2 ** 31][:max(1, min(4, T))] * T, dtype=torch.int32, device="cuda")[:T].contiguous()
    s["x"].fill_(float("nan"))
    assert torch.equal(call(s, ids), s["base"])
    s["base"] = None
    assert (call(s, ids) == 0).all()
    if T > 8:                                                            # among others that have one
        s = make(T, 3, 16, 256, 512, 3)
        ids = torch.full((T,), -1, dtype=torch.int32, device="cuda")
        ids[5], ids[T - 1] = 2, 0
        s["x"][6], s["x"][4] = float("nan"), float("inf")
        out = call(s, ids)
        rest = [t for t in range(T) if t not in (5, T - 1)]
        assert torch.equal(out[rest], s["base"][rest])
        few = [5, T - 1]
        part = {**s, "x": s["x"][few], "base": s["base"][few]}
        check(part, ids[few], out[few])


@pytest.mark.parametrize("T", [64, 2048, 2800])
def test_nan_stays_with_its_token_and_adapter(T):
    s = make(T, 4, 16, 256, 512, 4)
    ids = (torch.arange(T, device="cuda") % 4).to(torch.int32)
    clean = call(s, ids).clone()
    s["x"][10, 3] = float("nan")
    s["a"][3] = float("inf")
    out = call(s, ids)
    rest = [t for t in range(T) if t != 10 and t % 4 != 3]
    assert torch.equal(out[rest], clean[rest])
    assert torch.isnan(out[10]).all() and not torch.isfinite(out[3]).any()


@pytest.mark.parametrize("T", [3, 2000, 6000])
def test_every_digit_of_the_input_counts(T):
    """x = 1 + 2^-23 against weights that cancel its leading part: a rounded x would give zero."""
    s = make(T, 1, 8, 64, 64, 6, base=False, scale=False)
    s["x"].fill_(1.0)
    s["x"][:, 0] = 1.0 + 2.0 ** -23
    s["a"].zero_()
    s["a"][0, 0, 0], s["a"][0, 0, 1] = 1.0, -1.0
    s["b"].zero_()
    s["b"][0, :, 0] = 1.0
    out = call(s, torch.zeros(T, dtype=torch.int32, device="cuda"))
    assert torch.equal(out, torch.full_like(out, 2.0 ** -23))


@pytest.mark.parametrize("T", [2, 2000, 6000])
def test_largest_values_and_infinities(T):
    """The largest fp32 values stay finite on the way, an infinity is itself."""
    s = make(T, 1, 8, 64, 64, 6, base=False, scale=False)
    big = torch.finfo(torch.float32).max
    s["x"].zero_()
    s["x"][:, 0] = big
    s["x"][1, 0] = float("inf")
    s["a"].zero_()
    s["a"][0, :, 0] = 0.5
    s["b"].zero_()
    s["b"][0, :, 0] = 1.0
    s["b"][0, :, 1] = -0.5
    out = call(s, torch.zeros(T, dtype=torch.int32, device="cuda"))
    rest = torch.arange(T, device="cuda") != 1
    want = torch.full_like(out[rest], big * 0.25)
    assert ((out[rest] - want).abs() <= 4 * u * want).all() and not torch.isfinite(out[1]).any()


@pytest.mark.parametrize("T,n", [(7, 3), (6000, 3), (6000, 4000)])
@pytest.mark.parametrize("rank", [8, 24, 40])
def test_an_infinite_input_gives_infinities(T, n, rank):
    """Its token's outputs are infinite with the signs of the weights' products, not NaN, whatever rank the
    kernel pads to; the other tokens' stay what they are."""
    s = make(T, n, rank, 64, 136, 11)
    s["a"], s["b"] = s["a"].abs() + 0.25, s["b"].abs() + 0.25
    s["b"][:, ::3] *= -1
    ids = ids_of("random", T, n, s["g"])
    ids[1], ids[4] = 0, n - 1
    clean = call(s, ids).clone()
    s["x"][1, 5], s["x"][4, 63] = float("inf"), -float("inf")
    out = call(s, ids)
    sign = torch.ones(136, device="cuda")
    sign[::3] = -1
    assert torch.equal(out[1], sign * float("inf")) and torch.equal(out[4], -sign * float("inf"))
    rest = [t for t in range(T) if t not in (1, 4)]
    assert torch.equal(out[rest], clean[rest])


@pytest.mark.parametrize("T,n", [(7, 3), (6000, 3), (6000, 4000)])
@pytest.mark.parametrize("rank,x", [(8, "f32"), (24, "bf16"), (40, "f32"), (128, "f32"), (64, "bf16")])
def test_infinite_weights_give_what_the_formula_gives(T, n, rank, x):
    """Whatever the number of tokens: infinities of A, of B and of both, zeros of x among what they meet."""
    s = make(T, n, rank, 136, 72, 21, x)
    s["x"][::5, 17] = 0.0
    s["a"][0, 3, 17], s["a"][1, rank - 1, 135] = float("inf"), -float("inf")
    s["b"][1, 5, 2], s["b"][1, 71, rank - 1], s["b"][2, 9, 0], s["b"][2, 9, 1] = float("inf"), float("inf"), -float("inf"), float("inf")
    ids = ids_of("random", T, n, s["g"])
    ids[1], ids[4], ids[5], ids[6] = 0, 1, 0, 2
    out = host(call(s, ids))
    v = {k: host(s[k]) for k in ("x", "a", "b", "scale", "base")}
    i = ids.cpu().numpy()
    with np.errstate(invalid="ignore", over="ignore"):
        want = B.adapter_add(v["x"], i, v["a"], v["b"], v["scale"], v["base"])
    assert np.isposinf(want).any() and np.isneginf(want).any() and np.isnan(want).any() and np.isfinite(want).any()
    assert (np.isnan(out) == np.isnan(want)).all()
    assert (np.isposinf(out) == np.isposinf(want)).all() and (np.isneginf(out) == np.isneginf(want)).all()
    fine = (i != 0) & (i != 1) & (i != 2)
    few = torch.from_numpy(fine).cuda()
    check({**s, "x": s["x"][few], "base": s["base"][few]}, ids[few], torch.from_numpy(out).cuda()[few])


@pytest.mark.parametrize("o", ["f32", "bf16"])
@pytest.mark.parametrize("T", [5, 2800])
def test_base_of_negative_zeros(T, o):
    """A token without an adapter keeps its base bit for bit."""
    s = make(T, 3, 16, 64, 136, 9, o=o)
    s["base"].mul_(0.0).abs_().neg_()
    ids = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    ids[3] = 1
    out = call(s, ids)
    rest = [t for t in range(T) if t != 3]
    bits = torch.int32 if o == "f32" else torch.int16
    assert torch.equal(out[rest].view(bits), s["base"][rest].view(bits))
    assert torch.signbit(s["base"]).all()


@pytest.mark.parametrize("T,longest,rank,d_in,x", [(4032, 4096, 32, 4096, "bf16"), (1920, 4096, 32, 4096, "bf16"),
                                                   (640, 1024, 64, 2048, "f32"), (1984, 1985, 32, 2048, "f32"),
                                                   (100, 8192, 16, 1024, "f32")])
def test_the_workspace_of_more_tokens(T, longest, rank, d_in, x):
    """Fewer tokens in the workspace sized for more: the same sums."""
    s = make(T, 9, rank, d_in, 264, 15, x)
    ids = ids_of("runs", T, 9, s["g"])
    want = call(s, ids).clone()
    st, need = U.umem_adapter_workspace_size(s["desc"], longest)
    U.check(st)
    ws = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.full_like(want, 9.0)
    U.check(U.umem_adapter_add(s["desc"], T, s["x"], ids, s["a"], s["b"], s["scale"], s["base"], out, ws, need))
    assert torch.equal(out, want)


# tokens, adapters, rank, d_in, d_out: wide enough that a workgroup sums over several pieces of d_in, the last run
# and the last piece shorter
WIDE = [((4100, 5, 128, 8264, 72), "f32", "runs"), ((4100, 300, 24, 8264, 72), "f32", "random"),
        ((1300, 3, 32, 12616, 264), "f32", "one"), ((1300, 9, 40, 50248, 64), "bf16", "random"),
        ((4100, 6, 16, 16392, 136), "bf16", "runs"), ((4100, 7, 72, 16392, 64), "bf16", "one")]


@pytest.mark.parametrize("size,x,kind", WIDE, ids=["x".join(map(str, s)) for s, _, _ in WIDE])
def test_wide_inputs(size, x, kind):
    print(f"[case] wide adapters {size} {x} {kind}", flush=True)
    s = make(*size, 80, x, "f32")
    ids = ids_of(kind, size[0], size[1], s["g"])
    out = call(s, ids)
    check(s, ids, out)
    assert torch.equal(call(s, ids, torch.empty_like(out)), out)


@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_wide_inputs_of_few_adapted_tokens(x):
    """Whole tiles without an adapter, and NaN and infinities among the others."""
    T, d_in = 4100, 8264 if x == "f32" else 16392
    s = make(T, 3, 24, d_in, 72, 81, x)
    ids = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    at = [5, 70, 71, 2000, T - 1]
    ids[at] = torch.tensor([2, 0, 1, 1, 0], dtype=torch.int32, device="cuda")
    few = torch.tensor(at, device="cuda")
    s["x"][6], s["x"][72], s["x"][T - 2] = float("nan"), float("inf"), float("nan")
    out = call(s, ids)
    rest = torch.ones(T, dtype=torch.bool, device="cuda")
    rest[few] = False
    assert torch.equal(out[rest], s["base"][rest])
    check({**s, "x": s["x"][few], "base": s["base"][few]}, ids[few], out[few])
    s["a"], s["b"] = s["a"].abs() + 0.25, s["b"].abs() + 0.25
    s["x"][70, d_in - 1], s["x"][2000, 0] = float("inf"), float("nan")
    out = call(s, ids)
    assert (out[70] == float("inf")).all() and torch.isnan(out[2000]).all()
    assert torch.isfinite(out[[5, 71, T - 1]]).all()


def test_offsets_past_32_bits():
    """2^20 tokens of 2056: out has 2.16e9 elements."""
    T, d_out = 1 << 20, 2056
    s = make(64, 2, 8, 64, d_out, 8, x="bf16", o="bf16", base=False)
    s["x"] = torch.randn((T, 64), generator=s["g"], device="cuda").to(torch.bfloat16)
    s["out"] = torch.full((T, d_out), 9.0, dtype=torch.bfloat16, device="cuda")
    ids = (torch.arange(T, device="cuda") % 3 - 1).to(torch.int32)
    out = call(s, ids)
    at = torch.tensor([0, 1, 2, T // 2, T - 3, T - 2, T - 1], device="cuda")
    check({**s, "x": s["x"][at]}, ids[at], out[at])


@pytest.mark.parametrize("T", [3, 64, 900, 3000])
def test_captured_and_on_another_stream(T):
    s = make(T, 6, 16, 512, 1024, 12)
    ids = ids_of("random", T, 6, s["g"])
    st, need = U.umem_adapter_workspace_size(s["desc"], T)
    U.check(st)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")

    def step(out):
        U.check(U.umem_adapter_add(s["desc"], T, s["x"], ids, s["a"], s["b"], s["scale"], s["base"], out, ws, ws.numel()))

    want, out = torch.empty_like(s["out"]), torch.empty_like(s["out"])
    step(want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(out)
    side.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(out)
    for k in range(3):
        ids.copy_(torch.roll(ids, 1))
        s["x"].mul_(1.5)
        step(want)
        torch.cuda.synchronize()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want), k


# ---------------------------------------------------------------- beside the query linear

FRONT_ENDS = [
    # one new token of each sequence; a prompt each, cut off at ragged places; enough tokens for the tiles
    CF.FrontEnd("adapted-decode", B=24, L=1, d_model=256, conv_k=4, heads=2, dk=64, shared=True, seed=51),
    CF.FrontEnd("adapted-separate", B=3, L=37, d_model=1024, conv_k=3, heads=1, dk=40, shared=False, seed=52, history=False),
    CF.FrontEnd("adapted-prompts", B=4, L=431, d_model=512, conv_k=4, heads=2, dk=128, shared=True, seed=53),
    CF.FrontEnd("adapted-long-prompts", B=4, L=801, d_model=256, conv_k=4, heads=2, dk=64, shared=True, seed=54),
]


def qdesc(fe):
    return U.umem_query_desc(fe.d_model, fe.conv_k, fe.heads, fe.dk, int(fe.shared), fe.eps)


def row_err(got, want):
    """Of the largest value of each query."""
    got, want = got.reshape(-1, want.shape[-1]), want.reshape(-1, want.shape[-1])
    return float((np.abs(got - want).max(axis=1) / np.abs(want).max(axis=1)).max())


# fp32 accumulation, and a rare bf16 rounding of the convolved rows decided the other way
ROUNDED_RTOL = 2e-3


@pytest.mark.parametrize("fe", FRONT_ENDS, ids=[f.name for f in FRONT_ENDS])
def test_adapted_query(fe):
    """The front-end with an adapter for each sequence against the oracle's steps with the merged weights, from
    its own convolved rows rounded to bf16 as the linear takes them; without an adapter for any token, and
    with adapters of zeros, bit for bit umem_query."""
    print(f"[case] adapted query {fe.name}", flush=True)
    inp = CF.front_end_inputs(fe)
    A, n, rank, nq = (1 if fe.shared else 2), 3, 16, fe.n_queries
    s = make(fe.T, n, rank, fe.d_model, nq, fe.seed, "bf16", "f32")
    s["b"] *= 0.5                                                        # adapters of the size of the linear's output
    seq = torch.randint(-1, n, (fe.B,), generator=s["g"], device="cuda").to(torch.int32)
    seq[0], seq[1] = 0, -1
    ids = seq.repeat_interleave(fe.L).contiguous()
    st, need = U.umem_query_adapted_workspace_size(qdesc(fe), s["desc"], fe.B, fe.L)
    U.check(st)
    dev = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()   # noqa: E731
    args = [dev(inp["x"]), dev(inp["hist"]), dev(inp["conv_w"]), dev(CF.output_major(inp["w_q"]).view(np.int16))]
    norms = [dev(inp["gamma"]), dev(inp["beta"])]
    q_row = torch.empty((fe.T, fe.heads, fe.dk), device="cuda")
    q_col = q_row if fe.shared else torch.empty_like(q_row)
    st, plain = U.umem_query_workspace_size(qdesc(fe), fe.B, fe.L)
    U.check(st)
    ws = torch.empty(max(plain, 256), dtype=torch.uint8, device="cuda")
    U.check(U.umem_query(qdesc(fe), fe.B, fe.L, *args, *norms, q_row, None if fe.shared else q_col, ws, ws.numel()))

    def call(ids, b=s["b"]):
        ws = torch.full((max(need, 256),), 0xFF, dtype=torch.uint8, device="cuda")
        row = torch.empty_like(q_row)
        col = None if fe.shared else torch.empty_like(q_row)
        U.check(U.umem_query_adapted(qdesc(fe), s["desc"], fe.B, fe.L, *args, ids, s["a"], b, s["scale"], *norms, row, col,
                                     ws, ws.numel()))
        return row, (row if fe.shared else col)

    for got in (call(torch.full_like(ids, -1)), call(ids, torch.zeros_like(s["b"]))):
        assert torch.equal(got[0], q_row) and torch.equal(got[1], q_col)
    got = call(ids)
    y = Q.causal_conv(inp["x"], inp["conv_w"], inp["hist"]).reshape(fe.T, fe.d_model)
    y = S.bf16_bits_to_f32(S.f32_to_bf16_bits(y.astype(np.float32))).reshape(y.shape).astype(np.float64)
    wq = S.bf16_bits_to_f32(inp["w_q"]).reshape(inp["w_q"].shape).astype(np.float64)
    lin = B.adapter_add(y, ids.cpu().numpy(), host(s["a"]), host(s["b"]), host(s["scale"]), Q.query_linear(y, wq))
    want = Q.layer_norm(lin.reshape(fe.T, A, fe.heads, fe.dk), np.asarray(inp["gamma"], np.float64).reshape(A, fe.heads, fe.dk),
                        np.asarray(inp["beta"], np.float64).reshape(A, fe.heads, fe.dk), fe.eps)
    for x, a in ((got[0], 0), (got[1], A - 1)):
        assert row_err(host(x), want[:, a]) <= ROUNDED_RTOL
    off = ids.cpu().numpy() < 0                                          # sequences without one: as without any
    assert torch.equal(got[0][torch.from_numpy(off).cuda()], q_row[torch.from_numpy(off).cuda()])
    assert not torch.equal(got[0], q_row)
