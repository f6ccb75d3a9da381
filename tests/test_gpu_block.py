"""The norms before and after a block on the GPU, and their backward, against the float64 oracle.

Tolerances are sums of roundings.  u = 2^-24 is half a step of fp32.  A row's sum runs through at most 16 additions
in a thread, 6 in its wave and 16 over waves, so a mean is within 40 u of the mean of the magnitudes,
and 1 / spread within half of (40 + 8) u plus what the mean's error adds; x^ is then off by at most
EPS_XH = u (32 |x^| + 48 r max|x|).  Gradients add the same errors of their two row sums; sums over tokens
at most one rounding of the running sum a term.  A bf16 result adds half a step, 2^-8 of its value.
"""
import numpy as np
import pytest
import torch

import oracle.block_oracle as B
import paper_2411_12364_amd as U

pytestmark = pytest.mark.gpu
EPS = 1e-5
u = 2.0 ** -24
NORM = {"layer": U.UMEM_NORM_LAYER, "rms": U.UMEM_NORM_RMS, "none": U.UMEM_NORM_NONE}
GATE = {"none": U.UMEM_GATE_NONE, "channel": U.UMEM_GATE_CHANNEL, "token": U.UMEM_GATE_TOKEN, "full": U.UMEM_GATE_FULL}


def desc(d, norm="layer", norm_out="none", gate="none", act="linear", h="f32", y="f32", eps=EPS, a=1.0, s=1.0):
    return U.umem_block_desc(d, NORM[norm], NORM[norm_out], GATE[gate], int(act == "sigmoid"), int(h == "bf16"),
                             int(y == "bf16"), eps, a, s)


def dtype(t):
    return torch.bfloat16 if t == "bf16" else torch.float32


def host(x):
    return None if x is None else x.detach().double().cpu().numpy()


def half_step(t, value):
    return np.abs(value) * (2.0 ** -8 if t == "bf16" else u)


def within(got, want, tol, what):
    got, want = host(got), np.asarray(want)
    over = np.abs(got - want) - tol
    assert np.isfinite(got).all() and (over <= 0).all(), (what, float(over.max()), float(np.abs(got - want).max()))


class Inputs:
    def __init__(self, T, d, seed, h="f32", y="f32", gate="none", norm_out="layer", shift=True, lead=0):
        g = torch.Generator(device="cuda").manual_seed(seed)

        def rand(shape, t, mean=0.0, scale=1.0):
            # `lead` elements before the array, so that it is aligned to nothing but its elements
            n = int(np.prod(shape))
            x = (torch.randn(lead + n, generator=g, device="cuda") * scale + mean).to(dtype(t))
            return x[lead:].view(shape)

        self.h, self.y = rand((T, d), h, 0.3, 2.0), rand((T, d), y, -0.2, 1.5)
        self.dn, self.dres, self.dh_out = rand((T, d), y), rand((T, d), h), rand((T, d), h)
        self.gamma, self.beta = rand((d,), "f32", 1.0, 0.3), rand((d,), "f32") if shift else None
        self.gamma2, self.beta2 = rand((d,), "f32", 1.0, 0.3), rand((d,), "f32") if shift else None
        if norm_out == "none":
            self.gamma = self.beta = None
        shape = {"none": None, "channel": (d,), "token": (T,), "full": (T, d)}[gate]
        self.gate = None if shape is None else rand(shape, y if gate == "full" else "f32")
        self.rand = rand


def ws_for(bd, T):
    st, need = U.umem_block_backward_workspace_size(bd, T)
    U.check(st)
    return torch.full((max(need, 256),), 0xA5, dtype=torch.uint8, device="cuda")


def eps_xh(x, kind):
    xh, r = B.standardise(x, kind, EPS)
    return u * (32 * np.abs(xh) + 48 * r * np.abs(x).max(axis=1, keepdims=True)), xh, r


def norm_tol(x, kind, gamma, out, t):
    e, _, _ = eps_xh(x, kind)
    return np.abs(gamma) * e + 2 * u * (np.abs(out) + np.abs(gamma) * 0 + 1e-30) + half_step(t, out) + 4 * u


def back_tol(x, kind, gamma, dn, dn_err, extra, out, t):
    """|error| of dx = r (v - mean v - x^ mean(v x^)) + extra; dn_err bounds the error of dn itself."""
    e, xh, r = eps_xh(x, kind)
    v = np.abs(gamma * dn)
    ev = np.abs(gamma) * dn_err + 2 * u * v
    s1 = (v * np.abs(xh)).mean(axis=1, keepdims=True)
    es1 = 48 * u * s1 + (v * e + ev * np.abs(xh)).mean(axis=1, keepdims=True)
    es0 = 48 * u * v.mean(axis=1, keepdims=True) + ev.mean(axis=1, keepdims=True)
    size = v + v.mean(axis=1, keepdims=True) + np.abs(xh) * s1
    er = 32 * u + 48 * u * r * np.abs(x).max(axis=1, keepdims=True)
    return r * (ev + es0 + np.abs(xh) * es1 + e * s1 + size * (er + 4 * u)) + 2 * u * np.abs(extra) + half_step(t, out)


def column_tol(terms, terms_err):
    """|error| of sums over tokens: that of the terms, and one rounding of the running sum a term."""
    n = min(len(terms), 600) + 64
    return terms_err.sum(axis=0) + n * u * np.abs(terms).sum(axis=0) + 1e-30


# rows in a wave's registers, in a workgroup's of 256 and of 1024; odd widths; few rows and many
SIZES = [(1, 1), (3, 3), (5, 64), (1, 255), (7, 512), (1025, 513), (2, 1000), (1023, 1024), (1100, 1023),
         (1024, 2048), (4, 2048), (1, 2050), (33, 4096), (9, 4100), (3, 5001), (2, 16384),
         (520, 8192), (600, 9000), (515, 12289), (3, 16383), (700, 6001), (5, 8193), (530, 8197), (514, 16384),
         (4, 8190), (540, 4099)]
TYPES = [("f32", "f32"), ("bf16", "bf16"), ("f32", "bf16"), ("bf16", "f32")]


@pytest.mark.parametrize("i,size", enumerate(SIZES), ids=["%dx%d" % s for s in SIZES])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_entry(i, size, kind):
    (T, d), (h, y) = size, TYPES[i % 4]
    print(f"[case] entry {T}x{d} {kind} {h} {y}", flush=True)
    x = Inputs(T, d, i, h, y, shift=i % 3 != 0, lead=i % 2)
    bd = desc(d, kind, h=h, y=y)
    n = torch.full((T, d), 7.0, dtype=dtype(y), device="cuda")
    U.check(U.umem_block_in(bd, T, x.h, x.gamma, x.beta, n))
    want = B.block_in(host(x.h), kind, host(x.gamma), host(x.beta), EPS)
    within(n, want, norm_tol(host(x.h), kind, host(x.gamma), want, y), "n")
    if h == y:                                                           # in place: the same bits
        U.check(U.umem_block_in(bd, T, x.h, x.gamma, x.beta, x.h))
        assert torch.equal(x.h, n)


@pytest.mark.parametrize("i,size", enumerate(SIZES), ids=["%dx%d" % s for s in SIZES])
@pytest.mark.parametrize("norm_out", ["none", "layer", "rms"])
def test_exit(i, size, norm_out):
    (T, d), (h, y) = size, TYPES[(i + 1) % 4]
    gate = ["channel", "token", "full", "none"][(i + len(norm_out)) % 4]
    act = ["linear", "sigmoid"][i % 2]
    kind = ["rms", "layer"][(i // 2) % 2]
    print(f"[case] exit {T}x{d} {norm_out} {gate} {act} {h} {y}", flush=True)
    x = Inputs(T, d, 100 + i, h, y, gate, norm_out, shift=i % 3 != 1, lead=i % 2)
    bd = desc(d, kind, norm_out, gate, act, h, y, a=0.7, s=1.3)
    h_out, n = x.rand((T, d), h), x.rand((T, d), y)
    U.check(U.umem_block_out(bd, T, x.h, x.y, x.gate, x.gamma, x.beta, h_out, x.gamma2, x.beta2, n))
    a, s = np.float64(np.float32(0.7)), np.float64(np.float32(1.3))
    hh, yy = host(x.h), host(x.y)
    want = B.block_out(hh, yy, host(x.gate), gate, act, norm_out, host(x.gamma), host(x.beta), EPS, a, s)
    m = B.exit_norm(yy, norm_out, host(x.gamma), host(x.beta), EPS)
    g, _ = B.gate_value(host(x.gate), gate, act, T, d)
    em = 0.0 if norm_out == "none" else norm_tol(yy, norm_out, host(x.gamma), m, "f32")
    within(h_out, want, s * np.abs(g) * em + 10 * u * (np.abs(a * hh) + np.abs(s * g * m)) + half_step(h, want), "h_out")
    # the next entry reads the stream as it is stored, and is the entry's own kernel bit for bit
    stored = host(h_out)
    want = B.block_in(stored, kind, host(x.gamma2), host(x.beta2), EPS)
    within(n, want, norm_tol(stored, kind, host(x.gamma2), want, y), "n_next")
    alone = torch.empty_like(n)
    U.check(U.umem_block_in(bd, T, h_out, x.gamma2, x.beta2, alone))
    assert torch.equal(alone, n)
    again = x.rand((T, d), h)
    U.check(U.umem_block_out(bd, T, x.h, x.y, x.gate, x.gamma, x.beta, again))
    assert torch.equal(again, h_out)                                     # without the next entry
    U.check(U.umem_block_out(bd, T, x.h, x.y, x.gate, x.gamma, x.beta, x.h, x.gamma2, x.beta2, x.y))
    assert torch.equal(x.h, h_out) and torch.equal(x.y, n)               # in place


@pytest.mark.parametrize("i,size", enumerate(SIZES), ids=["%dx%d" % s for s in SIZES])
@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_entry_backward(i, size, kind):
    (T, d), (h, y) = size, TYPES[(i + 2) % 4]
    print(f"[case] entry backward {T}x{d} {kind} {h} {y}", flush=True)
    x = Inputs(T, d, 200 + i, h, y, shift=i % 3 != 0, lead=i % 2)
    dres = x.dres if i % 4 else None
    bd, ws = desc(d, kind, h=h, y=y), ws_for(desc(d), T)
    dh = x.rand((T, d), h)
    dg, db = x.rand((d,), "f32"), x.rand((d,), "f32") if x.beta is not None else None
    U.check(U.umem_block_in_backward(bd, T, x.h, x.gamma, x.dn, dres, dh, dg, db, 0, ws, ws.numel()))
    hh, gamma, dn = host(x.h), host(x.gamma), host(x.dn)
    want, wg, wb = B.block_in_backward(hh, kind, gamma, EPS, dn, host(dres))
    extra = 0.0 if dres is None else host(dres)
    tol = back_tol(hh, kind, gamma, dn, 0.0, extra, want, h)
    within(dh, want, tol, "dh")
    e, xh, _ = eps_xh(hh, kind)
    within(dg, wg, column_tol(dn * xh, np.abs(dn) * e), "dgamma")
    if db is not None:
        within(db, wb, column_tol(dn, np.zeros_like(dn)), "dbeta")
    # added to what is there: one more rounding of the sum
    g0, b0 = x.rand((d,), "f32"), x.rand((d,), "f32") if db is not None else None
    g1, b1 = g0.clone(), b0.clone() if db is not None else None
    same = x.h.clone()
    U.check(U.umem_block_in_backward(bd, T, same, x.gamma, x.dn, dres, same, g1, b1, 1, ws, ws.numel()))
    assert torch.equal(same, dh) and torch.equal(g1, g0 + dg) and (db is None or torch.equal(b1, b0 + db))


@pytest.mark.parametrize("i,size", enumerate(SIZES), ids=["%dx%d" % s for s in SIZES])
@pytest.mark.parametrize("norm_out", ["none", "layer", "rms"])
@pytest.mark.parametrize("gate", ["none", "channel", "token", "full"])
def test_exit_backward(i, size, norm_out, gate):
    (T, d), (h, y) = size, TYPES[(i + len(gate)) % 4]
    act = ["linear", "sigmoid"][(i + len(norm_out)) % 2]
    print(f"[case] exit backward {T}x{d} {norm_out} {gate} {act} {h} {y}", flush=True)
    x = Inputs(T, d, 300 + i, h, y, gate, norm_out, shift=i % 3 != 1, lead=i % 2)
    bd, ws = desc(d, "rms", norm_out, gate, act, h, y, a=0.7, s=1.3), ws_for(desc(d), T)
    a, s = np.float64(np.float32(0.7)), np.float64(np.float32(1.3))
    dh, dy = x.rand((T, d), h), x.rand((T, d), y)
    dgate = None if x.gate is None else x.rand(tuple(x.gate.shape), y if gate == "full" else "f32")
    dg = x.rand((d,), "f32") if x.gamma is not None else None
    db = x.rand((d,), "f32") if x.beta is not None else None
    U.check(U.umem_block_out_backward(bd, T, x.y, x.gate, x.gamma, x.beta, x.dh_out, dh, dy, dgate, dg, db, 0, ws,
                                      ws.numel()))
    yy, up, gamma, beta = host(x.y), host(x.dh_out), host(x.gamma), host(x.beta)
    want = B.block_out_backward(yy, host(x.gate), gate, act, norm_out, gamma, beta, EPS, a, s, up)
    within(dh, want["dh"], half_step(h, want["dh"]) + u * np.abs(want["dh"]), "dh")
    value, slope = B.gate_value(host(x.gate), gate, act, T, d)
    dm = s * up * value
    # the gate's value through exp, a sum and a division: 4 u of itself; its slope through a difference
    # from one as well, 5 u of the value
    edm = 8 * u * np.abs(dm)
    if norm_out == "none":
        within(dy, want["dy"], edm + half_step(y, want["dy"]), "dy")
    else:
        within(dy, want["dy"], back_tol(yy, norm_out, gamma, dm, edm, 0.0, want["dy"], y), "dy")
        e, xh, _ = eps_xh(yy, norm_out)
        within(dg, want["dgamma"], column_tol(dm * xh, np.abs(dm) * e + edm * np.abs(xh)), "dgamma")
        if db is not None:
            within(db, want["dbeta"], column_tol(dm, edm), "dbeta")
    if dgate is not None:
        m = B.exit_norm(yy, norm_out, gamma, beta, EPS)
        em = u * np.abs(m) if norm_out == "none" else norm_tol(yy, norm_out, gamma, m, "f32")
        terms = s * up * m * slope
        err = s * np.abs(up) * (em * np.abs(slope) + np.abs(m) * 6 * u * np.maximum(np.abs(value), np.abs(slope)))
        if gate == "full":
            within(dgate, want["dgate"], err + 4 * u * np.abs(terms) + half_step(y, want["dgate"]), "dgate")
        elif gate == "channel":
            within(dgate, want["dgate"], column_tol(terms, err + 4 * u * np.abs(terms)), "dgate")
        else:
            tol = err.sum(axis=1) + 52 * u * np.abs(terms).sum(axis=1) + 1e-30
            within(dgate, want["dgate"], tol, "dgate")
    # without the stream's gradient, in place, and added to what is there
    y2, gate2 = x.y.clone(), x.gate.clone() if gate == "full" else dgate
    acc = [None if t is None else x.rand(tuple(t.shape), "f32") for t in (dg, db, dgate if gate == "channel" else None)]
    add = [None if t is None else t.clone() for t in acc]
    out_gate = add[2] if gate == "channel" else gate2.clone() if gate == "token" else gate2
    U.check(U.umem_block_out_backward(bd, T, y2, gate2 if gate == "full" else x.gate, x.gamma, x.beta, x.dh_out, None,
                                      y2, out_gate, add[0], add[1], 1, ws, ws.numel()))
    assert torch.equal(y2, dy)
    if gate in ("token", "full"):
        assert torch.equal(out_gate, dgate)
    for before, after, alone in zip(acc, add, (dg, db, dgate)):
        assert before is None or torch.equal(after, before + alone)


@pytest.mark.parametrize("T,longest,d", [(512, 513, 2048), (256, 257, 5000), (2048, 2049, 512), (300, 16384, 300)])
def test_the_workspace_of_a_longer_batch(T, longest, d):
    """A batch in the workspace sized for a longer one: the same gradients."""
    x = Inputs(T, d, 17, gate="channel")
    bd = desc(d, "layer", "layer", "channel")
    need = U.umem_block_backward_workspace_size(bd, longest)[1]

    def grads(ws, n):
        dh, dy, dg, db, dg2, db2, dgate = (torch.empty_like(t) for t in (x.h, x.y, x.gamma, x.beta, x.gamma, x.beta, x.gate))
        U.check(U.umem_block_in_backward(bd, T, x.h, x.gamma, x.dn, x.dres, dh, dg, db, 0, ws, n))
        U.check(U.umem_block_out_backward(bd, T, x.y, x.gate, x.gamma, x.beta, x.dh_out, None, dy, dgate, dg2, db2, 0, ws, n))
        return dh, dy, dg, db, dg2, db2, dgate

    ws = ws_for(bd, T)
    want = grads(ws, ws.numel())
    ws = torch.full((need,), 0xA5, dtype=torch.uint8, device="cuda")
    assert all(torch.equal(a, b) for a, b in zip(grads(ws, need), want))


def test_rows_keep_to_themselves():
    """A token of NaN or infinities, one of zeros, and a gate of zero: every other row as without them."""
    T, d = 1200, 1024
    x = Inputs(T, d, 5, gate="token")
    bd = desc(d, "layer", "layer", "token", a=1.0, s=1.0)
    x.gate[7] = 0.0
    clean, n_clean = torch.empty_like(x.h), torch.empty_like(x.y)
    U.check(U.umem_block_out(bd, T, x.h, x.y, x.gate, x.gamma, x.beta, clean, x.gamma2, x.beta2, n_clean))
    x.y[3], x.y[4, 17], x.y[5] = float("nan"), float("inf"), 0.0
    out, n = torch.empty_like(x.h), torch.empty_like(x.y)
    U.check(U.umem_block_out(bd, T, x.h, x.y, x.gate, x.gamma, x.beta, out, x.gamma2, x.beta2, n))
    rest = torch.tensor([t for t in range(T) if t not in (3, 4, 5)], device="cuda")
    assert torch.equal(out[rest], clean[rest]) and torch.equal(n[rest], n_clean[rest])
    assert torch.isnan(out[3:5]).all() and torch.isnan(n[3:5]).all()
    assert torch.equal(out[7], x.h[7])                                  # a closed gate
    torch.testing.assert_close(out[5], x.h[5] + x.gate[5] * x.beta, rtol=4 * u, atol=4 * u)   # no spread: the shift


def test_offsets_past_32_bits():
    """2^20 rows of 2056: 2.16e9 elements, the last ones past 2^31."""
    T, d = 1 << 20, 2056
    g = torch.Generator(device="cuda").manual_seed(3)
    h = torch.empty((T, d), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    gamma = 1 + 0.1 * torch.randn(d, generator=g, device="cuda")
    n = torch.zeros_like(h)
    bd = desc(d, "rms", "rms", h="bf16", y="bf16")
    U.check(U.umem_block_in(bd, T, h, gamma, None, n))
    at = torch.tensor([0, 1, T // 2, T - 2, T - 1], device="cuda")
    few = torch.empty((len(at), d), dtype=torch.bfloat16, device="cuda")
    want = B.block_in(host(h[at]), "rms", host(gamma), None, EPS)
    within(n[at], want, norm_tol(host(h[at]), "rms", host(gamma), want, "bf16"), "n")
    ws = ws_for(bd, T)
    dg, dy = torch.empty(d, device="cuda"), torch.empty_like(h)
    U.check(U.umem_block_out_backward(bd, T, h, None, gamma, None, n, None, dy, None, dg, None, 0, ws, ws.numel()))
    U.check(U.umem_block_out_backward(bd, len(at), h[at].contiguous(), None, gamma, None, n[at].contiguous(), None, few,
                                      None, torch.empty_like(dg), None, 0, ws, ws.numel()))
    # another group of threads sums the few rows' statistics in another order
    torch.testing.assert_close(dy[at].float(), few.float(), rtol=2.0 ** -7, atol=2.0 ** -12)
    want = torch.zeros(d, dtype=torch.float64, device="cuda")
    for t in range(0, T, 1 << 16):
        x = h[t:t + (1 << 16)].double()
        xh = x * torch.rsqrt((x * x).mean(dim=1, keepdim=True) + EPS)
        want += (n[t:t + (1 << 16)].double() * xh).sum(dim=0)
    assert ((dg.double() - want).abs() <= 600 * u * T * 2).all()         # |terms| average below 2


def test_on_another_stream_and_captured():
    """The calls of a step on a stream of their own, and captured with replays on new inputs."""
    T, d = 1500, 1024
    x = Inputs(T, d, 9, gate="channel")
    bd = desc(d, "layer", "rms", "channel", "sigmoid", a=0.9)
    ws = ws_for(bd, T)
    outs = [torch.zeros_like(x.h) for _ in range(5)] + [torch.zeros(d, device="cuda") for _ in range(5)]

    def step():
        U.check(U.umem_block_out(bd, T, x.h, x.y, x.gate, x.gamma, x.beta, outs[0], x.gamma2, x.beta2, outs[1]))
        U.check(U.umem_block_in_backward(bd, T, outs[0], x.gamma2, x.dn, x.dres, outs[2], outs[5], outs[6], 0, ws,
                                         ws.numel()))
        U.check(U.umem_block_out_backward(bd, T, x.y, x.gate, x.gamma, x.beta, outs[2], outs[3], outs[4], outs[7],
                                          outs[8], outs[9], 0, ws, ws.numel()))

    step()
    torch.cuda.synchronize()
    want = [o.clone() for o in outs]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for o in outs:
        o.zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, outs))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(3):
        x.y.mul_(1.25)
        step()
        torch.cuda.synchronize()
        want = [o.clone() for o in outs]
        for o in outs:
            o.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, outs)), k
