"""Refusals of the block, gradient and adapter entry points, on the host: every call below fails
validation, sizes a workspace or has nothing to do, so no kernel is launched."""
import ctypes

import numpy as np
import pytest

import paper_2411_12364_amd as U

OK, ARG, UNS, WS = U.UMEM_OK, U.UMEM_ERR_INVALID_ARG, U.UMEM_ERR_UNSUPPORTED, U.UMEM_ERR_WORKSPACE
MB = 1 << 20


def at(i):
    """Addresses 64 MiB apart, never dereferenced."""
    return (i + 1) * 64 * MB


def bd(**kw):
    base = dict(d=256, norm_in=0, norm_out=0, gate=0, gate_act=0, htype=0, ytype=0, eps=1e-5, res_scale=1.0,
                out_scale=1.0)
    return U.umem_block_desc(*{**base, **kw}.values())


@pytest.mark.parametrize("kw,want", [
    (dict(), OK), (dict(d=0), ARG), (dict(d=16384), OK), (dict(d=16385), UNS), (dict(d=1), OK),
    (dict(norm_in=2), ARG), (dict(norm_in=-1), ARG), (dict(norm_out=3), ARG), (dict(norm_out=2), OK),
    (dict(gate=4), ARG), (dict(gate=-1), ARG), (dict(gate_act=2), ARG), (dict(htype=2), ARG), (dict(ytype=-1), ARG),
    (dict(eps=-1e-9), ARG), (dict(eps=float("nan")), ARG), (dict(eps=float("inf")), ARG), (dict(eps=0.0), OK),
    (dict(res_scale=float("inf")), ARG), (dict(out_scale=float("nan")), ARG),
])
def test_block_descriptor(kw, want):
    st, n = U.umem_block_backward_workspace_size(bd(**kw), 8)
    assert st == want and (n > 0) == (want == OK)
    assert U.umem_block_in(bd(**kw), 0, None, None, None, None, 0) == want
    assert U.umem_block_backward_workspace_size(bd(), -1)[0] == ARG
    assert U.umem_block_backward_workspace_size(bd(), (1 << 20) + 1)[0] == UNS
    assert U.umem_block_backward_workspace_size(bd(), 0) == (OK, 0)


def test_block_in_refusals():
    h, g, b, n = at(0), at(1), at(2), at(3)
    call = lambda h=h, g=g, b=b, n=n, d=bd(), T=8: U.umem_block_in(d, T, h, g, b, n, 0)   # noqa: E731
    assert call(h=None) == ARG and call(g=None) == ARG and call(n=None) == ARG
    assert call(h=h + 2) == ARG and call(n=n + 1) == ARG and call(g=g + 2) == ARG and call(b=b + 3) == ARG
    assert call(h=h + 1, d=bd(htype=1)) == ARG
    assert call(n=h + 4) == ARG                                        # overlaps h without being it
    assert call(n=h, d=bd(htype=1)) == ARG                             # ... in another type
    assert call(n=g) == ARG
    assert call(T=-1) == ARG and call(T=(1 << 20) + 1) == UNS


def test_block_out_refusals():
    names = ["h", "y", "gate", "gamma", "beta", "h_out", "gamma_next", "beta_next", "n_next"]
    base = {k: at(i) for i, k in enumerate(names)}

    def call(desc=bd(gate=1), T=8, **kw):
        return U.umem_block_out(desc, T, *{**base, **kw}.values(), 0)

    for k in ("h", "y", "h_out", "gate", "gamma"):
        assert call(**{k: None}) == ARG, k
    assert call(desc=bd(gate=0)) == ARG                                 # a gate that the descriptor lacks
    assert call(desc=bd(gate=1, norm_out=2)) == ARG                     # gamma without a norm
    assert call(desc=bd(gate=1, norm_out=2), gamma=None) == ARG         # beta without a norm
    assert call(gamma_next=None) == ARG and call(n_next=None) == ARG    # half of the next entry
    assert call(gamma_next=None, n_next=None) == ARG                    # its shift alone
    for k in names:
        assert call(**{k: base[k] + 1}) == ARG, k
    assert call(h_out=base["y"]) == ARG and call(h_out=base["h"] + 256) == ARG
    assert call(n_next=base["h"]) == ARG and call(n_next=base["h_out"]) == ARG
    assert call(desc=bd(gate=3), h_out=base["gate"]) == ARG


def test_block_backward_refusals():
    st, need = U.umem_block_backward_workspace_size(bd(gate=1), 8)
    assert st == OK
    names = ["h", "gamma", "dn", "dres", "dh", "dgamma", "dbeta"]
    base = {k: at(i) for i, k in enumerate(names)}
    ws = at(20)

    def call(T=8, acc=0, ws=ws, n=need, desc=bd(), **kw):
        return U.umem_block_in_backward(desc, T, *{**base, **kw}.values(), acc, ws, n, 0)

    for k in ("h", "gamma", "dn", "dh", "dgamma"):
        assert call(**{k: None}) == ARG, k
    for k in names:
        assert call(**{k: base[k] + 2}) == ARG, k
    assert call(acc=2) == ARG and call(acc=-1) == ARG and call(T=0, acc=2) == ARG and call(T=0) == OK
    assert call(ws=None) == WS and call(ws=ws + 8) == WS and call(n=need - 1) == WS
    assert call(dh=base["dn"]) == ARG and call(dgamma=base["dbeta"]) == ARG and call(dgamma=ws) == ARG
    assert call(dh=base["h"] + 512) == ARG and call(dh=ws) == ARG

    names = ["y", "gate", "gamma", "beta", "dh_out", "dh", "dy", "dgate", "dgamma", "dbeta"]
    base = {k: at(i) for i, k in enumerate(names)}

    def call(T=8, acc=0, ws=ws, n=need, desc=bd(gate=1), **kw):      # noqa: F811
        return U.umem_block_out_backward(desc, T, *{**base, **kw}.values(), acc, ws, n, 0)

    for k in ("y", "gate", "gamma", "dh_out", "dy", "dgate", "dgamma"):
        assert call(**{k: None}) == ARG, k
    assert call(beta=None) == ARG and call(dbeta=None) == ARG
    assert call(desc=bd(gate=0)) == ARG and call(desc=bd(gate=1, norm_out=2)) == ARG
    for k in names:
        assert call(**{k: base[k] + 1}) == ARG, k
    assert call(acc=3) == ARG and call(T=0) == OK
    assert call(ws=None) == WS and call(ws=ws + 4) == WS and call(n=0) == WS
    assert call(dy=base["dh_out"]) == ARG and call(dh=base["y"]) == ARG and call(dgate=base["gate"]) == ARG
    assert call(dy=base["dh"]) == ARG and call(dgamma=base["gamma"]) == ARG and call(dbeta=ws + 16) == ARG


@pytest.mark.parametrize("d", [1, 256, 257, 512, 513, 1024, 2048, 2049, 4096, 5000, 8192, 8193, 16384])
def test_block_workspace_never_falls_with_the_tokens(d):
    """A program sizes its workspace once, for its longest batch."""
    sizes = [U.umem_block_backward_workspace_size(bd(d=d), T) for T in range(4200)]
    assert all(st == OK for st, _ in sizes)
    sizes = [n for _, n in sizes] + [U.umem_block_backward_workspace_size(bd(d=d), T)[1] for T in (1 << 16, (1 << 16) + 1, 1 << 20)]
    assert all(a <= b for a, b in zip(sizes, sizes[1:]))
    assert sizes[-1] <= 512 * 3 * 4 * d + 256                            # whatever the batch


def test_block_backward_scratch_is_apart_from_the_inputs():
    """The scratch is written while other workgroups read."""
    desc = bd(gate=1)
    need = U.umem_block_backward_workspace_size(desc, 8)[1]
    names = ["h", "gamma", "dn", "dres", "dh", "dgamma", "dbeta"]
    base = {k: at(i) for i, k in enumerate(names)}
    for k in ("h", "gamma", "dn", "dres"):
        for ws in (base[k], base[k] + 16, base[k] - need + 16):
            assert U.umem_block_in_backward(bd(), 8, *base.values(), 0, ws, need, 0) == ARG, k
    names = ["y", "gate", "gamma", "beta", "dh_out", "dh", "dy", "dgate", "dgamma", "dbeta"]
    base = {k: at(i) for i, k in enumerate(names)}
    for k in ("y", "gate", "gamma", "beta", "dh_out"):
        for ws in (base[k], base[k] + 16, base[k] - need + 16):
            assert U.umem_block_out_backward(desc, 8, *base.values(), 0, ws, need, 0) == ARG, k


def grads(*rows):
    return (U.umem_grad * len(rows))(*[U.umem_grad(*r) for r in rows])


def test_grad_refusals():
    norm, ws = at(30), at(31)
    good = grads((at(0), at(1), None, 4, 100, 0), (at(2), at(2), at(3), 7, 33, 1))
    st, need = U.umem_grad_workspace_size(2, good)
    assert st == OK and need > 0
    assert U.umem_grad_workspace_size(0, None) == (OK, 0) and U.umem_grad_workspace_size(1, None)[0] == ARG
    assert U.umem_grad_workspace_size(-1, good)[0] == ARG
    assert U.umem_grad_workspace_size(2049, (U.umem_grad * 2049)())[0] == UNS
    assert U.umem_grad_norm(2, good, None, None, ws, need, 0) == ARG
    assert U.umem_grad_norm(2, good, norm + 2, None, ws, need, 0) == ARG
    assert U.umem_grad_norm(2, good, norm, norm + 4, ws, need, 0) == ARG
    assert U.umem_grad_norm(2, good, norm, None, None, need, 0) == WS
    assert U.umem_grad_norm(2, good, norm, None, ws, need - 1, 0) == WS
    assert U.umem_grad_norm(2, good, norm, None, ws + 8, need, 0) == WS
    assert U.umem_grad_clip(2, good, -1.0, norm, 0) == ARG and U.umem_grad_clip(2, good, float("nan"), norm, 0) == ARG
    assert U.umem_grad_clip(2, good, 1.0, None, 0) == ARG
    bad = {
        "rows": (at(0), at(1), None, -1, 4, 0), "row_len": (at(0), at(1), None, 4, -1, 0),
        "type": (at(0), at(1), None, 4, 4, 2), "null": (None, at(1), None, 4, 4, 0),
        "odd": (at(0) + 2, at(1), None, 4, 4, 0), "odd rows": (at(0), at(1), at(2) + 1, 4, 4, 0),
    }
    for name, row in bad.items():
        assert U.umem_grad_workspace_size(1, grads(row))[0] == ARG, name
        assert U.umem_grad_norm(1, grads(row), norm, None, ws, 1 << 20, 0) == ARG, name
        assert U.umem_grad_clip(1, grads(row), 1.0, norm, 0) == ARG, name
    for row in ((at(0), at(1), None, 1 << 30, 1 << 11, 0), (at(0), at(1), None, 1 << 62, 1 << 62, 0)):
        assert U.umem_grad_workspace_size(1, grads(row))[0] == UNS
    # without elements nothing of a gradient is looked at
    assert U.umem_grad_workspace_size(1, grads((None, None, None, 0, 100, 0))) == (OK, 0)
    assert U.umem_grad_clip(1, grads((None, None, None, 5, 0, 1)), 1.0, norm, 0) == OK
    assert U.umem_grad_clip(0, None, 1.0, norm, 0) == OK
    # no place to write, or one that another is read from or written to
    k = 4096
    for rows in ([(at(0), None, None, 1, k, 0)], [(at(0), at(1) + 2, None, 1, k, 0)],
                 [(at(0), at(0) + 4, None, 1, k, 0)],
                 [(at(0), at(1), None, 1, k, 0), (at(2), at(1) + 4 * k - 4, None, 1, k, 0)],
                 [(at(0), at(0), None, 1, k, 0), (at(0), at(0), None, 1, k, 0)],
                 [(at(0), at(1), None, 1, k, 0), (at(1) + 4, at(3), None, 1, 8, 0)],
                 [(at(2), at(3), None, 1, k, 0), (at(1), at(1), None, 1, k, 0), (at(0), at(2) - 4, None, 1, 2, 0)]):
        assert U.umem_grad_clip(len(rows), grads(*rows), 1.0, norm, 0) == ARG, rows


def test_a_clipped_gradient_is_apart_from_the_norm_and_the_row_counts():
    """What the kernels read while they write the outs."""
    row, k = (at(0), at(1), at(2), 4, 1024, 0), 4 * 4 * 1024
    assert U.umem_grad_clip(1, grads(row), 1.0, at(1), 0) == ARG
    assert U.umem_grad_clip(1, grads(row), 1.0, at(1) + k - 4, 0) == ARG
    assert U.umem_grad_clip(1, grads((at(0), at(1), at(1) + 8, 4, 1024, 0)), 1.0, at(9), 0) == ARG
    other = (at(3), at(4), None, 4, 1024, 1)
    assert U.umem_grad_clip(2, grads((at(0), at(1), at(4), 4, 1024, 0), other), 1.0, at(9), 0) == ARG
    assert U.umem_grad_norm(1, grads(row), at(9) + 4, at(9), at(10), 1 << 20, 0) == ARG
    # apart, in a table without elements, which launches nothing
    assert U.umem_grad_clip(1, grads((at(0), at(1), at(2), 0, 1024, 0)), 1.0, at(9), 0) == OK


def test_the_norm_is_apart_from_the_gradients_and_its_scratch():
    """What umem_grad_norm writes, against what it reads and against each other."""
    tab = grads((at(0), at(1), at(2), 4, 1024, 0), (at(3), at(4), None, 40, 1024, 1))
    st, need = U.umem_grad_workspace_size(2, tab)
    assert st == OK and need > 0
    call = lambda norm=at(9), sumsq=at(10), ws=at(11): U.umem_grad_norm(2, tab, norm, sumsq, ws, need, 0)   # noqa: E731
    last = at(3) + 2 * 40 * 1024
    for a in (at(0), at(0) + 4 * 4 * 1024 - 8, at(3) + 8, last - 8, at(2)):
        assert call(norm=a) == ARG and call(sumsq=a // 8 * 8) == ARG
    for a in (at(0), at(0) - need + 16, at(2) - 16, last - 16, at(9) - 16, at(10), at(9) // 16 * 16):
        assert call(ws=a) == ARG, a
    assert call(norm=at(10) + 4) == ARG and call(norm=at(11) + 8) == ARG and call(sumsq=at(11) + need - 8) == ARG


def test_grad_tables_of_the_binding():
    rows = [(at(0), at(1), 0, 4, 100, 0), (at(2), at(2), at(3), 7, 33, 1)]
    table = np.array(rows, dtype=np.int64)
    assert U.umem_grad_workspace_size(2, table) == U.umem_grad_workspace_size(2, grads(*rows))
    assert ctypes.sizeof(U.umem_grad) == 48
    for wrong in (table.astype(np.float64), table[:, :5], table.T, table[:1], table[0], table[:, ::-1]):
        with pytest.raises(ValueError):
            U.umem_grad_workspace_size(2, wrong)
    with pytest.raises(ValueError):
        U.umem_grad_workspace_size(2, grads(rows[0]))
    with pytest.raises(ValueError):
        U.umem_grad_workspace_size(2, (ctypes.c_int64 * 12)())


def ad(**kw):
    base = dict(n=4, rank=16, d_in=64, d_out=128, xtype=0, otype=0)
    return U.umem_adapter_desc(*{**base, **kw}.values())


@pytest.mark.parametrize("kw,want", [
    (dict(), OK), (dict(n=0), ARG), (dict(rank=0), ARG), (dict(d_in=0), ARG), (dict(d_out=-8), ARG),
    (dict(xtype=2), ARG), (dict(otype=-1), ARG), (dict(rank=12), UNS), (dict(rank=136), UNS), (dict(rank=128), OK),
    (dict(d_in=60), UNS), (dict(d_out=1 << 17), UNS), (dict(d_in=1 << 16), OK),
])
def test_adapter_descriptor(kw, want):
    assert U.umem_adapter_workspace_size(ad(**kw), 8)[0] == want
    assert U.umem_adapter_add(ad(**kw), 0, None, None, None, None, None, None, None, None, 0, 0) == want
    assert U.umem_adapter_workspace_size(ad(), -1)[0] == ARG
    assert U.umem_adapter_workspace_size(ad(), (1 << 20) + 1)[0] == UNS


@pytest.mark.parametrize("kw", [
    dict(d_in=1024, rank=16, xtype=1), dict(d_in=4096, rank=32, xtype=1), dict(d_in=2048, rank=64), dict(d_in=4096, rank=128),
    dict(d_in=1 << 16, rank=128, xtype=1), dict(d_in=1 << 16, rank=8), dict(d_in=72, rank=24), dict(d_in=264, rank=128),
    dict(d_in=8192, rank=8, xtype=1),
])
def test_adapter_workspace_never_falls_with_the_tokens(kw):
    """A program sizes its workspace once, for its longest prompts."""
    tokens = [*range(0, 9000), *range(9000, 70000, 61), 1 << 17, (1 << 20) - 1, 1 << 20]
    sizes = [U.umem_adapter_workspace_size(ad(**kw), T) for T in tokens]
    assert all(st == OK for st, _ in sizes)
    assert all(a[1] <= b[1] for a, b in zip(sizes, sizes[1:]))


def test_adapter_workspace_does_not_grow_with_the_input_width():
    for kw in (dict(rank=128), dict(rank=8), dict(rank=72, xtype=1), dict(rank=16, xtype=1)):
        r = (kw["rank"] + 15) // 16 * 16
        for d_in in (64, 2048, 4096 + 72, 1 << 16):
            for T in (*range(300, 20000, 119), 1 << 16, (1 << 17) + 1, 1 << 20):
                st, n = U.umem_adapter_workspace_size(ad(d_in=d_in, **kw), T)
                assert st == OK and n <= 4 * r * max(T, 1 << 17) + 256, (kw, d_in, T)


def test_adapter_refusals():
    names = ["x", "ids", "a", "b", "scale", "base", "out"]
    base = {k: at(i) for i, k in enumerate(names)}

    def call(T=8, **kw):
        return U.umem_adapter_add(ad(), T, *{**base, **kw}.values(), at(20), 32 * MB, 0)

    for k in ("x", "ids", "a", "b", "out"):
        assert call(**{k: None}) == ARG, k
    for k in names:
        assert call(**{k: base[k] + 2}) == ARG, k
    for k in ("x", "a", "b", "base", "out"):
        assert call(**{k: base[k] + 8}) == ARG, k
    assert call(out=base["x"]) == ARG and call(out=base["base"] + 16) == ARG and call(out=base["b"] + 1024) == ARG
    assert call(T=-1) == ARG
    for T in (1, 8, 100, 5000):
        st, need = U.umem_adapter_workspace_size(ad(), T)
        assert st == OK
        if need:
            args = [ad(), T, *base.values()]
            assert U.umem_adapter_add(*args, None, need, 0) == WS
            assert U.umem_adapter_add(*args, at(20), need - 1, 0) == WS
            assert U.umem_adapter_add(*args, at(20) + 16, need, 0) == WS


def test_adapter_scratch_is_apart_from_the_inputs():
    """Tiles write it while others read; calls that need none take whatever they are given."""
    desc = ad(rank=16, d_in=64)
    need = U.umem_adapter_workspace_size(desc, 5000)[1]
    assert need > 0 and U.umem_adapter_workspace_size(desc, 8)[1] == 0
    names = ["x", "ids", "a", "b", "scale", "base", "out"]
    base = {k: at(i) for i, k in enumerate(names)}
    for k in names:
        for ws in (base[k], base[k] + 256 if k in ("x", "ids", "base", "out") else base[k], base[k] - need // 256 * 256 + 256):
            assert U.umem_adapter_add(desc, 5000, *base.values(), ws, need, 0) == ARG, k


def test_tensors_of_another_device_are_refused(monkeypatch):
    """Without a stream the current device's is taken: a tensor that lives elsewhere is an error, not a launch."""
    class Elsewhere:
        is_cuda = True
        is_contiguous = staticmethod(lambda: True)
        data_ptr = staticmethod(lambda: at(0))
        get_device = staticmethod(lambda: 1)

    monkeypatch.setattr(U, "_get_device", lambda: 0)
    monkeypatch.setattr(U, "_raw_stream", lambda device: 0)
    x = Elsewhere()
    calls = [lambda s: U.umem_block_in(bd(), 0, x, x, x, x, s), lambda s: U.umem_block_out(bd(), 0, x, x, None, x, x, x, stream=s),
             lambda s: U.umem_block_in_backward(bd(), 0, x, x, x, x, x, x, x, 0, x, 0, s),
             lambda s: U.umem_block_out_backward(bd(), 0, x, None, x, x, x, x, x, None, x, x, 0, x, 0, s),
             lambda s: U.umem_grad_norm(-1, None, x, None, x, 0, s), lambda s: U.umem_grad_clip(-1, None, 1.0, x, s),
             lambda s: U.umem_adapter_add(ad(), 0, x, x, x, x, x, x, x, stream=s)]
    for call in calls:
        with pytest.raises(ValueError):
            call(None)
        assert call(7) in (OK, ARG)                                     # a stream given: the caller's word


def never_falls(size, tokens=(*range(0, 5000), *range(5000, 40000, 61), 1 << 16, 1 << 18, (1 << 18) + 1)):
    sizes = [size(T) for T in tokens]
    assert all(st == OK for st, _ in sizes)
    assert all(a[1] <= b[1] for a, b in zip(sizes, sizes[1:]))


@pytest.mark.parametrize("q", [(64, 3, 2, 32, 0), (2048, 5, 2, 224, 0), (1024, 3, 2, 64, 1), (768, 3, 4, 128, 0), (4096, 1, 1, 64, 1)])
def test_query_workspaces_never_fall_with_the_tokens(q):
    """Also where the query linear is split over d_model, in more ways for fewer tokens."""
    qd = U.umem_query_desc(*q, 1e-5)
    never_falls(lambda T: U.umem_query_workspace_size(qd, T, 1))
    a = ad(d_in=q[0], d_out=(2 - q[4]) * q[2] * q[3], xtype=1, rank=32)
    never_falls(lambda T: U.umem_query_adapted_workspace_size(qd, a, 1, T))


@pytest.mark.parametrize("shape", [(1, 1024, 1024, 0), (4, 512, 1024, 2048), (1, 2048, 0, 2048), (1, 4096, 0, 1024), (1, 1 << 18, 0, 128),
                                   (4, 896, 896, 2048), (6, 512, 336, 1024), (16, 2048, 256, 0)])
def test_projection_workspaces_never_fall_with_the_tokens(shape):
    never_falls(lambda T: U.umem_project_workspace_size(T, *shape))


@pytest.mark.parametrize("n,dv,dv_virt,d_out", [(16, 128, 512, 2048), (16, 512, 0, 2048), (512, 1024, 0, 512), (64, 512, 1024, 512)])
def test_layer_workspaces_never_fall_with_the_tokens(n, dv, dv_virt, d_out):
    d = U.umem_desc(2, 256, n, 2, 16, 16, 1, 0, n * n, dv, 1, 1, dv_virt, d_out, 1)
    never_falls(lambda T: U.umem_workspace_size(d, T))


@pytest.mark.parametrize("bag,dv", [(1, 8), (32, 512), (64, 512), (84, 448)])
def test_backward_workspaces_never_fall_with_the_tokens(bag, dv):
    """Also past 2^19 entries, from where the sort takes larger tiles."""
    tokens = range(0, (1 << 20) // bag, max(1, 32 // bag))
    never_falls(lambda T: U.umem_gather_backward_workspace_size(T, bag, dv), tokens)
    d = U.umem_desc(2, 256, 64, 2, 16, 16, 1, 0, 64 * 64, 128, 1, 1, 0, 0, 1)
    never_falls(lambda T: U.umem_score_backward_workspace_size(d, T), range(0, 30000, 5))


def test_adapted_query_refusals():
    qd = U.umem_query_desc(64, 3, 2, 32, 0, 1e-5)                        # 2 axes of 2 heads of 32: 128 outputs
    good = dict(xtype=1)
    st, need = U.umem_query_adapted_workspace_size(qd, ad(**good), 4, 5)
    assert st == OK and need >= U.umem_query_workspace_size(qd, 4, 5)[1]
    assert U.umem_query_adapted_workspace_size(qd, ad(**good), 0, 5)[0] == OK
    for kw, want in ((dict(d_in=72), ARG), (dict(d_out=64), ARG), (dict(xtype=0), ARG), (dict(otype=1), ARG), (dict(n=0), ARG),
                     (dict(rank=12), UNS)):
        assert U.umem_query_adapted_workspace_size(qd, ad(**{**good, **kw}), 4, 5)[0] == want, kw
    assert U.umem_query_adapted_workspace_size(U.umem_query_desc(60, 3, 2, 32, 0, 1e-5), ad(**good), 4, 5)[0] == UNS
    assert U.umem_query_adapted_workspace_size(qd, ad(**good), -1, 5)[0] == ARG
    names = ["x", "hist", "conv", "wq", "ids", "a", "b", "scale", "gamma", "beta", "q_row", "q_col"]
    base = {k: at(i) for i, k in enumerate(names)}

    def call(ws=at(20), n=need, B=4, **kw):
        return U.umem_query_adapted(qd, ad(**good), B, 5, *{**base, **kw}.values(), ws, n, 0)

    for k in ("x", "conv", "wq", "ids", "a", "b", "gamma", "beta", "q_row", "q_col"):
        assert call(**{k: None}) == ARG, k
    for k in names:
        assert call(**{k: base[k] + 2}) == ARG, k
    assert call(ws=None) == WS and call(ws=at(20) + 8) == WS and call(n=need - 1) == WS
    assert call(B=0, x=None) == OK and call(B=-1) == ARG


def test_adapted_query_outputs_are_apart():
    """The queries and the scratch, from what is read and from each other."""
    qd = U.umem_query_desc(64, 3, 2, 32, 0, 1e-5)
    desc = ad(xtype=1)
    need = U.umem_query_adapted_workspace_size(qd, desc, 4, 5)[1]
    names = ["x", "hist", "conv", "wq", "ids", "a", "b", "scale", "gamma", "beta", "q_row", "q_col"]
    base = {k: at(i) for i, k in enumerate(names)}
    sizes = dict(x=4 * 5 * 64 * 4, hist=4 * 2 * 64 * 4, conv=3 * 64 * 4, wq=128 * 64 * 2, ids=20 * 4, a=4 * 16 * 64 * 2, b=4 * 128 * 16 * 2,
                 scale=16, gamma=512, beta=512, q_row=20 * 64 * 4, q_col=20 * 64 * 4)

    def call(ws=at(20), **kw):
        return U.umem_query_adapted(qd, desc, 4, 5, *{**base, **kw}.values(), ws, need, 0)

    for k in names:
        for out in ("q_row", "q_col"):
            if out == k:
                continue
            for a in (base[k], base[k] + sizes[k] - 4, base[k] - sizes[out] + 4):
                assert call(**{out: a}) == ARG, (k, out)
        for a in (base[k], base[k] + sizes[k] - 16, base[k] - need + 16):
            assert call(ws=a) == ARG, k
