"""Refusals of the token-row, head and orthogonalised-update entry points, and their workspaces' sizes, on the host:
every call below fails validation, sizes a workspace or has nothing to do, so no kernel is launched."""
import pytest

import paper_2411_12364_amd as U

OK, ARG, UNS, WS = U.UMEM_OK, U.UMEM_ERR_INVALID_ARG, U.UMEM_ERR_UNSUPPORTED, U.UMEM_ERR_WORKSPACE
MB = 1 << 20
INF, NAN = float("inf"), float("nan")


def at(i):
    """Addresses 64 MiB apart, never dereferenced."""
    return (i + 1) * 64 * MB


def ed(**kw):
    return U.umem_embed_desc(*{**dict(vocab=100, d=64, wtype=0, otype=0, scale=1.0), **kw}.values())


def hd(**kw):
    return U.umem_head_desc(*{**dict(vocab=100, d=64, xtype=0, gtype=0, scale=1.0), **kw}.values())


def od(**kw):
    base = dict(n=2, rows=32, cols=48, gtype=0, otype=0, steps=5, a=3.4445, b=-4.775, c=2.0315, eps=1e-7, decay=0.0,
                scale=1.0)
    return U.umem_orth_desc(*{**base, **kw}.values())


SCALES = [(dict(scale=NAN), ARG), (dict(scale=INF), ARG), (dict(scale=0.0), OK), (dict(scale=-2.0), OK)]


@pytest.mark.parametrize("kw,want", SCALES + [
    (dict(), OK), (dict(vocab=0), ARG), (dict(vocab=2 ** 31 - 1), OK), (dict(d=0), ARG), (dict(d=16384), OK),
    (dict(d=16385), UNS), (dict(d=1), OK), (dict(wtype=2), ARG), (dict(wtype=-1), ARG), (dict(otype=2), ARG)])
def test_embed_descriptor(kw, want):
    st, n = U.umem_embed_backward_workspace_size(ed(**kw), 8)
    assert st == want and (n > 0) == (want == OK)
    assert U.umem_embed(ed(**kw), 0, None, None, None, 0) == want
    assert U.umem_embed_backward(ed(**kw), 0, None, None, None, None, 0, 0) == want
    assert U.umem_embed_backward_rows(ed(**kw), 0, None, None, None, None, None, None, 0, 0) == want


def test_embed_tokens():
    for T, want in ((-1, ARG), (0, OK), (1 << 20, OK), ((1 << 20) + 1, UNS)):
        assert U.umem_embed_backward_workspace_size(ed(), T)[0] == want
        if want != OK:
            assert U.umem_embed(ed(), T, at(0), at(1), at(2), 0) == want
            assert U.umem_embed_backward(ed(), T, at(0), at(1), at(2), at(3), 1 << 40, 0) == want
    assert U.umem_embed_backward_workspace_size(ed(), 0) == (OK, 0)


def test_embed_refusals():
    base = dict(table=at(0), ids=at(1), out=at(2))
    call = lambda desc=ed(), T=8, **kw: U.umem_embed(desc, T, *{**base, **kw}.values(), 0)   # noqa: E731
    for k in base:
        assert call(**{k: None}) == ARG and call(**{k: base[k] + 2}) == ARG, k
    b16 = ed(wtype=1, otype=1)
    assert call(desc=b16, table=at(0) + 1) == ARG and call(desc=b16, out=at(2) + 1) == ARG
    assert call(out=at(0)) == ARG and call(out=at(0) + 64 * 4 * 99) == ARG and call(out=at(1)) == ARG
    assert call(out=at(1) - 8 * 64 * 4 + 4) == ARG


def test_embed_backward_refusals():
    need = U.umem_embed_backward_workspace_size(ed(), 8)[1]
    base = dict(ids=at(0), dout=at(1), dtable=at(2))

    def call(desc=ed(), ws=at(9), n=need, **kw):
        return U.umem_embed_backward(desc, 8, *{**base, **kw}.values(), ws, n, 0)

    for k in base:
        assert call(**{k: None}) == ARG and call(**{k: base[k] + 2}) == ARG, k
    assert call(desc=ed(otype=1), dout=at(1) + 1) == ARG
    assert call(ws=None) == WS and call(ws=at(9) + 8) == WS and call(n=need - 1) == WS
    assert call(dtable=at(0)) == ARG and call(dtable=at(1)) == ARG and call(dtable=at(9)) == ARG
    assert call(ws=at(0)) == ARG and call(ws=at(1)) == ARG

    base = dict(ids=at(0), dout=at(1), rows=at(2), d_rows=at(3), n_rows=at(4))

    def call(desc=ed(), ws=at(9), n=need, **kw):      # noqa: F811
        return U.umem_embed_backward_rows(desc, 8, *{**base, **kw}.values(), ws, n, 0)

    for k in base:
        assert call(**{k: None}) == ARG and call(**{k: base[k] + 2}) == ARG, k
    assert call(ws=None) == WS and call(n=0) == WS
    outs = ["rows", "d_rows", "n_rows"]
    for i, k in enumerate(outs):
        for other in ["ids", "dout"] + outs[:i] + outs[i + 1:]:
            assert call(**{k: base[other]}) == ARG, (k, other)
        assert call(**{k: at(9)}) == ARG


@pytest.mark.parametrize("kw,want", SCALES + [
    (dict(), OK), (dict(vocab=0), ARG), (dict(vocab=1 << 20), OK), (dict(vocab=(1 << 20) + 1), UNS), (dict(d=0), ARG),
    (dict(d=60), UNS), (dict(d=8), OK), (dict(d=16384), OK), (dict(d=16392), UNS), (dict(xtype=2), ARG),
    (dict(gtype=-1), ARG), (dict(vocab=1), OK)])
def test_head_descriptor(kw, want):
    for size in (U.umem_head_loss_workspace_size, U.umem_head_backward_workspace_size):
        st, n = size(hd(**kw), 8)
        assert st == want and (n > 0) == (want == OK)
        assert size(hd(**kw), 0) == (want, 0)
        assert size(hd(), -1) == (ARG, 0) and size(hd(), (1 << 20) + 1) == (UNS, 0)
    assert U.umem_head_loss(hd(**kw), 0, *[None] * 6, 0, 0) == want
    assert U.umem_head_backward(hd(**kw), 0, *[None] * 7, 0, None, 0, 0) == want


def test_head_loss_refusals():
    need = U.umem_head_loss_workspace_size(hd(), 8)[1]
    base = dict(x=at(0), w=at(1), targets=at(2), loss=at(3), lse=at(4))

    def call(ws=at(9), n=need, T=8, **kw):
        return U.umem_head_loss(hd(), T, *{**base, **kw}.values(), ws, n, 0)

    for k in base:
        assert call(**{k: None}) == ARG and call(**{k: base[k] + 2}) == ARG, k
    assert call(x=at(0) + 8) == ARG and call(w=at(1) + 8) == ARG
    assert call(ws=None) == WS and call(ws=at(9) + 128) == WS and call(n=need - 1) == WS
    for k in ("x", "w", "targets"):
        assert call(loss=base[k]) == ARG and call(lse=base[k]) == ARG and call(ws=base[k]) == ARG, k
    assert call(loss=at(4) + 4) == ARG and call(loss=at(9)) == ARG and call(T=-1) == ARG


def test_head_backward_refusals():
    need = U.umem_head_backward_workspace_size(hd(), 8)[1]
    base = dict(x=at(0), w=at(1), targets=at(2), lse=at(3), dloss=at(4), dx=at(5), dw=at(6))

    def call(desc=hd(), acc=0, ws=at(9), n=need, T=8, **kw):
        return U.umem_head_backward(desc, T, *{**base, **kw}.values(), acc, ws, n, 0)

    for k in base:
        assert k == "dloss" or call(**{k: None}) == ARG, k
        assert call(**{k: base[k] + 2}) == ARG, k
    for k in ("x", "w", "dx", "dw"):
        assert call(**{k: base[k] + 8}) == ARG, k
    assert call(acc=2) == ARG and call(acc=-1) == ARG and call(T=0, acc=2) == ARG
    assert call(desc=hd(gtype=1), acc=1) == ARG and call(desc=hd(gtype=1), acc=1, T=0) == ARG
    assert call(ws=None) == WS and call(ws=at(9) + 16) == WS and call(n=need - 1) == WS
    for k in ("x", "w", "targets", "lse", "dloss"):
        assert call(dx=base[k]) == ARG and call(dw=base[k]) == ARG and call(ws=base[k]) == ARG, k
    assert call(dx=at(6)) == ARG and call(dx=at(9)) == ARG and call(dw=at(9)) == ARG


@pytest.mark.parametrize("kw,want", SCALES + [
    (dict(), OK), (dict(n=0), ARG), (dict(n=65535, rows=1, cols=1), OK), (dict(n=65536, rows=1, cols=1), UNS),
    (dict(rows=0), ARG), (dict(cols=-1), ARG), (dict(rows=65536), OK), (dict(cols=65537), UNS),
    (dict(rows=65536, cols=65536), OK), (dict(n=3, rows=65536, cols=65536), UNS), (dict(gtype=2), ARG),
    (dict(otype=-1), ARG), (dict(steps=0), ARG), (dict(steps=16), OK), (dict(steps=17), UNS), (dict(a=NAN), ARG),
    (dict(b=INF), ARG), (dict(c=-INF), ARG), (dict(eps=-1e-9), ARG), (dict(eps=NAN), ARG), (dict(eps=0.0), OK),
    (dict(decay=NAN), ARG), (dict(decay=0.99), OK)])
def test_orth_descriptor(kw, want):
    st, n = U.umem_orthogonalize_workspace_size(od(**kw))
    assert st == want and (n > 0) == (want == OK)
    if want != OK:
        assert U.umem_orthogonalize(od(**kw), at(0), at(1), at(2), 1 << 50, 0) == want


def test_orth_refusals():
    need = U.umem_orthogonalize_workspace_size(od())[1]
    call = lambda desc=od(), g=at(0), out=at(1), ws=at(2), n=need: U.umem_orthogonalize(desc, g, out, ws, n, 0)   # noqa: E731
    assert call(g=None) == ARG and call(out=None) == ARG and call(g=at(0) + 2) == ARG and call(out=at(1) + 1) == ARG
    assert call(ws=None) == WS and call(ws=at(2) + 64) == WS and call(n=need - 1) == WS
    assert call(out=at(0) + 4) == ARG and call(out=at(2)) == ARG and call(g=at(2)) == ARG
    assert call(desc=od(gtype=1), out=at(0)) == ARG                     # the same place in another type


def sizes(lo, hi, n=60):
    step = (hi / lo) ** (1 / n)
    got, x = set(), float(lo)
    while x <= hi:
        got |= {int(x), int(x) + 1, int(x) // 64 * 64 + 1, int(x) // 256 * 256 + 1}
        x *= step
    return sorted(v for v in got if lo <= v <= hi)


@pytest.mark.parametrize("vocab,d,xtype,gtype", [(1, 8, 0, 0), (100, 64, 1, 0), (129, 64, 1, 1), (50000, 2048, 1, 0),
                                                  (32003, 1024, 0, 1), (1 << 20, 16384, 0, 0)])
def test_workspaces_never_fall_as_the_tokens_grow(vocab, d, xtype, gtype):
    Ts = sizes(1, 1 << 20)
    for size, desc in ((U.umem_head_loss_workspace_size, hd(vocab=vocab, d=d, xtype=xtype, gtype=gtype)),
                       (U.umem_head_backward_workspace_size, hd(vocab=vocab, d=d, xtype=xtype, gtype=gtype)),
                       (U.umem_embed_backward_workspace_size, ed(vocab=vocab, d=d))):
        got = [size(desc, T)[1] for T in Ts]
        assert got == sorted(got)
