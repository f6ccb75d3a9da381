"""The oracle of the operators around the layer against things other than itself: hand-worked values,
central differences along random directions, loops; and planted mistakes that those have to catch."""
import numpy as np
import pytest

import oracle.block_oracle as B

EPS = 1e-5


def test_hand_worked_norms():
    x = np.array([[1.0, 3.0], [3.0, 4.0]])
    np.testing.assert_allclose(B.standardise(x, "layer", 0.0)[0], [[-1, 1], [-1, 1]])
    xh, r = B.standardise(x, "rms", 0.0)
    np.testing.assert_allclose(r[:, 0], [1 / np.sqrt(5.0), 1 / np.sqrt(12.5)])
    np.testing.assert_allclose(xh[1], [3 / np.sqrt(12.5), 4 / np.sqrt(12.5)])
    np.testing.assert_allclose(B.block_in(x, "layer", [2.0, 3.0], [10.0, 20.0], 0.0), [[8, 23], [8, 23]])
    # a row without spread: zeros under a positive eps
    assert (B.standardise(np.full((1, 7), 2.5), "layer", EPS)[0] == 0).all()


def test_hand_worked_exit():
    h, y = np.array([[1.0, 2.0]]), np.array([[10.0, 20.0]])
    args = ("none", None, None, EPS, 0.5, 2.0)
    np.testing.assert_allclose(B.block_out(h, y, None, "none", "linear", *args), [[20.5, 41.0]])
    np.testing.assert_allclose(B.block_out(h, y, [0.0, 0.1], "channel", "linear", *args), [[0.5, 5.0]])
    np.testing.assert_allclose(B.block_out(h, y, [0.0], "token", "sigmoid", *args), [[10.5, 21.0]])
    np.testing.assert_allclose(B.block_out(h, y, [[1.0, -1.0]], "full", "linear", *args), [[20.5, -39.0]])


def _difference(f, at, direction, step=1e-6):
    return (f(at + step * direction) - f(at - step * direction)) / (2 * step)


@pytest.mark.parametrize("kind", ["layer", "rms"])
def test_entry_gradients_against_differences(kind):
    rng = np.random.default_rng(1)
    h, gamma, beta = rng.normal(size=(4, 9)), 1 + 0.3 * rng.normal(size=9), rng.normal(size=9)
    dn, dres = rng.normal(size=(4, 9)), rng.normal(size=(4, 9))
    dh, dg, db = B.block_in_backward(h, kind, gamma, EPS, dn, dres)
    loss = lambda h, g, b: (B.block_in(h, kind, g, b, EPS) * dn).sum() + (h * dres).sum()   # noqa: E731
    for grad, at, f in ((dh, h, lambda v: loss(v, gamma, beta)), (dg, gamma, lambda v: loss(h, v, beta)),
                        (db, beta, lambda v: loss(h, gamma, v))):
        u = rng.normal(size=at.shape)
        np.testing.assert_allclose((grad * u).sum(), _difference(f, at, u), rtol=1e-6)


def exit_errors(backward, kind, gate_kind, act):
    """The largest relative error of a backward's gradients against central differences."""
    rng = np.random.default_rng(2)
    T, d = 5, 8
    h, y, up = rng.normal(size=(T, d)), 0.3 + rng.normal(size=(T, d)), rng.normal(size=(T, d))
    gate = None if gate_kind == "none" else rng.normal(size={"channel": d, "token": T, "full": (T, d)}[gate_kind])
    gamma, beta = (None, None) if kind == "none" else (1 + 0.3 * rng.normal(size=d), rng.normal(size=d))
    a, s = 0.7, 1.6
    got = backward(y, gate, gate_kind, act, kind, gamma, beta, EPS, a, s, up)
    loss = lambda h, y, z, g, b: (B.block_out(h, y, z, gate_kind, act, kind, g, b, EPS, a, s) * up).sum()   # noqa: E731
    worst = 0.0
    for name, at, f in (("dh", h, lambda v: loss(v, y, gate, gamma, beta)),
                        ("dy", y, lambda v: loss(h, v, gate, gamma, beta)),
                        ("dgate", gate, lambda v: loss(h, y, v, gamma, beta)),
                        ("dgamma", gamma, lambda v: loss(h, y, gate, v, beta)),
                        ("dbeta", beta, lambda v: loss(h, y, gate, gamma, v))):
        if at is None:
            assert got[name] is None or name in ("dgamma", "dbeta")
            continue
        u = rng.normal(size=at.shape)
        want = _difference(f, at, u)
        worst = max(worst, abs((got[name] * u).sum() - want) / max(abs(want), 1e-3))
    return worst


CASES = [(k, g, a) for k in ("none", "layer", "rms") for g in ("none", "channel", "token", "full")
         for a in ("linear", "sigmoid")]


@pytest.mark.parametrize("kind,gate_kind,act", CASES)
def test_exit_gradients_against_differences(kind, gate_kind, act):
    assert exit_errors(B.block_out_backward, kind, gate_kind, act) < 1e-6


def _mutant(change):
    def backward(y, gate, gate_kind, act, kind, gamma, beta, eps, a, s, up):
        return change(B.block_out_backward(y, gate, gate_kind, act, kind, gamma, beta, eps, a, s, up),
                      dict(y=y, gate=gate, gate_kind=gate_kind, act=act, kind=kind, gamma=gamma, beta=beta,
                           eps=eps, a=a, s=s, up=up))
    return backward


MUTANTS = {
    "residual scale lost": lambda g, k: {**g, "dh": np.array(k["up"])},
    "rms centred": lambda g, k: {**g, "dy": g["dy"] - g["dy"].mean(axis=1, keepdims=True)} if k["kind"] == "rms" else g,
    "gate's gradient without the shift": lambda g, k: {**g, "dgate": B.block_out_backward(
        k["y"], k["gate"], k["gate_kind"], k["act"], k["kind"], k["gamma"], None, k["eps"], k["a"], k["s"],
        k["up"])["dgate"]} if k["gate_kind"] == "channel" and k["kind"] != "none" else g,
    "slope of the sigmoid lost": lambda g, k: {**g, "dgate": B.block_out_backward(
        k["y"], 1 / (1 + np.exp(-np.asarray(k["gate"]))), k["gate_kind"], "linear", k["kind"], k["gamma"], k["beta"],
        k["eps"], k["a"], k["s"], k["up"])["dgate"]} if k["act"] == "sigmoid" and k["gate_kind"] != "none" else g,
    "out scale twice in gamma": lambda g, k: {**g, "dgamma": k["s"] * g["dgamma"]} if k["kind"] != "none" else g,
}


@pytest.mark.parametrize("name", MUTANTS)
def test_planted_mistakes_are_caught(name):
    assert max(exit_errors(_mutant(MUTANTS[name]), *case) for case in CASES) > 1e-3


def test_norm_and_clip_by_hand():
    assert B.global_norm([np.array([3.0]), np.array([[0.0, 4.0]])]) == 5.0
    assert B.global_norm([]) == 0.0
    assert B.clip_factor(5.0, 1.0) == 0.2 and B.clip_factor(0.5, 1.0) == 1.0 and B.clip_factor(1.0, 1.0) == 1.0
    assert np.isnan(B.clip_factor(float("nan"), 1.0)) and B.clip_factor(float("inf"), 1.0) == 0.0
    assert B.clip_factor(0.0, 0.0) == 1.0


def test_adapters_against_the_merged_weight():
    """B_i A_i as one matrix, added to a shared projection's weight."""
    rng = np.random.default_rng(3)
    a, b, scale = rng.normal(size=(3, 2, 6)), rng.normal(size=(3, 5, 2)), np.array([0.5, -1.0, 2.0])
    x, w, ids = rng.normal(size=(7, 6)), rng.normal(size=(5, 6)), [0, 2, -1, 1, 2, 3, 0]
    got = B.adapter_add(x, ids, a, b, scale, x @ w.T)
    for t, i in enumerate(ids):
        merged = w if not 0 <= i < 3 else w + scale[i] * (b[i] @ a[i])
        np.testing.assert_allclose(got[t], merged @ x[t], rtol=1e-12)
