"""The oracle of layer norm, the gated delta rule and beam search (oracle/layer.py, oracle/search.py):
gradients against differences of the forward formulas, known answers, and that the bounds and
tolerances of the GPU tests tell a wrong result from a right one."""
import numpy as np
import pytest

from oracle import layer as ol
from oracle import search as os_


def _differences(f, x, step=1e-5):
    g = np.zeros_like(x)
    for i in np.ndindex(x.shape):
        keep = x[i]
        x[i] = keep + step
        up = f()
        x[i] = keep - step
        g[i] = (up - f()) / (2 * step)
        x[i] = keep
    return g


def test_layer_norm_gradients_are_differences():
    rng = np.random.default_rng(1)
    x, w, b, dy = rng.standard_normal((3, 7)), rng.standard_normal(7), rng.standard_normal(7), rng.standard_normal((3, 7))
    r = ol.layer_norm_backward(x, w, dy)
    f = lambda: (ol.layer_norm(x, w, b)["y"] * dy).sum()
    # central differences: step^2 times third derivatives of order 10, and 2^-52 / step
    for name, leaf in (("dx", x), ("dw", w), ("db", b)):
        assert np.abs(_differences(f, leaf) - r[name]).max() < 1e-8, name


def _delta_case(lens, Hk, H, Dk, Dv, seed, full=True):
    rng = np.random.default_rng(seed)
    T, n = sum(lens), len(lens)
    unit = lambda a: a / np.linalg.norm(a, axis=-1, keepdims=True)
    return dict(q=unit(rng.standard_normal((T, Hk, Dk))), k=unit(rng.standard_normal((T, Hk, Dk))),
                v=rng.standard_normal((T, H, Dv)), g=-rng.exponential(0.3, (T, H)), beta=rng.uniform(0.1, 1, (T, H)),
                offs=np.concatenate([[0], np.cumsum(lens)]),
                state=rng.standard_normal((n, H, Dk, Dv)) if full else None)


def test_delta_rule_gradients_are_differences():
    a = _delta_case([4, 0, 3], 1, 2, 3, 2, 2)
    rng = np.random.default_rng(3)
    do, dend = rng.standard_normal(a["v"].shape), rng.standard_normal(a["state"].shape)
    r = ol.delta_rule_backward(do=do, dend=dend, **a)

    def f():
        o = ol.delta_rule(**a)
        return (o["o"] * do).sum() + (o["end"] * dend).sum()

    for name in ("q", "k", "v", "g", "beta", "state"):
        assert np.abs(_differences(f, a[name]) - r["d" + name]).max() < 1e-7, name


def test_delta_rule_known_answers():
    """One key written twice holds the second value (beta 1, no decay); a decay of 0 forgets."""
    k = np.zeros((3, 1, 8))
    k[:, 0, 2] = 1.0
    v = np.arange(24.0).reshape(3, 1, 8)
    one, zero = np.ones((3, 1)), np.zeros((3, 1))
    r = ol.delta_rule(k, k, v, zero, one, [0, 3], scale=1.0)
    assert np.array_equal(r["o"], v) and np.array_equal(r["end"][0, 0, 2], v[2, 0])
    r = ol.delta_rule(k, k, v, np.full((3, 1), -np.inf), 0.5 * one, [0, 3], scale=1.0)
    assert np.array_equal(r["o"], 0.5 * v)


def test_beam_known_answers():
    x = np.log(np.array([[0.5, 0.25, 0.25], [0.9, 0.1, 0.0001], [1.0, 1.0, 1.0], [9.0, 1.0, 1.0]]))
    r = os_.beam_select(x, np.array([[0.0, -10.0], [-1.0, -1.0]]), 4, ended=np.array([[-1, -1], [-1, 7]]))
    assert r["parent"].tolist() == [[0, 0, 0, 1], [3, 2, 2, 2]]
    assert r["token"].tolist() == [[0, 1, 2, 0], [7, 0, 1, 2]]
    assert np.allclose(r["score"][0, :3], np.log([0.5, 0.25, 0.25])) and r["score"][1, 0] == -1.0
    pool = np.arange(6.0)
    new, pools = os_.beam_reorder(np.array([[1, 1, 1, 3]]), np.array([[5, 2, 0, 4]]), 6, [pool])
    assert new.tolist() == [[2, 5, 0, 4]] and pools[0].tolist() == [2, 1, 2, 3, 4, 2]


def test_layer_norm_bounds_refuse_mistakes():
    rng = np.random.default_rng(4)
    for C in (1, 7, 300):
        x, w, b, dy = rng.standard_normal((20, C)) + 3.0, rng.standard_normal(C), rng.standard_normal(C), rng.standard_normal((20, C))
        r, g = ol.layer_norm(x, w, b), ol.layer_norm_backward(x, w, dy)
        for wrong in (ol.layer_norm(x, None, b)["y"] if C > 1 else 0 * r["y"], ol.layer_norm(x, w, None)["y"], -r["y"]):
            assert (np.abs(wrong - r["y"]) > r["bound"] + 2.0 ** -8 * np.abs(r["y"])).any()
        if C > 1:
            for name, wrong in (("dx", ol.layer_norm_backward(x, None, dy)["dx"]), ("dw", -g["dw"]), ("db", 0 * g["db"]),
                                ("dx", g["dx"] + 0.05 * np.abs(g["dx"]).mean())):
                assert (np.abs(wrong - g[name]) > g["bound"][name] + 2.0 ** -8 * np.abs(g[name])).mean() > 0.3, name


def test_delta_tolerance_refuses_mistakes():
    """What the GPU tests compare per head by 2-norm: a missing term is outside by far."""
    from tests.test_gpu_delta import GRADS, head_errors, tolerance
    a = _delta_case([70, 9], 1, 2, 16, 8, 5)
    rng = np.random.default_rng(6)
    do, dend = rng.standard_normal(a["v"].shape), rng.standard_normal(a["state"].shape)
    r = ol.delta_rule_backward(do=do, dend=dend, **a)
    f = ol.delta_rule(**a)
    tol = tolerance(16, [70, 9]) + 2.0 ** -8
    no_state = ol.delta_rule(**dict(a, state=None))
    cut = ol.delta_rule(**dict(a, offs=np.array([0, 64, 70, 79]), state=np.concatenate([a["state"][:1], 0 * a["state"][:1], a["state"][1:]])))
    assert head_errors(no_state["o"], f["o"]).min() > tol and head_errors(cut["o"], f["o"]).min() > tol
    grads = lambda **kw: ol.delta_rule_backward(**{**a, "do": do, "dend": dend, **kw})
    wrong = [(grads(dend=None), ("dk", "dv", "dg", "dbeta", "dstate")), (grads(state=None), ("dq", "dk", "dg", "dbeta")),
             (grads(g=0 * a["g"]), GRADS)]
    for x, names in wrong:
        for name in names:
            assert head_errors(x[name], r[name]).min() > tol, name
