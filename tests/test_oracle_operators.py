"""Pins of the oracles of the sequence and logit operators: closed forms, and
gradients against differences of the loss."""
import numpy as np
import pytest

from oracle import logits as ol
from oracle import sequence as osq


def _scan_inputs(rng, lens, E, N):
    T = sum(lens)
    offs = np.concatenate([[0], np.cumsum(lens)])
    r = rng.standard_normal
    return dict(u=r((T, E)), dt=r((T, E)) - 1, A_log=0.3 * r((E, N)), B=r((T, N)), C=r((T, N)), offs=offs, D=r(E),
                z=r((T, E)), b_dt=r(E), state=r((len(lens), E, N)))


def test_scan_is_the_explicit_convolution():
    rng = np.random.default_rng(0)
    a = _scan_inputs(rng, [6, 0, 1], 3, 4)
    o = osq.scan(**a)
    d, A = osq.softplus(a["dt"] + a["b_dt"]), -np.exp(a["A_log"])
    for i in range(3):
        for t in range(a["offs"][i], a["offs"][i + 1]):
            lo = a["offs"][i]
            s = a["state"][i] * np.exp(A * d[lo:t + 1].sum(0)[:, None])
            for k in range(lo, t + 1):
                s = s + np.exp(A * d[k + 1:t + 1].sum(0)[:, None]) * (d[k] * a["u"][k])[:, None] * a["B"][k]
            y = ((s * a["C"][t]).sum(1) + a["D"] * a["u"][t]) * a["z"][t] * osq.sigmoid(a["z"][t])
            np.testing.assert_allclose(o["y"][t], y, rtol=1e-11, atol=1e-12)
    np.testing.assert_array_equal(o["end"][1], a["state"][1])  # an empty sequence passes its state on


def test_scan_in_pieces_is_the_whole():
    rng = np.random.default_rng(1)
    a = _scan_inputs(rng, [9], 3, 4)
    whole = osq.scan(**a)
    st, ys = a["state"], []
    for lo, hi in [(0, 1), (1, 6), (6, 9)]:
        part = {k: v[lo:hi] if k in ("u", "dt", "B", "C", "z") else v for k, v in a.items()}
        part.update(offs=np.array([0, hi - lo]), state=st)
        o = osq.scan(**part)
        st = o["end"]
        ys.append(o["y"])
    np.testing.assert_allclose(np.concatenate(ys), whole["y"], rtol=1e-12, atol=1e-13)
    np.testing.assert_allclose(st, whole["end"], rtol=1e-12, atol=1e-13)


@pytest.mark.parametrize("gate", [True, False])
def test_scan_gradients_are_differences(gate):
    rng = np.random.default_rng(2)
    a = _scan_inputs(rng, [4, 0, 3], 2, 3)
    if not gate:
        a["z"] = None
    dy, dend = rng.standard_normal(a["u"].shape), rng.standard_normal(a["state"].shape)

    def loss(**kw):
        o = osq.scan(**dict(a, **kw))
        return (o["y"] * dy).sum() + (o["end"] * dend).sum()

    b = {k: v for k, v in a.items() if k != "offs"}
    g = osq.scan_backward(**b, dy=dy, offs=a["offs"], dend=dend)
    names = dict(du="u", ddt="dt", dB="B", dC="C", dA_log="A_log", dD="D", db_dt="b_dt", dstate="state")
    if gate:
        names["dz"] = "z"
    for out, name in names.items():
        v = a[name]
        for i in np.ndindex(v.shape):
            e = np.zeros_like(v)
            e[i] = 1e-6
            fd = (loss(**{name: v + e}) - loss(**{name: v - e})) / 2e-6
            assert abs(fd - g[out][i]) < 1e-7 * (1 + abs(fd)), (out, i)


@pytest.mark.parametrize("K", [1, 2, 4])
def test_conv_gradients_are_differences(K):
    rng = np.random.default_rng(3)
    lens, E = [5, 0, 1, 3], 2
    offs = np.concatenate([[0], np.cumsum(lens)])
    r = rng.standard_normal
    a = dict(x=r((9, E)), w=r((E, K)), b=r(E), state=r((4, K - 1, E)))
    du, dend = r((9, E)), r((4, K - 1, E))

    def loss(**kw):
        o = osq.conv(offs=offs, **dict(a, **kw))
        return (o["u"] * du).sum() + (o["end"] * dend).sum()

    g = osq.conv_backward(du=du, offs=offs, dend=dend, **a)
    for out, name in dict(dx="x", dw="w", db="b", dstate="state").items():
        v = a[name]
        for i in np.ndindex(v.shape):
            e = np.zeros_like(v)
            e[i] = 1e-6
            fd = (loss(**{name: v + e}) - loss(**{name: v - e})) / 2e-6
            assert abs(fd - g[out][i]) < 1e-7 * (1 + abs(fd)), (out, i)


def test_conv_in_pieces_is_the_whole():
    rng = np.random.default_rng(4)
    x, w, b = rng.standard_normal((7, 3)), rng.standard_normal((3, 4)), rng.standard_normal(3)
    whole = osq.conv(x, w, b, np.array([0, 7]))
    st, us = None, []
    for lo, hi in [(0, 1), (1, 3), (3, 7)]:
        o = osq.conv(x[lo:hi], w, b, np.array([0, hi - lo]), st)
        st = o["end"]
        us.append(o["u"])
    np.testing.assert_allclose(np.concatenate(us), whole["u"], rtol=1e-13)
    np.testing.assert_array_equal(st[0], x[4:])


def test_logprobs_closed_forms():
    o = ol.logprobs([np.zeros(8), np.array([np.log(3.0), 0.0, -np.inf]), np.array([]), np.full(3, -np.inf),
                     np.array([1.0, np.nan, 1.0])], np.array([2, 0, 0, 1, 1]), 3)
    np.testing.assert_allclose(o["entropy"], [np.log(8), -(0.75 * np.log(0.75) + 0.25 * np.log(0.25)), 0, 0,
                                              np.log(2)])
    np.testing.assert_allclose(o["logp"][:2], [-np.log(8), np.log(0.75)])
    assert np.isnan(o["logp"][2]) and o["logp"][3] == -np.inf and o["logp"][4] == -np.inf
    np.testing.assert_array_equal(o["top"], [[0, 1, 2], [0, 1, 2], [-1, -1, -1], [0, 1, 2], [0, 2, 1]])


def test_distill_gradient_is_differences():
    rng = np.random.default_rng(5)
    rows = [rng.standard_normal(6), rng.standard_normal(4), rng.standard_normal(3)]
    top = np.array([[1, 4, 1], [3, -1, 9], [-1, -1, -1]])  # an entry twice, entries outside, none
    teacher, w = rng.standard_normal((3, 3)), np.array([0.5, 2.0, 1.0])
    g = ol.distill(rows, top, teacher, w, 1.7)
    assert g["loss"][2] == 0 and not g["grad"][2].any()
    for r, x in enumerate(rows):
        for v in range(x.size):
            e = np.zeros(x.size)
            e[v] = 1e-6
            f = [ol.distill([x + s * e], top[r:r + 1], teacher[r:r + 1], None, 1.7)["loss"][0] for s in (1, -1)]
            assert abs((f[0] - f[1]) / 2e-6 * w[r] - g["grad"][r][v]) < 1e-8


def test_distill_is_zero_where_the_student_agrees():
    x = np.array([0.3, -1.0, 2.0])
    g = ol.distill([x], np.array([[2, 0, 1]]), np.array([[2.0, 0.3, -1.0]]) + 5.0)
    np.testing.assert_allclose(g["loss"], 0, atol=1e-15)
    np.testing.assert_allclose(g["grad"][0], 0, atol=1e-15)
