"""The delta rule's products keep fp32's digits whatever the activations' type (tcl_delta_rule and its gradients): inputs whose
large terms cancel to some 2^-12 of themselves, so that what a product leaves out shows in a bf16 result too.

Each result here is a sum of few terms whose absolute values sum to M. Between the inputs and the sum lie at most 16
roundings (a term's factors and its decay, the sums over up to eight columns, the joining of the parts' sums, the scale), each
of at most 2^-24 of what it rounds, so of at most 2^-24 M: 2^-20 M in all, and half a step of the result's type. Of a
factor in two bf16 parts up to 2^-17 is left out, eight times as much."""
import numpy as np
import pytest
import torch

from oracle import layer as ol

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}
T, SMALL = 64, 2.0 ** -12


def _near(got, ref, M, dtype):
    got = got.double().cpu().numpy()
    off, tol = np.abs(got - ref), 2.0 ** -20 * M + HALF[dtype] * np.abs(ref)
    assert (np.abs(ref) <= 2.0 ** -10 * M).all()  # (the terms cancel)
    assert (off <= tol).all(), (float((off / tol).max()), int((off > tol).sum()), off.size)


def _inputs(D, Dv, rng):
    """Nothing written, nothing asked, no decay; values and their gradients in [1, 2], of eight bits."""
    b16 = lambda a: torch.from_numpy(a).bfloat16().double().numpy()
    one = lambda *shape: b16(1.0 + rng.random(shape))
    a = dict(q=np.zeros((T, 1, D)), k=np.zeros((T, 1, D)), v=one(T, 1, Dv), g=np.zeros((T, 1)), beta=np.zeros((T, 1)), scale=1.0)
    return a, one(T, 1, Dv)


def _gpu(a, dtype):
    x = {n: torch.from_numpy(a[n]).to(DT[dtype]).cuda() for n in ("q", "k", "v")}
    x.update({n: torch.from_numpy(a[n]).float().cuda() for n in ("g", "beta")})
    for n, t in x.items():  # (both sides compute with the same numbers)
        a[n] = t.double().cpu().numpy()
    return dict(x, scale=a["scale"], offs=torch.tensor([0, T], dtype=torch.int32, device="cuda"))


def _forward(a, dtype, state=None):
    from paper_2604_12891_amd import binding as tb
    x = _gpu(a, dtype)
    S = None if state is None else torch.from_numpy(state).float().cuda()
    a["state"] = None if S is None else S.double().cpu().numpy()
    return tb.delta_rule(**x, state=S)[:, 0], ol.delta_rule(**a, offs=[0, T])["o"][:, 0]


def _backward(a, do, dtype):
    from paper_2604_12891_amd import binding as tb
    x = _gpu(a, dtype)
    g = tb.delta_rule_backward(**x, do=torch.from_numpy(do).to(DT[dtype]).cuda())
    r = ol.delta_rule_backward(**a, do=do, offs=[0, T])
    return {n: (g[n][:, 0], r[n][:, 0]) for n in ("dq", "dk")}


both = pytest.mark.parametrize("dtype", ["f32", "bf16"])
wide = pytest.mark.parametrize("D", [64, 128])


@both
@wide
def test_answers_from_the_state(D, dtype):
    """o = S^T (e_a - e_b), rows of the state that are nearly the same."""
    rng = np.random.default_rng(0)
    a, _ = _inputs(D, 32, rng)
    S = (1.0 + rng.random((1, 1, 1, 32)) + SMALL * rng.random((1, 1, D, 32))).astype(np.float32)
    t = np.arange(T)
    a["q"][t, 0, t % D], a["q"][t, 0, (t + 5) % D] = 1.0, -1.0
    got, ref = _forward(a, dtype, S)
    _near(got, ref, 4.0, dtype)


@both
@wide
def test_answers_from_the_chunks_products(D, dtype):
    """o_t = scale d_t (v - (1 - 2^-8) v - 2^-8 (1 - 2^-8) v): the factors scale d_t have all of fp32's digits."""
    rng = np.random.default_rng(1)
    a, _ = _inputs(D, 32, rng)
    t = np.arange(T)
    a["k"][t, 0, t] = 1.0
    a["beta"][:3] = 1.0
    a["v"][1:3] = a["v"][0]
    a["scale"] = float(np.float32(0.7310586))
    a["g"][3:, 0] = -0.02 * rng.random(T - 3)
    a["q"][3:, 0, :3] = [1.0, -(1 - 2.0 ** -8), -2.0 ** -8 * (1 - 2.0 ** -8)]
    got, ref = _forward(a, dtype)
    d = a["scale"] * np.exp(np.cumsum(a["g"][:, 0]))[3:, None]
    _near(got[3:], ref[3:], 2 * d * np.abs(a["v"][0]), dtype)


@both
@wide
def test_answers_from_the_chunks_values(D, dtype):
    """o = (beta_a - beta_b) v: what tokens a and b have written has all of fp32's digits."""
    rng = np.random.default_rng(2)
    a, _ = _inputs(D, 32, rng)
    t = np.arange(T)
    a["k"][t, 0, t] = 1.0
    a["v"][:] = a["v"][0]
    a["beta"][:, 0] = 0.5 + SMALL * rng.random(T)
    a["q"][t[2:], 0, t[2:] - 1], a["q"][t[2:], 0, t[2:] - 2] = 1.0, -1.0
    got, ref = _forward(a, dtype)
    _near(got[2:], ref[2:], np.abs(a["v"][0]) * 1.0005, dtype)


def _forgotten(a, rng):
    """Token 0 writes its value under e_0, token 1 takes all but 2^-12 of it away."""
    a["k"][:2, 0, 0] = 1.0
    a["v"][1] = 0.0
    a["beta"][0], a["beta"][1] = 1.0, 1.0 - SMALL * rng.random()


@both
@wide
def test_gradients_of_queries(D, dtype):
    """dq_t along e_0: scale dO_t . (u_0 + u_1)."""
    rng = np.random.default_rng(3)
    a, do = _inputs(D, 8, rng)
    _forgotten(a, rng)
    a["scale"] = float(np.float32(0.7310586))
    got, ref = _backward(a, do, dtype)["dq"]
    _near(got[2:, 0], ref[2:, 0], 2 * a["scale"] * (np.abs(do[2:, 0]) * np.abs(a["v"][0, 0])).sum(1), dtype)


@both
@wide
def test_gradients_of_keys_from_queries(D, dtype):
    """dk_j along e_c: scale (D_ij - D_i'j) dO . u_j for queries e_c and -e_c of neighbours i, i' with one dO."""
    rng = np.random.default_rng(4)
    a, do = _inputs(D, 8, rng)
    j, pair = np.arange(32), np.arange(16)
    a["k"][j, 0, j] = 1.0
    a["beta"][j] = 1.0
    i = 32 + 2 * pair
    a["q"][i, 0, 32 + pair], a["q"][i + 1, 0, 32 + pair] = 1.0, -1.0
    do[i + 1] = do[i]
    a["g"][i + 1, 0] = -SMALL * (0.5 + 0.5 * rng.random(16))
    a["scale"] = float(np.float32(0.7310586))
    got, ref = _backward(a, do, dtype)["dk"]
    M = 2 * a["scale"] * np.abs(a["v"][j, 0]) @ np.abs(do[i, 0]).T
    _near(got[:32, 32:48], ref[:32, 32:48], M, dtype)


@both
@wide
def test_gradients_of_keys_from_earlier_keys(D, dtype):
    """dk_i along e_0: -beta_i dR_i . (u_0 + u_1), dR_i = scale dO_i."""
    rng = np.random.default_rng(5)
    a, do = _inputs(D, 8, rng)
    _forgotten(a, rng)
    t = np.arange(2, T)
    a["k"][t, 0, t], a["q"][t, 0, t] = 1.0, 1.0
    a["beta"][t, 0] = 0.5 + 0.5 * rng.random(T - 2)
    a["scale"] = float(np.float32(0.7310586))
    got, ref = _backward(a, do, dtype)["dk"]
    _near(got[2:, 0], ref[2:, 0], 2 * a["scale"] * (np.abs(do[2:, 0]) * np.abs(a["v"][0, 0])).sum(1), dtype)


@both
@wide
def test_gradients_of_keys_from_later_keys(D, dtype):
    """dk_j along e_c, which tokens i and i' = i + 1 write under: -beta' (1 - beta) scale dO_i' . u_j."""
    rng = np.random.default_rng(6)
    a, do = _inputs(D, 8, rng)
    j, pair = np.arange(32), np.arange(16)
    a["k"][j, 0, j] = 1.0
    a["beta"][j] = 1.0
    i = 32 + 2 * pair
    a["k"][i, 0, 32 + pair] = a["k"][i + 1, 0, 32 + pair] = a["k"][i + 1, 0, 48 + pair] = 1.0
    a["q"][i + 1, 0, 48 + pair] = 1.0
    a["beta"][i, 0], a["beta"][i + 1, 0] = 1.0 - SMALL * rng.random(16), 0.9 + 0.1 * rng.random(16)
    a["scale"] = float(np.float32(0.7310586))
    got, ref = _backward(a, do, dtype)["dk"]
    M = 2 * a["scale"] * np.abs(a["v"][j, 0]) @ np.abs(do[i + 1, 0]).T
    _near(got[:32, 32:48], ref[:32, 32:48], M, dtype)
