"""The bounds that the scan's oracle gives (oracle/sequence.py) tell a right result from a wrong one: in
the cases that the GPU tests compare by them (of batches of many sequences the first 200), results that are zero, have the wrong sign or lack
one of their terms are outside. The mistakes are the oracle's own results on other inputs."""
import numpy as np
import pytest

from oracle import sequence as osq
from tests import test_gpu_sequence as cases

GRADS = ["du", "ddt", "dz", "dB", "dC", "dA_log", "dD", "db_dt", "dstate"]
ROWS = ("du", "ddt", "dz", "dB", "dC", "y")


def _outside(wrong, r, name, dtype):
    """The part of the (nonzero) elements that a comparison refuses."""
    ref, bound = r[name], r["bound"][name]
    half = cases.HALF[dtype if name in ROWS else "f32"]
    tol = bound + half * (np.abs(ref) + bound) + 1e-37
    some = ref != 0
    return (np.abs(wrong[name] - ref) > tol)[some].mean() if some.any() else None


def _refuses(r, names, dtype, mistakes):
    """mistakes: (what, a wrong result, names of the outputs that show it)."""
    for name in names:
        for wrong in ({name: 0 * r[name]}, {name: -r[name]}):
            part = _outside(wrong, r, name, dtype)
            assert part is None or part > 0.95, (name, part)
    for what, wrong, shown in mistakes:
        for name in shown:
            part = _outside(wrong, r, name, dtype)
            assert part is None or part > 0, (what, name)


def _cut(offs, every=30):
    """The sequences cut every `every` tokens, as if nothing went on from one part to the next."""
    cuts = [np.arange(a, b, every) for a, b in zip(offs[:-1], offs[1:])]
    return np.concatenate(cuts + [offs[-1:]])


def _grad_case(lens, E, N, dtype, full, seed, dseed):
    a = cases._scan_case(lens, E, N, dtype, seed, full)
    rng = np.random.default_rng(dseed)
    dy = cases._round(rng.standard_normal((sum(lens), E)), dtype)
    dend = rng.standard_normal((len(lens), E, N)).astype(np.float32) if full else None
    return dict(a, dy=dy, dend=dend, offs=cases._offs(lens))


def _check_grads(k, dtype):
    r = osq.scan_backward(**k)
    wrong = lambda **kw: osq.scan_backward(**dict(k, **kw))
    m = []
    if k.get("z") is not None and len(k["u"]):
        m = [("D", wrong(D=None), ["du", "dz"]),
             ("end states' gradient", wrong(dend=None), ["du", "ddt", "dB", "dA_log", "db_dt", "dstate"]),
             ("states", wrong(state=None), ["dC", "ddt", "dz", "dA_log", "db_dt"]),
             ("bias", wrong(b_dt=None), ["du", "ddt", "dz", "dB", "dC", "dA_log", "db_dt"]),
             ("gate", wrong(z=None), ["du", "ddt", "dB", "dC", "dA_log", "dD", "db_dt"])]
    elif len(_cut(k["offs"])) > len(k["offs"]):
        m = [("what goes from part to part", wrong(offs=_cut(k["offs"])), ["du", "ddt", "dB", "dC", "dA_log", "db_dt"])]
    _refuses(r, GRADS, dtype, m)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [8, 16])
@pytest.mark.parametrize("full", [True, False])
@pytest.mark.parametrize("lens,E,ld", cases.SCAN)
def test_scan_bounds(lens, E, ld, full, N, dtype):
    _check_grads(_grad_case(lens, E, N, dtype, full, E + N + 1, E), dtype)
    a = cases._scan_case(lens, E, N, dtype, E + N, full)
    offs = cases._offs(lens)
    a["offs"] = offs
    r = osq.scan(**a)
    wrong = lambda **kw: osq.scan(**dict(a, **kw))
    m = []
    if full and sum(lens):
        m = [("D", wrong(D=None), ["y"]), ("states", wrong(state=None), ["y", "end"]),
             ("bias", wrong(b_dt=None), ["y", "end"]), ("gate", wrong(z=None), ["y"])]
    elif len(_cut(offs, 32)) > len(offs):
        m = [("what goes from part to part", wrong(offs=_cut(offs, 32)), ["y"])]
    _refuses(r, ["y", "end"], dtype, m)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_single_token_bounds(dtype):
    _check_grads(_grad_case([1] * 9, 130, 16, dtype, True, 3, 4), dtype)


@pytest.mark.parametrize("packed", [True, False])
def test_many_short_sequences_bounds(packed):
    rng = np.random.default_rng(8)
    lens = rng.integers(0, 4, 1400).tolist() if packed else [1] * 1400
    _check_grads(_grad_case(lens[:200], 1500, 16, "f32", True, 9, 8), "f32")


@pytest.mark.parametrize("N", [8, 16])
def test_bounds_by_length(N):
    lens = np.random.default_rng(18).integers(0, 31, 700).tolist()
    _check_grads(_grad_case(lens[:200], 70, N, "f32", True, 19, 18), "f32")
